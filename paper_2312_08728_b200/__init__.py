"""B200-native buffered mini-batch gradient descent (BMGD).

The computation runs in a CUDA library (csrc/, C ABI in include/bmgd.h); `binding`
wraps it with ctypes, `operators` holds the parts of a training step of a gated network
(the block with its backward pass, the softmax residual, AdamW), `network` the model
trained with them, `inputs` draws the seeded synthetic workloads, `build` compiles the
library in-tree with nvcc.
"""
from . import inputs  # noqa: F401
from .inputs import WORKLOADS, Workload, buffer_seed  # noqa: F401


def __getattr__(name):
    # the binding loads (and if need be builds) the CUDA library: only on first use
    if name in ("Bmgd", "BmgdError", "load_library", "binding"):
        import importlib
        binding = importlib.import_module(__name__ + ".binding")
        return binding if name == "binding" else getattr(binding, name)
    if name in ("operators", "network", "GatedSoftmax"):
        import importlib
        module = importlib.import_module(__name__ + (".operators" if name == "operators" else ".network"))
        return getattr(module, name) if name == "GatedSoftmax" else module
    raise AttributeError(name)
