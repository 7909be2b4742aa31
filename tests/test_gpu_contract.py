"""What every operator's call keeps to: tangents of forward-mode differentiation are refused, not dropped; outputs are what torch itself would allocate."""
import gc

import pytest
import torch
from torch.autograd import forward_ad

from paper_2312_08728_b200 import operators as ops

pytestmark = pytest.mark.gpu


def test_tangents_are_refused():
    x, w = torch.randn(4, 16, device="cuda"), torch.randn(16, device="cuda")
    q, qs = ops.quantize_rows(x)
    b, m = x.bfloat16(), torch.randn(16, 16, device="cuda").bfloat16()
    calls = [
        (lambda t: ops.rms_norm(t, w), x), (lambda t: ops.rms_norm(x, t), w), (lambda t: ops.rms_norm(x, w, residual=t), x), (lambda t: ops.rms_norm_int8(t, w), x),
        (lambda t: ops.quantize_rows(t), x), (lambda t: ops.quantize_rows(x, gate=t), x), (lambda t: ops.int8_linear(q, t, q, qs), qs), (lambda t: ops.log_probs(t), x),
        (lambda t: ops.dropout(t, 0.5, 1), x), (lambda t: ops.dropout(x, 0.5, 1, residual=t), x), (lambda t: ops.gated_ffn(t, m, m, m), b), (lambda t: ops.gated_ffn(b, m, m, t), m),
    ]
    for k, (call, t) in enumerate(calls):
        call(t)
        with forward_ad.dual_level():
            call(t)                                     # (no tangent of its own: taken)
            dual = forward_ad.make_dual(t, torch.ones_like(t))
            for context in (torch.enable_grad(), torch.no_grad()):
                with context, pytest.raises(ValueError, match="graph"):
                    call(dual)
                    pytest.fail(f"call {k} was taken")
            call(forward_ad.unpack_dual(dual).primal)


@pytest.mark.parametrize("size,stride,dtype", [((5, 7), (7, 1), torch.bfloat16), ((5, 7), (16, 1), torch.int8), ((3,), (1,), torch.float32), ((0, 4), (4, 1), torch.float16),
                                               ((6, 0), (1, 1), torch.int32), ((9,), (1,), torch.uint8)])
def test_outputs_are_torchs_own(size, stride, dtype):
    """The short way to an output's memory, and the long one."""
    got, want = ops._strided(size, stride, dtype), torch.empty_strided(size, stride, dtype=dtype, device="cuda")
    assert (got.shape, got.stride(), got.dtype, got.device, got.storage_offset()) == (want.shape, want.stride(), want.dtype, want.device, want.storage_offset())
    assert got.untyped_storage().nbytes() == want.untyped_storage().nbytes() and not got.requires_grad
    gc.collect()
    before = torch.cuda.memory_allocated()
    big = ops._strided((1 << 20,), (1,), torch.float32)
    assert torch.cuda.memory_allocated() - before >= 4 << 20        # from the allocator that torch counts
    del big
    assert torch.cuda.memory_allocated() == before
