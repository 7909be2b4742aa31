"""The gated block's GELU far below zero: (act(x Wg) * (x Wu)) Wd with every gate between -7 and -4, and its slope.

The inputs are chosen so that nothing but the activation is rounded before the block's own roundings: one input of 1, gates and factors that the type holds, and
an identity behind them."""
import math

import pytest
import torch

from paper_2312_08728_b200 import operators as ops
from test_gpu_gates import gated, relative
from test_gpu_norm import inside
from test_gpu_operators import E32, TINY, U

pytestmark = pytest.mark.gpu

DTYPES = [torch.bfloat16, torch.float16]
NAMES = ["bf16", "fp16"]


# the form for few rows and the one for many
@pytest.mark.parametrize("dtype", DTYPES, ids=NAMES)
@pytest.mark.parametrize("rows,hidden", [(1, 64), (40, 264), (2100, 640)])
@pytest.mark.parametrize("save", [False, True])
def test_gelu(rows, hidden, save, dtype):
    x = torch.zeros(rows, 16, device="cuda", dtype=dtype)
    x[:, 0] = 1
    gates = torch.linspace(-7.0, -4.0, hidden, device="cuda").to(dtype)
    wg, wu = torch.zeros(16, hidden, device="cuda", dtype=dtype), torch.zeros(16, hidden, device="cuda", dtype=dtype)
    wg[0], wu[0] = gates, 4096.0
    wd = torch.eye(hidden, device="cuda", dtype=dtype)
    y = ops.gated_ffn(x, wg, wu, wd, ops.ACT_GELU, save=save)
    y, saved = y if save else (y, None)
    g = gates.double()
    value = gated(ops.ACT_GELU, g)
    slope = value / g + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
    want = value * 4096.0
    u, tiny = U[dtype], TINY[dtype]
    rel = relative(ops.ACT_GELU, g) + 2 * E32
    bound = ((1 + rel) * (1 + u) ** 2 - 1) * want.abs() + 2 * tiny      # rounded as the hidden value and as the result
    inside(y, want.expand_as(y), bound.expand_as(y).contiguous(), "y")
    if not save:
        return
    # dWg[0] = sum over the rows of dH u act'(g): with one row's gradient a one-hot, each weight gets its own slope
    dy = torch.zeros(rows, hidden, device="cuda", dtype=dtype)
    dy[0] = 1
    _, dwg, _, _ = ops.gated_ffn_backward(dy, x, wg, wu, wd, saved, ops.ACT_GELU)
    want = slope * 4096.0
    # act' = Phi(g) + g phi(g): a density of e^(-g^2 / 2), whose exponent is rounded, and a tail of at most 1 / g^2 of it
    rel = (16 + 4 * g.square()) * E32
    bound = ((1 + rel) * (1 + u) ** 2 - 1) * want.abs() + 2 * tiny
    inside(dwg[0], want, bound, "slope")
