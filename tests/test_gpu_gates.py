"""Gates far below zero, where an activation is a small difference of large numbers unless it is computed as a tail.

Bounds, relative to act(g).  GELU, as g e^(-g^2 / 2) R(|g|): the exponent is rounded in three places (2 g^2 E32 at most), the exponential is good to 4 E32, the ratio R to 7 E32 and
the reciprocal inside it to 2, three products more; above zero 1 less that, half as much.  SiLU, sigmoid: an exponential of -g, off by 2 |g| E32, and a reciprocal.  Every row
is held to its own bound."""
import math

import pytest
import torch

from paper_2312_08728_b200 import operators as ops
from test_gpu_norm import inside, rows_of
from test_gpu_operators import ACTS, E32, activation

pytestmark = pytest.mark.gpu

DTYPES = [torch.bfloat16, torch.float16, torch.float32]
NAMES = ["bf16", "fp16", "fp32"]
ACT_NAMES = ["silu", "gelu", "relu", "sigmoid"]


def gated(act, g):
    """act(g) in 64 bits, GELU by its tail there too."""
    return 0.5 * g * torch.special.erfc(-g / math.sqrt(2)) if act == ops.ACT_GELU else activation(act, g)[0]


def relative(act, g):
    if act == ops.ACT_GELU:
        return (16 + 2 * g.clamp(max=0).square()) * E32
    return 0.0 * g if act == ops.ACT_RELU else (8 + 2 * g.abs()) * E32


def check_rows(x, gate, act):
    """quantize_rows against 64 bits, with a bound for each row: that of its own values, as a share of its own largest."""
    codes, scale = ops.quantize_rows(x, gate=gate, activation=act)
    g = gate.double()
    h = gated(act, g) * x.double()
    top = h.abs().amax(dim=1)
    some = top >= 2.0 ** -119
    share = ((relative(act, g) + 2 * E32) * h.abs()).amax(dim=1) / top.clamp(min=2.0 ** -119)
    assert float(share.max()) < 2.0 ** -15, "the bound would hide errors"
    inside(scale[some], top[some] / 127, (share[some] + 2 * E32) * top[some] / 127, "scale")
    exact = h[some] * (127.0 / top[some])[:, None]
    inside(codes[some], exact, (0.5 + 127 * (2 * share[some] + 4 * E32))[:, None].expand_as(exact), "codes")
    assert bool((codes[some].int().abs().amax(dim=1) == 127).all())
    none = top < 2.0 ** -121
    assert not scale[none].any() and not codes[none].any()


# a warp's rows, blocks with two, four and six pieces a thread, rows on any boundary, rows read twice
WIDTHS = [1, 2, 7, 8, 64, 100, 501, 768, 6144, 11008, 11007, 20000, 40000]


@pytest.mark.parametrize("dtype", DTYPES, ids=NAMES)
@pytest.mark.parametrize("act", ACTS, ids=ACT_NAMES)
@pytest.mark.parametrize("width", WIDTHS)
def test_rows_in_8_bits(width, act, dtype):
    gen = torch.Generator(device="cuda").manual_seed(width + act)
    for n, extra, shift in ((1, 0, 0), (45, 0, 0), (20, 3, 1)):
        x = rows_of(gen, n, width, dtype, extra, shift)
        check_rows(x, rows_of(gen, n, width, dtype, extra, shift, scale=2.0), act)
        if act == ops.ACT_RELU:
            continue
        # every gate of a row between -8 and -4
        gate = (torch.rand(n, width + extra, generator=gen, device="cuda") * 4 - 8).to(dtype)[:, :width]
        check_rows(x, gate, act)


@pytest.mark.parametrize("dtype", DTYPES, ids=NAMES)
def test_one_gate_a_row(dtype):
    """Each row is one value: its code is 127 of its sign, its scale says how far off act(g) is."""
    gate = torch.linspace(-12.0, 6.0, 1801, device="cuda").to(dtype)[:, None].contiguous()
    x = torch.where(torch.arange(1801, device="cuda") % 2 == 0, 1.5, -3.0).to(dtype)[:, None].contiguous()
    for act in (ops.ACT_SILU, ops.ACT_GELU, ops.ACT_SIGMOID):
        kept = gate[:, 0] != 0 if act != ops.ACT_SIGMOID else gate[:, 0] == gate[:, 0]
        check_rows(x[kept], gate[kept], act)


@pytest.mark.parametrize("dtype", DTYPES, ids=NAMES)
def test_gates_of_infinity(dtype):
    """gelu(inf) = inf, and where 0 meets infinity NaN: either way the row's scale is NaN and its codes are 0, and the others' are not touched."""
    gate = torch.randn(4, 40, device="cuda").to(dtype)
    gate[0, 3], gate[1, 5], gate[2, 7] = float("inf"), float("-inf"), float("nan")
    for act in (ops.ACT_SILU, ops.ACT_GELU):
        codes, scale = ops.quantize_rows(torch.ones_like(gate), gate=gate, activation=act)
        assert bool(torch.isnan(scale[:3]).all()) and not codes[:3].any() and bool(torch.isfinite(scale[3])) and int(codes[3].abs().max()) == 127
