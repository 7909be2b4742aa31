"""Bounds on the operators' sums that do not grow with the worst order of a long sum: a piece of a row left out of a softmax,
or bits lost in a contraction, would pass the element-wise worst cases and fails here."""
import math

import pytest
import torch

from paper_2312_08728_b200 import operators as ops
from test_gpu_operators import ACTS, E32, SHAPES, TINY, U, Block, activation, residual_reference

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.bfloat16, torch.float16]
NAMES = ["fp32", "bf16", "fp16"]


# ---------------------------------------------------------------- softmax residual

def threads(C, dtype):
    """Fewest threads that share a row of C logits."""
    pieces = -(-C * dtype.itemsize // 16)
    return 2 if C <= 64 else 32 if pieces <= 256 else 128 if pieces <= 1024 else 256


def check(z, y, scale):
    """In units of 2^-24, relative: a term exp(z - max) is 8 + 4 |z - max| off; the sum the average of that over its terms, at most
    8 + 4 log C, and one unit for each term that a thread adds and for each of the joins, of which there are fewer than 64."""
    residual, loss = ops.softmax_residual(z, y, scale)
    r, l = residual_reference(z, y, scale)
    C = z.shape[1]
    one = torch.nn.functional.one_hot(y.long(), C).double()
    p = r / scale + one
    zd = z.double()
    top = zd.amax(dim=1, keepdim=True)
    total = (8 + 4 * math.log(C) + C / threads(C, z.dtype) + 64) * E32
    err = abs(scale) * (p * ((12 + 4 * (top - zd)) * E32 + total) + 2 * E32 * one)
    bound = err + U[z.dtype] * (r.abs() + err) + TINY[z.dtype] + 2.0 ** -126
    over = (residual.double() - r).abs() - bound
    assert float(over.max()) <= 0, float(over.max())
    # the largest less the label's logit and log of the sum, each rounded, and their sum
    at_label = top.squeeze(1) - zd.gather(1, y.long()[:, None]).squeeze(1)
    over = (loss.double() - l).abs() - (total + 4 * E32 * (l.abs() + at_label + math.log(C)))
    assert float(over.max()) <= 0, float(over.max())


ROWS = [(1, 2), (256, 10), (7, 31), (65, 33), (3, 257), (130, 1000), (33, 1025), (5, 4097), (40, 10007), (2, 16391), (1, 40001), (9, 50257),
        (3, 131071), (2, 270001), (70, 35001), (3, 600011), (400, 36865)]


@pytest.mark.parametrize("dtype", TYPES, ids=NAMES)
@pytest.mark.parametrize("rows,C", ROWS)
def test_residual(rows, C, dtype):
    gen = torch.Generator(device="cuda").manual_seed(rows + C)
    z = (torch.randn(rows, C, generator=gen, device="cuda") * 4).to(dtype)
    check(z, torch.randint(0, C, (rows,), generator=gen, device="cuda", dtype=torch.int32), 1.0)


@pytest.mark.parametrize("dtype", TYPES, ids=NAMES)
@pytest.mark.parametrize("rows,C", ROWS)
def test_residual_of_equal_logits(rows, C, dtype):
    """Every exponential is 1 and every partial sum a whole number below 2^24, so the sum is C without error: what is left are the
    roundings of its logarithm (2 units of 2^-24), of 1 / C and of the product."""
    for value in (0.0, -7.5):
        z = torch.full((rows, C), value, device="cuda", dtype=dtype)
        y = torch.arange(rows, device="cuda", dtype=torch.int32) * 7919 % C
        residual, loss = ops.softmax_residual(z, y, 1.0)
        assert bool(((loss.double() - math.log(C)).abs() <= 4 * E32 * math.log(C)).all())
        want = torch.full((rows, C), 1.0 / C, device="cuda", dtype=torch.float64) - torch.nn.functional.one_hot(y.long(), C).double()
        bound = want.abs() * (U[dtype] + 6 * E32) + TINY[dtype]
        assert bool(((residual.double() - want).abs() <= bound).all())


@pytest.mark.parametrize("dtype", TYPES, ids=NAMES)
@pytest.mark.parametrize("rows,C,shift", [(24, 10, 0), (24, 33, 1), (24, 1000, 3), (24, 4097, 1), (24, 16391, 0), (24, 40001, 1), (24, 131071, 0), (60, 40001, 1),
                                          (60, 131071, 3), (60, 300007, 1)])
def test_residual_sees_every_place(rows, C, dtype, shift):
    """One logit of 20 among zeros, each row with another place for it: the first and last ones, on either side of the 16-byte
    boundaries, and a spread over all threads, blocks and turns; left out of the maximum or the sum it would change the loss by about 20."""
    ends = [k for k in list(range(10)) + list(range(C - 10, C)) if 0 <= k < C]
    gen = torch.Generator().manual_seed(C)
    places = torch.tensor((ends + torch.randint(0, C, (8 * rows,), generator=gen).tolist())[:8 * rows], device="cuda")
    for part in places.split(rows):
        n = len(part)
        z = torch.zeros(n * C + shift, device="cuda", dtype=dtype)[shift:].view(n, C)
        z[torch.arange(n, device="cuda"), part] = 20.0
        check(z, ((part + C // 2 + 1) % C).int(), 1.0)
        check(z, part.int(), 1.0)


# ---------------------------------------------------------------- gated block

def largest(a):
    """Largest singular value."""
    a = a if a.shape[0] >= a.shape[1] else a.T
    return float(torch.linalg.eigvalsh(a.T @ a)[-1].clamp(min=0).sqrt())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("shape", [s for s in SHAPES if s[1] > 1], ids=lambda s: "x".join(map(str, s)))
def test_block_as_a_whole(shape, dtype):
    """Norms of the errors.  An operand rounded by u of each value moves a product by at most u times its norm times the other's largest
    singular value; the result is rounded by u.  A sum of K products on the tensor cores is added up 16 at a time, each partial
    sum cut off by at most 2^-23 of itself: K / 16 times that of the norm where terms are random, 8 times as much allowed."""
    b = Block(*shape, dtype, ACTS[(sum(shape) + 1) % 4], seed=sum(shape))
    got = b.run()
    x, wg, wu, wd, dy = (t.double() for t in (b.x, b.wg, b.wu, b.wd, b.dy))
    n, d, f, c = shape
    g, up = x @ wg, x @ wu
    a, da, _ = activation(b.act, g)
    h, dh = a * up, dy @ wd.T
    du, dg = dh * a, dh * up * da
    u, tiny = U[dtype], TINY[dtype]
    size = torch.linalg.norm
    # a factor's own error: that of G and U, of dH, and of the activation (units of 2^-24, see the element-wise bounds)
    first = (d + 64) * E32
    second = (d + c + 64) * E32

    def near(k, value, terms, K):
        err = float(size(got[k].double() - value))
        lost = tiny * math.sqrt(value.numel())
        bound = sum((u + e) * float(size(p)) * largest(q) + tiny * math.sqrt(p.numel()) * largest(q) for p, e, q in terms)
        bound += (u + K * E32) * float(size(value)) + lost
        assert err <= bound, (k, err / float(size(value)), bound / float(size(value)))
    near("y", h @ wd, [(h, first, wd)], f)
    near("dx", dg @ wg.T + du @ wu.T, [(dg, second, wg), (du, second, wu)], 2 * f)
    near("dw_gate", x.T @ dg, [(dg, second, x)], n)
    near("dw_up", x.T @ du, [(du, second, x)], n)
    near("dw_down", h.T @ dy, [(h, first, dy)], n)


@pytest.mark.parametrize("rows", [5, 200, 1500])
@pytest.mark.parametrize("act", ACTS)
def test_activations_value_by_value(act, rows):
    """G = g, U = 1 and Wd = 1 exactly, so Y is act(g) rounded, and what the forward pass saves is act(g) and act'(g) in fp32.  In units
    of 2^-24: exp(-g) is off by 2 (3 + 1.2 |g|) at most, a quotient by 4, further operations by 1 each; where 1 + erf cancels, GELU is
    off by |g| 2^-22."""
    f = 8
    gen = torch.Generator(device="cuda").manual_seed(rows)
    g = ((torch.rand(rows, generator=gen, device="cuda") * 40 - 20)).bfloat16()
    g[0] = 0.0
    x = torch.stack([g, torch.ones_like(g)], dim=1)
    gate, up = torch.zeros(2, f, device="cuda", dtype=torch.bfloat16), torch.zeros(2, f, device="cuda", dtype=torch.bfloat16)
    gate[0], up[1] = 1.0, 1.0
    y, saved = ops.gated_ffn(x, gate, up, torch.eye(f, device="cuda", dtype=torch.bfloat16), act, save=True)
    flat = saved.view(-1).view(torch.float32)
    value, slope = (flat[k * rows * f:(k + 1) * rows * f].view(rows, f).double() for k in (0, 1))
    gd = g.double()
    a, da, _ = activation(act, gd)
    unit = (16 + 4 * gd.abs()) * E32
    if act == ops.ACT_RELU:
        ea, eda = 0 * a, 0 * a
    elif act == ops.ACT_SIGMOID:
        ea, eda = unit * a, unit * da + a * (unit * a + E32)
    elif act == ops.ACT_SILU:
        s = torch.sigmoid(gd)
        ea, eda = unit * a.abs(), unit * da.abs() + s * gd.abs() * (unit * s + E32) + 4 * unit * s
    else:
        ea = unit * a.abs() + gd.abs() * 2.0 ** -22
        eda = unit * (1 + gd.abs() * torch.exp(-gd * gd / 2)) * 2 + gd.abs() * torch.exp(-gd * gd / 2) * gd * gd * E32
    ea, eda, a, da = (t[:, None] for t in (ea, eda, a, da))
    assert float(((value - a).abs() - ea - 2.0 ** -126).max()) <= 0
    assert float(((slope - da).abs() - eda - 2.0 ** -126).max()) <= 0
    u = U[torch.bfloat16]
    assert float(((y.double() - a).abs() - (ea + u * (a.abs() + ea)) * 1.0001 - 2.0 ** -133).max()) <= 0
