"""The operators of a gated network's training step against their definitions in 64 bits.

Tolerances are bounds, element by element, worked out from the roundings that each operator makes: u is half a step of
the storage type relative to the value, 2^-24 that of fp32."""
import math

import numpy as np
import pytest
import torch

import oracle
from paper_2312_08728_b200 import operators as ops

pytestmark = pytest.mark.gpu

U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
TINY = {torch.bfloat16: 0.0, torch.float16: 2.0 ** -25, torch.float32: 0.0}  # half a step of the subnormals
E32 = 2.0 ** -24
ACTS = (ops.ACT_SILU, ops.ACT_GELU, ops.ACT_RELU, ops.ACT_SIGMOID)


# ---------------------------------------------------------------- gated block

def activation(act, g):
    """act, act' and a bound on |act''| in 64 bits."""
    if act == ops.ACT_RELU:
        return g.clamp(min=0), (g > 0).double(), 0.0
    if act == ops.ACT_GELU:
        return g * torch.special.ndtr(g), torch.special.ndtr(g) + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi), 0.8
    s = torch.sigmoid(g)
    if act == ops.ACT_SIGMOID:
        return s, s * (1 - s), 0.1
    return g * s, s + g * s * (1 - s), 0.5


class Block:
    """Inputs, 64-bit results and bounds of one block."""

    def __init__(self, rows, d, f, c, dtype, act, seed=0, extra=0, shift=0):
        gen = torch.Generator(device="cuda").manual_seed(seed)

        def make(n, k, scale):
            # rows of a wider matrix (extra), starting `shift` values into an allocation
            flat = torch.randn(shift + n * (k + extra), generator=gen, device="cuda") * scale
            return flat.to(dtype)[shift:].view(n, k + extra)[:, :k]
        self.x, self.wg, self.wu = make(rows, d, 1.0), make(d, f, d ** -0.5), make(d, f, d ** -0.5)
        self.wd, self.dy = make(f, c, f ** -0.5), make(rows, c, 0.5)
        self.act, self.dtype = act, dtype

    def reference(self):
        u, tiny = U[self.dtype], TINY[self.dtype]
        x, wg, wu, wd, dy = (t.double() for t in (self.x, self.wg, self.wu, self.wd, self.dy))
        n, (d, f), c = x.shape[0], wg.shape, wd.shape[1]
        g, up = x @ wg, x @ wu
        a, da, dda = activation(self.act, g)
        # fp32 sums: at most K roundings of partial sums bounded by the sum of magnitudes; activations in fp32: a few
        # units of 2^-24 relative, exp(-g) about |g| more, and |g| 2^-22 absolute where 1 + erf cancels
        eg, eu = d * E32 * (x.abs() @ wg.abs()), d * E32 * (x.abs() @ wu.abs())
        ea = (8 + 2 * g.abs()) * E32 * a.abs() + g.abs() * 2.0 ** -22 + (da.abs() + dda * eg) * eg
        eda = (16 + 4 * g.abs()) * E32 * (1 + g.abs()) + dda * eg
        h = a * up
        eh = a.abs() * eu + up.abs() * ea + ea * eu
        eh = eh + u * (h.abs() + eh) + tiny
        y = h @ wd
        ey = eh @ wd.abs() + f * E32 * (h.abs() @ wd.abs())
        out = {"y": (y, ey + u * (y.abs() + ey) + tiny)}
        # backward: act(G) and U act'(G) are kept in fp32; dG, dU and H are rounded
        sg, su = eg, eu
        dh = dy @ wd.T
        edh = c * E32 * (dy.abs() @ wd.abs().T)
        ea = (da.abs() + dda * sg) * sg + (8 + 2 * g.abs()) * E32 * a.abs() + g.abs() * 2.0 ** -22
        eda = (0.0 if self.act == ops.ACT_RELU else 1.0) * (dda * sg + eda)
        if self.act == ops.ACT_RELU:  # within its error of zero the sign of G, and with it act', may be either
            eda = eda + (g.abs() <= sg).double()
        du, dg, hh = dh * a, dh * up * da, a * up
        edu = (dh.abs() + edh) * ea + edh * a.abs()
        edg = (dh.abs() + edh) * (up.abs() + su) * eda + (dh.abs() + edh) * su * da.abs() + edh * up.abs() * da.abs()
        ehh = (a.abs() + ea) * su + up.abs() * ea
        edu, edg, ehh = (e + u * (v.abs() + e) * 1.01 + tiny + 4 * E32 * v.abs() for e, v in ((edu, du), (edg, dg), (ehh, hh)))

        def contraction(*terms):
            value = sum(p @ q for p, _, q in terms)
            size = sum((p.abs() + e) @ q.abs() for p, e, q in terms)
            k = sum(p.shape[1] for p, _, _ in terms)
            err = sum(e @ q.abs() for _, e, q in terms) + k * E32 * size
            return value, err + u * (value.abs() + err) + tiny
        out["dx"] = contraction((dg, edg, wg.T), (du, edu, wu.T))
        for name, v, e, left in (("dw_gate", dg, edg, x), ("dw_up", du, edu, x)):
            value, err = contraction((v.T, e.T, left))
            out[name] = (value.T, err.T)
        out["dw_down"] = contraction((hh.T, ehh.T, dy))
        return out

    def run(self, **kw):
        w = (self.wg, self.wu, self.wd)
        y, saved = ops.gated_ffn(self.x, *w, self.act, save=True, **kw)
        dx, dw_gate, dw_up, dw_down = ops.gated_ffn_backward(self.dy, self.x, *w, saved, self.act, **kw)
        return {"y": y, "dx": dx, "dw_gate": dw_gate, "dw_up": dw_up, "dw_down": dw_down}

    def check(self, got, names=("y", "dx", "dw_gate", "dw_up", "dw_down")):
        ref = self.reference()
        for k in names:
            value, bound = ref[k]
            assert got[k].dtype == self.dtype and got[k].shape == value.shape, k
            over = ((got[k].double() - value).abs() - bound * 1.0001 - 1e-30)
            worst = int(over.argmax())
            assert float(over.max()) <= 0, (k, worst, got[k].flatten()[worst].item(), value.flatten()[worst].item(),
                                            bound.flatten()[worst].item())


SHAPES = [
    (1, 8, 8, 8), (1, 64, 128, 64), (3, 1, 1, 1), (2, 17, 33, 5), (128, 64, 64, 64), (129, 65, 129, 257), (127, 200, 63, 10),
    (256, 512, 1024, 2), (300, 500, 1371, 500), (1000, 136, 264, 72), (1, 1000, 777, 1000), (64, 264, 2056, 24),
    (513, 1024, 640, 1032), (5, 2048, 4096, 2048), (17, 520, 1000, 8), (33, 4096, 264, 4104),
]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_gated_block(shape, dtype):
    b = Block(*shape, dtype, ACTS[sum(shape) % 4], seed=sum(shape))
    b.check(b.run())
    y = ops.gated_ffn(b.x, b.wg, b.wu, b.wd, b.act)  # without saving: same result up to its own bound
    b.check({"y": y}, ("y",))


@pytest.mark.parametrize("act", ACTS)
def test_gated_block_activations(act):
    b = Block(70, 96, 200, 40, torch.bfloat16, act, seed=act)
    b.check(b.run())


@pytest.mark.parametrize("extra,shift", [(8, 0), (3, 0), (0, 1), (24, 8), (1, 3)])
@pytest.mark.parametrize("rows", [1, 40, 200])
def test_gated_block_strides_and_alignment(rows, extra, shift):
    """Rows of wider matrices, and matrices that start anywhere."""
    b = Block(rows, 72, 136, 56, torch.float16, ops.ACT_SILU, seed=extra + shift, extra=extra, shift=shift)
    b.check(b.run())


@pytest.mark.parametrize("rows", [1, 100, 600])
def test_gated_block_without_the_gradient_of_the_rows(rows):
    b = Block(rows, 72, 136, 40, torch.bfloat16, ops.ACT_SILU, seed=rows)
    want = b.run()
    _, saved = ops.gated_ffn(b.x, b.wg, b.wu, b.wd, b.act, save=True)
    dx, *grads = ops.gated_ffn_backward(b.dy, b.x, b.wg, b.wu, b.wd, saved, b.act, need_dx=False)
    assert dx is None
    for g, k in zip(grads, ("dw_gate", "dw_up", "dw_down")):
        assert torch.equal(g, want[k]), k


def test_gated_block_large():
    b = Block(2304, 1024, 2816, 1024, torch.bfloat16, ops.ACT_SILU, seed=5)
    b.check(b.run())


def test_gated_block_is_reproducible_and_leaves_its_inputs():
    b = Block(777, 264, 520, 136, torch.bfloat16, ops.ACT_GELU, seed=9)
    before = [t.clone() for t in (b.x, b.wg, b.wu, b.wd, b.dy)]
    first, second = b.run(), b.run()
    for k in first:
        assert torch.equal(first[k], second[k]), k
    for t, s in zip((b.x, b.wg, b.wu, b.wd, b.dy), before):
        assert torch.equal(t, s)


def test_gated_block_without_rows():
    b = Block(0, 64, 128, 10, torch.bfloat16, ops.ACT_SILU)
    out = b.run()
    assert out["y"].shape == (0, 10) and out["dx"].shape == (0, 64)
    for k in ("dw_gate", "dw_up", "dw_down"):
        assert not out[k].any()


def test_gated_block_against_differences():
    """Directional derivatives of sum(dy * Y) in 64 bits, by central differences, against the backward pass."""
    b = Block(24, 32, 40, 16, torch.float16, ops.ACT_SILU, seed=3)
    got = b.run()
    gen = torch.Generator(device="cuda").manual_seed(1)
    tensors = {"dx": b.x, "dw_gate": b.wg, "dw_up": b.wu, "dw_down": b.wd}
    ref = b.reference()

    def value(**at):
        x, wg, wu, wd = (at.get(k, t.double()) for k, t in tensors.items())
        return float(((activation(b.act, x @ wg)[0] * (x @ wu)) @ wd * b.dy.double()).sum())
    for k, t in tensors.items():
        direction = torch.randn(t.shape, generator=gen, device="cuda", dtype=torch.float64)
        step = 1e-4
        slope = (value(**{k: t.double() + step * direction}) - value(**{k: t.double() - step * direction})) / (2 * step)
        bound = float((ref[k][1] * direction.abs()).sum())
        # the error of the central difference: step^2 times a third derivative, below 1e-4 of the sum of magnitudes here
        assert abs(float((got[k].double() * direction).sum()) - slope) <= bound + 1e-5 * float((ref[k][0] * direction).abs().sum()), k


@pytest.mark.parametrize("rows", [2, 130])
def test_gated_block_nan_stays_in_its_row(rows):
    b = Block(rows, 64, 128, 32, torch.bfloat16, ops.ACT_SILU, seed=4)
    clean = ops.gated_ffn(b.x, b.wg, b.wu, b.wd, b.act)
    b.x[1, 5] = float("nan")
    y = ops.gated_ffn(b.x, b.wg, b.wu, b.wd, b.act)
    assert torch.isnan(y[1]).all()
    assert torch.equal(y[0], clean[0]) and torch.equal(y[2:], clean[2:])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("rows,f", [(1, 40), (9, 264), (300, 136), (700, 2048)])
def test_gated_block_relu_of_minus_infinity(rows, f, dtype):
    """max(-Inf, 0) is 0: units switched off by a weight of -Inf give what they give when a finite weight does it."""
    d, c = 64, 48
    b = Block(rows, d, f, c, dtype, ops.ACT_RELU, seed=rows)
    b.x[:, 5] = 1.0
    off = torch.arange(0, f, 3, device="cuda")
    b.wg[5, off] = -1000.0
    want, y = b.run(), ops.gated_ffn(b.x, b.wg, b.wu, b.wd, b.act)
    b.wg[5, off] = -math.inf
    got = b.run()
    assert torch.equal(ops.gated_ffn(b.x, b.wg, b.wu, b.wd, b.act), y)
    others = torch.arange(d, device="cuda") != 5
    for k in ("y", "dw_gate", "dw_up", "dw_down"):
        assert torch.equal(got[k], want[k]), k
    assert torch.equal(got["dx"][:, others], want["dx"][:, others])
    assert torch.isnan(got["dx"][:, 5]).all()  # 0 times -Inf
    b.x[0, 7] = math.nan
    assert torch.isnan(ops.gated_ffn(b.x, b.wg, b.wu, b.wd, b.act)[0]).all()


@pytest.mark.parametrize("rows", [1, 9, 300])
def test_gated_block_captured_and_on_another_stream(rows):
    b = Block(rows, 128, 264, 64, torch.bfloat16, ops.ACT_SILU, seed=6)
    eager = b.run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = b.run(stream=side)
    side.synchronize()
    for k in eager:
        assert torch.equal(eager[k], other[k]), k
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = b.run()
    b.x.copy_(torch.flip(b.x, (0,)))
    graph.replay()
    torch.cuda.synchronize()
    again = b.run()
    for k in eager:
        assert torch.equal(captured[k], again[k]), k
    ops.stream_check()


def test_gated_block_calls_at_once():
    """Calls of different forms under way on three streams at the same time give what they give alone."""
    jobs = [Block(*shape, torch.bfloat16, ops.ACT_SILU, seed=i) for i, shape in
            enumerate([(3, 512, 1376, 512), (700, 256, 1024, 256), (100, 1024, 2048, 40)])]
    alone = [b.run() for b in jobs]
    streams = [torch.cuda.Stream() for _ in jobs]
    torch.cuda.synchronize()
    for _ in range(20):
        together = []
        for b, s in zip(jobs, streams):
            together.append(b.run(stream=s))
    torch.cuda.synchronize()
    for one, other in zip(alone, together):
        for k in one:
            assert torch.equal(one[k], other[k]), k
    ops.stream_check()


# ---------------------------------------------------------------- softmax residual

def residual_reference(z, y, scale):
    z = z.double()
    C = z.shape[1]
    fine = (y >= 0) & (y < C) & ~(z == -math.inf).all(dim=1)
    # relative to the row's largest logit: next to 1e38 the logarithm of a sum is lost even in 64 bits
    z = z - z.amax(dim=1, keepdim=True).clamp(min=torch.finfo(torch.float64).min)
    lse = torch.logsumexp(z, dim=1)
    one = torch.zeros_like(z)
    at = y.long().clamp(0, C - 1)
    one[torch.arange(len(y)), at] = 1.0
    r = (torch.exp(z - lse[:, None]) - one) * scale
    loss = lse - z[torch.arange(len(y)), at]
    broken = torch.isnan(lse)  # NaN, or infinity less infinity: the row has no values
    r, loss = torch.where(broken[:, None], math.nan, r), torch.where(broken, math.nan, loss)
    return torch.where(fine[:, None], r, 0.0), torch.where(fine, loss, 0.0)


def check_residual(z, y, scale=None):
    residual, loss = ops.softmax_residual(z, y, scale)
    s = 1.0 / z.shape[0] if scale is None else scale
    r, l = residual_reference(z, y, s)
    C, u = z.shape[1], U[z.dtype]
    span = (z.double().clamp(min=-1e30) - z.double().amax(dim=1, keepdim=True)).abs().clamp(max=200.0)
    # a probability: the exponential is within 2^-22 + |z - max| 2^-23 of itself; the sum of C such terms, one partial sum after
    # another in each thread, at most C 2^-24 relative in the worst order
    p = (r / s + torch.nn.functional.one_hot(y.long().clamp(0, C - 1), C)).abs()
    err = abs(s) * ((8 + 4 * span + C) * E32 * p + 2 * E32)
    bound = err + u * (r.abs() + err) + TINY[z.dtype] + 2.0 ** -126
    ok = ((residual.double() - r).abs() <= bound) | (torch.isnan(r) & torch.isnan(residual))
    assert bool(ok.all()), (residual.double() - r).abs().max()
    top = z.double().amax(dim=1).abs().clamp(max=1e30)
    lb = (C + 16) * E32 + 4 * E32 * (l.abs().clamp(max=1e30) + top)
    fine = torch.isfinite(l)
    assert bool(((loss.double() - l).abs() <= lb)[fine].all())
    assert torch.equal(torch.isnan(l), torch.isnan(loss)) and torch.equal(l == math.inf, loss == math.inf)
    return residual, loss


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16], ids=["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("rows,C", [(1, 1), (1, 2), (256, 10), (1000, 16), (7, 31), (65, 33), (3, 257), (130, 1000), (33, 1025), (5, 4097),
                                    (40, 10007), (2, 16391), (1, 40001), (9, 50257), (3, 131071),
                                    (2, 270001), (70, 35001), (3, 600011),
                                    (700, 32771), (400, 36865), (333, 53249)])
def test_residual(rows, C, dtype):
    gen = torch.Generator(device="cuda").manual_seed(rows * C)
    z = (torch.randn(rows, C, generator=gen, device="cuda") * 4).to(dtype)
    y = torch.randint(0, C, (rows,), generator=gen, device="cuda", dtype=torch.int32)
    check_residual(z, y)
    check_residual(z, y, scale=0.75)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["fp32", "bf16"])
@pytest.mark.parametrize("C", [10, 300, 5000, 70001])
def test_residual_masks_and_labels(C, dtype):
    gen = torch.Generator(device="cuda").manual_seed(C)
    z = (torch.randn(12, C, generator=gen, device="cuda") * 4).to(dtype)
    y = torch.randint(0, C, (12,), generator=gen, device="cuda", dtype=torch.int32)
    y[0], y[1], y[2] = -1, C, -2 ** 31
    z[3] = -math.inf                          # nothing left
    z[4, 1:] = -math.inf; y[4] = 0            # one class left, the label's: probability one
    z[5, : C // 2] = -math.inf                # a masked half
    y[5] = C - 1
    z[6, 0] = -math.inf; y[6] = 0             # the label itself masked: loss infinite
    z[7, C // 3] = math.nan
    z[8, C - 1] = math.inf
    z[9] = torch.finfo(dtype).min             # masked with the type's lowest value throughout
    z[10, ::2] = torch.finfo(dtype).min; y[10] = 1
    z[11] = 0.0
    residual, loss = check_residual(z, y)
    for i in (0, 1, 2, 3):
        assert not residual[i].any() and loss[i] == 0
    assert not residual[4].any() and loss[4] == 0
    assert loss[6] == math.inf and torch.isnan(residual[7]).all() and torch.isnan(residual[8]).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16], ids=["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("rows,C", [(9, 1), (9, 2), (9, 3), (9, 17), (9, 64), (9, 65), (9, 1025), (9, 40001), (64, 35001), (64, 70001), (9, 300007)])
def test_residual_rows_far_below_zero(rows, C, dtype):
    """exp(-max) overflows: threads that hold only masked logits, or none, must still count for nothing."""
    gen = torch.Generator(device="cuda").manual_seed(C)
    z = torch.randn(rows, C, generator=gen, device="cuda") * 4
    y = torch.randint(0, C, (rows,), generator=gen, device="cuda", dtype=torch.int32)
    z[0::3] -= 100.0
    z[1::3] -= 60000.0
    z[2::3] = torch.finfo(dtype).min
    if C > 2:
        z[3:, 1::2] = -math.inf
        z[6:, : C - 1] = -math.inf            # one class left, at the end of the row
    check_residual(z.to(dtype), y)


@pytest.mark.parametrize("C", [12, 1003])
def test_residual_rows_of_a_wider_matrix(C):
    z = torch.randn(37, C + 5, device="cuda", dtype=torch.bfloat16)[:, 2:C + 2]
    check_residual(z, torch.randint(0, C, (37,), device="cuda", dtype=torch.int32))


# ---------------------------------------------------------------- mini-batches

@pytest.mark.parametrize("p,dtype", [(8, torch.bfloat16), (13, torch.bfloat16), (200, torch.float32), (7, torch.uint8)])
def test_gather_batch_takes_the_rows_of_the_shuffle(p, dtype):
    rows = 1013
    x = torch.arange(rows * p, device="cuda").remainder(251).to(dtype).view(rows, p)
    y = torch.arange(rows, device="cuda", dtype=torch.int32)
    pi = torch.from_numpy(oracle.perm(77, 2, 5, rows).astype(np.int64)).cuda()
    bx, by = ops.gather_batch(x, y, 77, 2, 5, 100, 300)
    assert torch.equal(by.long(), pi[100:400]) and torch.equal(bx, x[pi[100:400]])
    bx, by = ops.gather_batch(x, None, 77, 2, 5, 1000, 13)
    assert by is None and torch.equal(bx, x[pi[1000:]])
    assert ops.gather_batch(x, y, 77, 2, 5, rows, 0)[0].shape == (0, p)


# ---------------------------------------------------------------- refusals that need device tensors

def test_refusals():
    b = Block(6, 16, 24, 8, torch.bfloat16, ops.ACT_SILU)
    w = [b.wg, b.wu, b.wd]
    y, saved = ops.gated_ffn(b.x, *w, save=True)

    def backward(dy=b.dy, saved=saved):
        return ops.gated_ffn_backward(dy, b.x, *w, saved)
    calls = [
        lambda: ops.gated_ffn(b.x.float(), *w), lambda: ops.gated_ffn(b.x.half(), *w), lambda: ops.gated_ffn(b.x.cpu(), *w),
        lambda: ops.gated_ffn(b.x[:, :8], *w), lambda: ops.gated_ffn(b.x, b.wg, b.wu[:, :16], b.wd), lambda: ops.gated_ffn(b.x, b.wg, b.wu, b.wd[:16]),
        lambda: ops.gated_ffn(b.x.t().contiguous().t(), *w), lambda: ops.gated_ffn(b.x, *w, activation=9),
        lambda: ops.gated_ffn(b.x, b.wg.cpu(), b.wu, b.wd), lambda: ops.gated_ffn(b.x[0], *w), lambda: ops.gated_ffn(b.x, b.wg[:, :0], b.wu[:, :0], b.wd[:0]),
        lambda: backward(dy=b.dy[:, :4]), lambda: backward(dy=b.dy[:3]), lambda: backward(dy=b.dy.float()), lambda: backward(saved=y),
        lambda: backward(saved=saved[:5]), lambda: backward(saved=saved[:, :24]), lambda: backward(saved=saved.half()), lambda: backward(saved=saved.cpu()),
        lambda: ops.softmax_residual(y, torch.zeros(6, dtype=torch.int64, device="cuda")), lambda: ops.softmax_residual(y, torch.zeros(5, dtype=torch.int32, device="cuda")),
        lambda: ops.softmax_residual(y, torch.zeros(6, dtype=torch.int32)), lambda: ops.softmax_residual(y.double(), torch.zeros(6, dtype=torch.int32, device="cuda")),
        lambda: ops.gather_batch(b.x, None, 0, 0, 0, 3, 4), lambda: ops.gather_batch(b.x[:, :8], None, 0, 0, 0, 0, 1), lambda: ops.gather_batch(b.x, None, 0, 0, 0, -1, 1),
    ]
    for k, call in enumerate(calls):
        with pytest.raises(ValueError):
            call()
            raise AssertionError(f"call {k} was not refused")
