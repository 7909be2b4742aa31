"""The norm with the residual's addition and rows in 8 bits against their definitions in 64 bits.

Tolerances are bounds, element by element: u is half a step of the storage type relative to the value, E32 that of fp32.  A sum over a
row of `width` values has at most width / 128 + 64 additions in a row (what a thread adds up by itself, lanes, warps)."""
import pytest
import torch

from paper_2312_08728_b200 import operators as ops
from test_gpu_operators import E32, TINY, U, activation

pytestmark = pytest.mark.gpu

DTYPES = [torch.bfloat16, torch.float16, torch.float32]
NAMES = ["bf16", "fp16", "fp32"]
EPS = 1e-5


def rows_of(gen, n, d, dtype, extra=0, shift=0, scale=1.0):
    """[n, d], rows of a wider matrix (extra), starting `shift` values into an allocation."""
    flat = torch.randn(shift + n * (d + extra), generator=gen, device="cuda") * scale
    return flat.to(dtype)[shift:].view(n, d + extra)[:, :d]


def inside(got, want, bound, what):
    over = (got.double() - want).abs() - bound * 1.0001 - 1e-30
    assert bool((over <= 0).all()), (what, float(over.max()), int(over.argmax()))


def check_total(total, x, r):
    if r is None:
        assert total is x
        return
    want = x.double() + r.double()
    u, tiny = U[x.dtype], TINY[x.dtype]
    inside(total, want, (u * (1 + E32) + E32) * want.abs() + tiny, "total")


def root_error(width):
    """Relative error of 1 / sqrt(mean + eps): half that of the sum, and of the root's approximation."""
    return ((width / 128 + 64) / 2 + 8) * E32


def normed(total, w):
    t = total.double()
    s = 1.0 / torch.sqrt(t.square().mean(dim=1, keepdim=True) + EPS)
    return t * s * (1.0 if w is None else w.double()), s


def check_codes(codes, scale, y, rel):
    """codes and scale of rows whose values are known within `rel` of their row's largest."""
    top = y.abs().amax(dim=1)
    some = top >= 2.0 ** -119
    assert codes.dtype == torch.int8 and scale.dtype == torch.float32
    inside(scale[some], top[some] / 127, (rel + 2 * E32) * top[some] / 127, "scale")
    exact = y[some] * (127.0 / top[some])[:, None]
    inside(codes[some], exact, torch.full_like(exact, 0.5 + 127 * (2 * rel + 4 * E32)), "codes")
    none = top < 2.0 ** -121
    assert not scale[none].any() and not codes[none].any()


def check_norm(x, w, r, save=True, **kw):
    y, total, rstd = ops.rms_norm(x, w, residual=r, eps=EPS, save=True, **kw)
    check_total(total, x, r)
    want, s = normed(total, w)
    u, tiny, rel = U[x.dtype], TINY[x.dtype], root_error(x.shape[1])
    inside(rstd, s.squeeze(1), rel * s.squeeze(1), "rstd")
    inside(y, want, ((rel + 3 * E32) * (1 + u) + u) * want.abs() + tiny, "y")
    q, scale, total2 = ops.rms_norm_int8(x, w, residual=r, eps=EPS, **kw)
    assert torch.equal(total2, total)
    check_codes(q, scale, want, rel + 3 * E32)
    return y, total, rstd


def check_backward(dy, total, w, rstd, dtotal):
    dx, dw = ops.rms_norm_backward(dy, total, w, rstd, dtotal)
    n, d = total.shape
    t, s, g0 = total.double(), rstd.double()[:, None], dy.double()
    g = g0 if w is None else g0 * w.double()
    mean = (g * t * s).mean(dim=1, keepdim=True)
    want = s * (g - t * s * mean)
    e_mean = (d / 128 + 80) * E32 * (g * t * s).abs().mean(dim=1, keepdim=True)
    e = s * (4 * E32 * g.abs() + (t * s).abs() * (e_mean + 4 * E32 * mean.abs()))
    if dtotal is not None:
        want = want + dtotal.double()
        e = e + E32 * (want.abs() + e)
    u, tiny = U[total.dtype], TINY[total.dtype]
    inside(dx, want, e + u * (want.abs() + e) + tiny, "dx")
    if w is None:
        assert dw is None
        return
    assert dw.dtype == w.dtype
    want, size = (g0 * t * s).sum(dim=0), (g0 * t * s).abs().sum(dim=0)
    e = (n + 64) * E32 * size
    inside(dw, want, e + U[w.dtype] * (want.abs() + e) + TINY[w.dtype], "dw")


# widths of every form: single values, a warp's row, blocks with two and four pieces a thread, rows read more than once
WIDTHS = [1, 2, 7, 8, 16, 31, 100, 256, 264, 501, 512, 1000, 2048, 2056, 4095, 4096, 8192, 11008]


@pytest.mark.parametrize("dtype", DTYPES, ids=NAMES)
@pytest.mark.parametrize("width", WIDTHS)
def test_norm(width, dtype):
    gen = torch.Generator(device="cuda").manual_seed(width)
    for n, wtype, with_r in ((3, dtype, True), (70, torch.float32, False), (1, torch.float32, True), (33, None, True)):
        x, r = rows_of(gen, n, width, dtype), rows_of(gen, n, width, dtype, scale=3.0) if with_r else None
        w = None if wtype is None else (1 + 0.3 * torch.randn(width, generator=gen, device="cuda")).to(wtype)
        _, total, rstd = check_norm(x, w, r)
        dy = rows_of(gen, n, width, dtype, scale=0.3)
        check_backward(dy, total, w, rstd, rows_of(gen, n, width, dtype) if with_r else None)


@pytest.mark.parametrize("dtype,width", [(torch.bfloat16, 16392), (torch.float16, 20001), (torch.float32, 9000), (torch.bfloat16, 40000),
                                         (torch.float32, 60004), (torch.bfloat16, 33000)])
def test_long_rows(dtype, width):
    gen = torch.Generator(device="cuda").manual_seed(width)
    x, r, dy = (rows_of(gen, 5, width, dtype) for _ in range(3))
    w = 1 + 0.3 * torch.randn(width, generator=gen, device="cuda")
    _, total, rstd = check_norm(x, w, r)
    check_backward(dy, total, w, rstd, r)
    check_backward(dy, total, None, rstd, None)


@pytest.mark.parametrize("dtype", DTYPES, ids=NAMES)
@pytest.mark.parametrize("width,extra,shift", [(512, 1, 0), (512, 8, 3), (501, 11, 0), (501, 0, 5), (4096, 8, 0), (4096, 2, 1), (13, 3, 2)])
def test_strides_and_boundaries(width, extra, shift, dtype):
    gen = torch.Generator(device="cuda").manual_seed(width + extra)
    x, r = rows_of(gen, 37, width, dtype, extra, shift), rows_of(gen, 37, width, dtype, 0, shift + 1)
    w = torch.randn(width + 3, generator=gen, device="cuda")[3:]
    _, total, rstd = check_norm(x, w, r)
    check_norm(x, w, None)
    check_backward(rows_of(gen, 37, width, dtype, extra, 1), total, w, rstd, rows_of(gen, 37, width, dtype, extra + 1, shift))
    check_backward(rows_of(gen, 37, width, dtype, extra, 1), x, w, rstd, None)


def test_many_rows_give_equal_bits():
    """More rows than blocks; the weight's gradient is a sum in a fixed order."""
    gen = torch.Generator(device="cuda").manual_seed(4)
    for width in (64, 300, 768, 4096):
        x, r, dy = (rows_of(gen, 9000, width, torch.bfloat16) for _ in range(3))
        w = 1 + 0.1 * torch.randn(width, generator=gen, device="cuda")
        y, total, rstd = check_norm(x, w, r)
        check_backward(dy, total, w, rstd, r)
        first = ops.rms_norm_backward(dy, total, w, rstd, r)
        for _ in range(3):
            again = ops.rms_norm_backward(dy, total, w, rstd, r)
            assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


@pytest.mark.parametrize("dtype", DTYPES, ids=NAMES)
@pytest.mark.parametrize("width", [24, 4096, 501, 40000])
def test_rows_of_zeros_infinities_and_nan(width, dtype):
    x = torch.randn(6, width, device="cuda").to(dtype)
    x[0] = 0
    x[1, width // 2] = float("inf")
    x[2, 3] = float("nan")
    x[3, -1] = float("-inf")
    w = torch.ones(width, device="cuda")
    y, _, rstd = ops.rms_norm(x, w, eps=EPS, save=True)
    assert not y[0].any() and bool(torch.isnan(y[2]).all())
    for row, at in ((1, width // 2), (3, width - 1)):       # 1 / sqrt(Inf) is 0, and 0 times Inf NaN
        assert rstd[row] == 0 and bool(torch.isnan(y[row, at])) and int(torch.isnan(y[row]).sum()) == 1
    codes, scale, _ = ops.rms_norm_int8(x, w, eps=EPS)
    assert scale[0] == 0 and not codes[0].any()
    for row in (1, 2, 3):
        assert bool(torch.isnan(scale[row])) and not codes[row].any()
    for row in (4, 5):
        assert bool(torch.isfinite(scale[row])) and int(codes[row].abs().max()) == 127
    y0, _, _ = ops.rms_norm(x[:1], w, eps=0.0, save=True)
    assert bool(torch.isnan(y0).all())                      # 0 / 0


def test_nothing_and_one():
    for dtype in DTYPES:
        x = torch.randn(0, 40, device="cuda").to(dtype)
        w = torch.ones(40, device="cuda")
        y, total, rstd = ops.rms_norm(x, w, residual=x, save=True)
        assert y.shape == (0, 40) and total.shape == (0, 40) and rstd.shape == (0,)
        dx, dw = ops.rms_norm_backward(y, total, w, rstd, total)
        assert dx.shape == (0, 40) and dw.shape == (40,) and not dw.any()
        q, scale, _ = ops.rms_norm_int8(x, w)
        assert q.shape == (0, 40) and scale.shape == (0,)


def test_the_gradient_against_differences():
    """Along random directions, in fp32.  The sum over all values of dy y is differentiable; central differences with step h are off by
    h^2 / 6 times its third derivative (below 30 here) and by rounding, 2^-24 of the terms over h."""
    gen = torch.Generator(device="cuda").manual_seed(8)
    x, dy, r = (torch.randn(9, 70, generator=gen, device="cuda") for _ in range(3))
    w = 1 + 0.3 * torch.randn(70, generator=gen, device="cuda")
    dtotal = torch.randn(9, 70, generator=gen, device="cuda")
    _, total, rstd = ops.rms_norm(x, w, residual=r, eps=EPS, save=True)
    dx, dw = ops.rms_norm_backward(dy, total, w, rstd, dtotal)

    def value(x, w):
        y, total = ops.rms_norm(x, w, residual=r, eps=EPS)
        return float((y.double() * dy.double()).sum() + (total.double() * dtotal.double()).sum())
    h = 2.0 ** -7
    for _ in range(5):
        v, a = torch.randn(9, 70, generator=gen, device="cuda"), torch.randn(70, generator=gen, device="cuda")
        along = (value(x + h * v, w) - value(x - h * v, w)) / (2 * h)
        terms = float((dy.abs() * 4).sum() + (total * dtotal).abs().sum())
        assert abs(along - float((dx.double() * v.double()).sum())) < 630 * 30 * h * h / 6 + 4 * E32 * terms / h
        along = (value(x, w + h * a) - value(x, w - h * a)) / (2 * h)
        assert abs(along - float((dw.double() * a.double()).sum())) < 1e-3 + 4 * E32 * terms / h


# ---------------------------------------------------------------- rows in 8 bits

def gate_error(act, g):
    """Relative (to act(g)) and absolute error of act(g): exponential and reciprocal, or where 1 + erf cancels."""
    return (8 + 2 * g.abs()) * E32, g.abs() * 2.0 ** -22 if act == ops.ACT_GELU else 0.0 * g


@pytest.mark.parametrize("dtype", DTYPES, ids=NAMES)
@pytest.mark.parametrize("width", [1, 7, 8, 64, 100, 501, 768, 1024, 6144, 6152, 11008, 11007, 16384, 40000])
def test_quantize_rows(width, dtype):
    gen = torch.Generator(device="cuda").manual_seed(width)
    for n, extra, shift in ((1, 0, 0), (45, 0, 0), (20, 3, 1), (300, 8, 0)):
        x = rows_of(gen, n, width, dtype, extra, shift)
        codes, scale = ops.quantize_rows(x)
        f = x.float()
        top = f.abs().amax(dim=1)
        # bit for bit: the definition in fp32, with 127 times the reciprocal (a tensor over a number is not a division in torch)
        assert torch.equal(scale, top / torch.full_like(top, 127.0))
        assert torch.equal(codes.float(), (f * (top.reciprocal() * 127.0)[:, None]).round())
        gate = rows_of(gen, n, width, dtype, extra, shift, scale=2.0)
        for act in (ops.ACT_SILU, ops.ACT_GELU, ops.ACT_RELU, ops.ACT_SIGMOID):
            codes, scale = ops.quantize_rows(x, gate=gate, activation=act)
            g = gate.double()
            value, rel, off = activation(act, g)[0], *gate_error(act, g)
            h = value * x.double()
            top = h.abs().amax(dim=1, keepdim=True).clamp(min=1e-300)
            error = (((rel + 2 * E32) * value.abs() + off) * x.double().abs()).amax(dim=1, keepdim=True) / top
            # (what cancels in 1 + erf(g / sqrt 2) counts only in rows that hold nothing larger)
            assert (act == ops.ACT_GELU and width < 64) or float(error.max()) < 2.0 ** -16, "the bound would hide errors"
            check_codes(codes, scale, h, float(error.max()))


def test_halves_of_one_matrix():
    """Gate and value side by side, as a product of both leaves them."""
    both = torch.randn(50, 2 * 344, device="cuda").bfloat16()
    codes, scale = ops.quantize_rows(both[:, 344:], gate=both[:, :344])
    want = ops.quantize_rows(both[:, 344:].contiguous(), gate=both[:, :344].contiguous())
    assert torch.equal(codes, want[0]) and torch.equal(scale, want[1])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_smallest_rows(dtype):
    x = torch.zeros(4, 64, device="cuda")
    x[0, 5], x[1, 5], x[2, 5] = 2.0 ** -120, 2.0 ** -121, 3e38
    codes, scale = ops.quantize_rows(x.to(dtype))
    assert codes[0, 5] == 127 and float(scale[0]) > 0
    assert not codes[1].any() and scale[1] == 0 and codes[2, 5] == 127 and not codes[3].any() and scale[3] == 0


@pytest.mark.parametrize("dtype", DTYPES, ids=NAMES)
@pytest.mark.parametrize("inputs,outputs,extra", [(1, 1, 0), (7, 33, 0), (128, 64, 0), (500, 31, 5), (1000, 1371, 8)])
def test_quantize_weight(inputs, outputs, extra, dtype):
    gen = torch.Generator(device="cuda").manual_seed(inputs)
    w = rows_of(gen, inputs, outputs, dtype, extra)
    codes, scale = ops.quantize_weight(w)
    rows, row_scale = ops.quantize_rows(w.T.contiguous())
    assert codes.shape == (outputs, inputs) and torch.equal(codes, rows) and torch.equal(scale, row_scale)


# ---------------------------------------------------------------- streams, graphs, refusals

def test_other_stream_and_graph():
    gen = torch.Generator(device="cuda").manual_seed(2)
    x, r, dy = (rows_of(gen, 100, 776, torch.bfloat16) for _ in range(3))
    w = torch.ones(776, device="cuda")

    def all_of(**kw):
        y, total, rstd = ops.rms_norm(x, w, residual=r, save=True, **kw)
        dx, dw = ops.rms_norm_backward(dy, total, w, rstd, r, **kw)
        q, s, _ = ops.rms_norm_int8(x, w, residual=r, **kw)
        return [y, total, rstd, dx, dw, q, s, *ops.quantize_rows(x, gate=r, **kw), *ops.quantize_weight(x, **kw)]
    want = all_of()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = all_of(stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = all_of()
    for t in got:
        t.zero_()
    for _ in range(2):
        graph.replay()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_refusals():
    x = torch.randn(4, 8, device="cuda")
    w = torch.ones(8, device="cuda")
    rstd = torch.ones(4, device="cuda")
    bad = [
        lambda: ops.rms_norm(x.double(), w), lambda: ops.rms_norm(x.cpu(), w), lambda: ops.rms_norm(x, w.bfloat16()),
        lambda: ops.rms_norm(x, torch.ones(7, device="cuda")), lambda: ops.rms_norm(x, w, residual=x.bfloat16()),
        lambda: ops.rms_norm(x, w, residual=x[:3]), lambda: ops.rms_norm(x.T, w), lambda: ops.rms_norm(x, w, eps=-1.0),
        lambda: ops.rms_norm(x, w, eps=float("nan")), lambda: ops.rms_norm(x[0], w), lambda: ops.rms_norm(x[:, :0], None),
        lambda: ops.rms_norm(x.requires_grad_(), w), lambda: ops.rms_norm_backward(x, x[:, :7], w, rstd),
        lambda: ops.rms_norm_backward(x, x, w, rstd[:3]), lambda: ops.rms_norm_backward(x, x, w, rstd.double()),
        lambda: ops.rms_norm_backward(x, x, w, rstd, dtotal=x[:2]), lambda: ops.quantize_rows(x.detach(), gate=x.detach()[:, :4]),
        lambda: ops.quantize_rows(x.detach(), gate=x.detach(), activation=4), lambda: ops.quantize_rows(x.detach().int()),
        lambda: ops.quantize_weight(x.detach()[:, :0]), lambda: ops.quantize_weight(x.detach().T),
    ]
    for k, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            pytest.fail(f"call {k} was taken")
    with torch.no_grad():
        ops.rms_norm(x, w)
