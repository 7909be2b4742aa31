"""Log probabilities, entropies, alternatives and their gradient against their definitions in 64 bits.

Bounds: a sum of C terms has at most C / 64 + 256 roundings of 2^-24 in a row, its exponentials included; a log probability eight more of
its own size (differences, their multiples of log2 e)."""
import math

import pytest
import torch

from paper_2312_08728_b200 import operators as ops
from test_gpu_norm import inside, rows_of
from test_gpu_operators import E32, TINY, U

pytestmark = pytest.mark.gpu

DTYPES = [torch.bfloat16, torch.float16, torch.float32]
NAMES = ["bf16", "fp16", "fp32"]
INF = float("inf")


def reference(z, y):
    """Rows that have a distribution: (logp, entropy) in 64 bits."""
    z = z.double() - z.double().amax(dim=1, keepdim=True)   # (log C beside 3e38 is lost in 64 bits too)
    logp = z - torch.logsumexp(z, dim=1, keepdim=True)
    p = torch.exp(logp)
    return logp, -(p * torch.where(p > 0, logp, torch.zeros_like(logp))).sum(dim=1)


def check(z, y, top, **kw):
    """Rows whose logits are finite or -Inf, not all of them -Inf."""
    rows, C = z.shape
    logprob, entropy, classes, values, saved = ops.log_probs(z, y, top=top, save=True, **kw)
    logp, want = reference(z, y)
    sums = (C / 64 + 256) * E32
    inside(entropy, want, sums * (2 + want) * 2, "entropy")
    has = (y >= 0) & (y < C)
    at = y.clamp(0, C - 1).long()[:, None]
    picked = torch.where(has, logp.gather(1, at).squeeze(1), torch.zeros_like(want))
    finite = torch.isfinite(picked.float())       # (the lowest value below the highest is beyond fp32: -Inf)
    inside(logprob[finite], picked[finite], sums + 8 * E32 * picked[finite].abs(), "logprob")
    assert bool((logprob[~finite] == -INF).all())
    if top:
        best = torch.sort(z.double() + 0.0, dim=1, descending=True, stable=True).indices[:, :top]
        assert torch.equal(classes.long(), best)
        v = logp.gather(1, best)
        f = torch.isfinite(v.float())
        inside(values[f], v[f], sums + 8 * E32 * v[f].abs(), "values")
        assert bool((values[~f] == -INF).all())
    else:
        assert classes.shape == (rows, 0) and values.shape == (rows, 0)
    return saved, logp, want


def check_backward(z, y, dl, de, saved, logp, entropy):
    rows, C = z.shape
    dz = ops.log_probs_backward(dl, de, z, y, saved)
    has = (y >= 0) & (y < C)
    a = torch.where(has, dl.double(), torch.zeros_like(entropy))[:, None] if dl is not None else torch.zeros_like(entropy)[:, None]
    b = de.double()[:, None] if de is not None else torch.zeros_like(a)
    p, lp = torch.exp(logp), torch.where(torch.isfinite(logp), logp, torch.zeros_like(logp))
    h = entropy[:, None]
    want = -p * (a + b * (lp + h))
    sums = (C / 64 + 256) * E32
    e = p * ((a.abs() + b.abs() * (lp + h).abs()) * (sums + 8 * E32 * lp.abs()) + b.abs() * (sums * (2 + h) * 2 + 16 * E32 * (lp.abs() + h)) + 4 * E32 * a.abs())
    want.scatter_add_(1, y.clamp(0, C - 1).long()[:, None], a)
    e = e + 2 * E32 * want.abs() + a.abs() * 2 * E32
    u, tiny = U[z.dtype], TINY[z.dtype] + 2.0 ** -126      # (below that p is 0)
    assert dz.dtype == z.dtype and dz.is_contiguous()
    inside(dz, want, e + u * (want.abs() + e) + tiny, "dlogits")


# a warp's row with its pieces in registers and one full round, blocks of 64 and of 512 threads, several rounds and what is left of them
CLASSES = [1, 2, 7, 10, 33, 100, 511, 1000, 1024, 1025, 2048, 4000, 8200, 32000, 50257, 131072]


@pytest.mark.parametrize("dtype", DTYPES, ids=NAMES)
@pytest.mark.parametrize("C", CLASSES)
def test_log_probs(C, dtype):
    gen = torch.Generator(device="cuda").manual_seed(C)
    for rows in (1, 37, 700 if C < 20000 else 600):
        z = rows_of(gen, rows, C, dtype, scale=3.0)
        y = torch.randint(0, C, (rows,), generator=gen, device="cuda", dtype=torch.int32)
        y[::5] = -1
        y[1::7] = C
        for top in {0, 1, min(5, C), min(32, C)}:
            saved, logp, entropy = check(z, y, top)
        dl, de = torch.randn(rows, generator=gen, device="cuda"), torch.randn(rows, generator=gen, device="cuda")
        for a, b in ((dl, de), (dl, None), (None, de)):
            check_backward(z, y, a, b, saved, logp, entropy)


@pytest.mark.parametrize("dtype", DTYPES, ids=NAMES)
@pytest.mark.parametrize("C,extra,shift", [(100, 1, 0), (1000, 3, 1), (5000, 8, 0), (5001, 2, 3), (50257, 7, 5)])
def test_strides_and_boundaries(C, extra, shift, dtype):
    gen = torch.Generator(device="cuda").manual_seed(C)
    z = rows_of(gen, 40, C, dtype, extra, shift, scale=2.0)
    y = torch.randint(0, C, (40,), generator=gen, device="cuda", dtype=torch.int32)
    saved, logp, entropy = check(z, y, 7)
    check_backward(z, y, torch.randn(40, generator=gen, device="cuda"), torch.randn(40, generator=gen, device="cuda"), saved, logp, entropy)


@pytest.mark.parametrize("dtype", DTYPES, ids=NAMES)
@pytest.mark.parametrize("C", [10, 700, 3000, 50257])
def test_ties_and_masks(C, dtype):
    """Equal logits go by their class; masks that leave fewer than the alternatives; ordered rows; one row far above the rest."""
    gen = torch.Generator(device="cuda").manual_seed(C)
    ramp = torch.arange(C, device="cuda", dtype=torch.float32)
    few = torch.full((C,), -INF, device="cuda")
    few[C // 2], few[C // 3], few[1] = 1.0, 2.0, 1.0
    half = torch.randn(C, generator=gen, device="cuda")
    half[torch.rand(C, generator=gen, device="cuda") < 0.5] = -INF
    half[0] = 0.5
    one = torch.full((C,), -INF, device="cuda")
    one[C - 1] = -7.0
    coarse = (torch.randn(C, generator=gen, device="cuda") * 2).round()
    signs = torch.where(ramp % 2 == 0, torch.zeros_like(ramp), -torch.zeros_like(ramp))
    peak = torch.zeros(C, device="cuda")
    peak[C // 2] = 300.0
    blocks = torch.where(ramp < C // 2, torch.ones_like(ramp), torch.zeros_like(ramp))
    z = torch.stack([torch.zeros(C, device="cuda"), ramp / C * 8, -ramp / C * 8, few, half, one, coarse, signs, peak, blocks, torch.full((C,), -3.0, device="cuda")]).to(dtype)
    y = torch.tensor([0, C - 1, 0, C // 2, 0, C - 1, 5, 3, C // 2, C - 1, 2], device="cuda", dtype=torch.int32) % C
    y2 = torch.tensor([1, 2, 3, 0, 1, 0, 1, 2, 1, 0, 3], device="cuda", dtype=torch.int32) % C       # also classes that a mask rules out
    for top in (1, min(3, C), min(20, C), min(32, C)):
        saved, logp, entropy = check(z, y, top)
        check(z, y2, top)
        check(z.repeat(60, 1), y.repeat(60), top)       # (the form for many rows)
    ones = torch.ones(len(z), device="cuda")
    check_backward(z, y, ones, ones, saved, logp, entropy)
    check_backward(z, y2, ones, -ones, saved, logp, entropy)
    # one class left: its sum is one but for the rounding of its exponent's base, which log s takes back: two roundings of at most 2^-24 each
    assert float(ops.log_probs_backward(ones, ones, z, y, saved)[5].abs().max()) <= 8 * E32


@pytest.mark.parametrize("dtype", DTYPES, ids=NAMES)
@pytest.mark.parametrize("C", [10, 700, 3000, 50257])
def test_extremes(C, dtype):
    low, high = torch.finfo(dtype).min, torch.finfo(dtype).max
    gen = torch.Generator(device="cuda").manual_seed(C)
    z = torch.randn(8, C, generator=gen, device="cuda").to(dtype)
    z[0] = low                                           # masked throughout by the lowest value
    z[1, 2:] = low                                       # two classes left
    z[2] = high
    z[3] = low
    z[3, 4] = -INF
    z[4] = high
    z[4, 1:] = low
    z[5] += torch.tensor(3e4 if dtype == torch.float16 else 1e30, dtype=dtype, device="cuda")
    z[6] -= torch.tensor(6e4 if dtype == torch.float16 else 1e37, dtype=dtype, device="cuda")
    y = torch.zeros(8, dtype=torch.int32, device="cuda")
    for rows in (8, 640):
        zz, yy = z.repeat(rows // 8, 1), y.repeat(rows // 8)
        saved, logp, entropy = check(zz, yy, min(20, C))
        check_backward(zz, yy, torch.ones(rows, device="cuda"), torch.ones(rows, device="cuda"), saved, logp, entropy)


@pytest.mark.parametrize("dtype", DTYPES, ids=NAMES)
@pytest.mark.parametrize("C", [10, 700, 3000, 50257])
def test_nothing_nan_and_infinity(C, dtype):
    z = torch.randn(7, C, device="cuda").to(dtype)
    z[0] = -INF
    z[1, 3] = float("nan")
    z[2, C - 1] = INF
    z[3, 0] = z[3, 5] = INF
    z[4] = float("nan")
    y = torch.tensor([2, 0, 0, 1, 0, 0, -1], dtype=torch.int32, device="cuda")
    top = min(20, C)
    for rows in (7, 700):
        logprob, entropy, classes, values, saved = ops.log_probs(z.repeat(rows // 7, 1), y.repeat(rows // 7), top=top, save=True)
        ones = torch.ones(rows, device="cuda")
        dz = ops.log_probs_backward(ones, ones, z.repeat(rows // 7, 1), y.repeat(rows // 7), saved)
        for at in (0, rows - 7):
            assert logprob[at] == 0 and entropy[at] == 0 and bool((values[at] == -INF).all()) and not dz[at].any()
            assert classes[at].tolist() == list(range(top))
            for row in (1, 2, 3, 4):
                assert bool(torch.isnan(logprob[at + row])) and bool(torch.isnan(entropy[at + row])) and bool(torch.isnan(values[at + row]).all())
                assert bool(torch.isnan(dz[at + row]).all())
            assert classes[at + 1, 0] == 3 and classes[at + 2, 0] == C - 1 and classes[at + 3, :2].tolist() == [0, 5]
            assert classes[at + 4].tolist() == list(range(top))
            assert bool(torch.isfinite(entropy[at + 5:at + 7]).all()) and logprob[at + 6] == 0
    # rows without a class, and without anything asked of their entropy, count for nothing, whatever they hold
    none = torch.full((7,), -1, dtype=torch.int32, device="cuda")
    _, _, _, _, saved = ops.log_probs(z, none, save=True)
    assert not ops.log_probs_backward(torch.ones(7, device="cuda"), None, z, none, saved).any()
    assert not ops.log_probs_backward(None, None, z, y, saved).any()


def test_no_labels_and_no_rows():
    z = torch.randn(5, 300, device="cuda")
    logprob, entropy, classes, values = ops.log_probs(z, top=3)
    assert not logprob.any() and classes.shape == (5, 3)
    assert torch.equal(classes[:, 0].long(), z.argmax(dim=1))
    logprob, entropy, classes, values, saved = ops.log_probs(z[:0], torch.zeros(0, dtype=torch.int32, device="cuda"), top=3, save=True)
    assert logprob.shape == (0,) and classes.shape == (0, 3)
    assert ops.log_probs_backward(None, None, z[:0], None, saved).shape == (0, 300)


def test_the_loss_of_softmax_residual():
    """The log probability is the loss with its sign turned, its gradient the residual."""
    z = (torch.randn(100, 777, device="cuda") * 2).bfloat16()
    y = torch.randint(-1, 777, (100,), device="cuda", dtype=torch.int32)
    residual, loss = ops.softmax_residual(z, y, scale=1.0)
    logprob, _, _, _, saved = ops.log_probs(z, y, save=True)
    assert torch.allclose(logprob, -loss, rtol=1e-5, atol=1e-5)
    dz = ops.log_probs_backward(torch.full((100,), -1.0, device="cuda"), None, z, y, saved)
    assert torch.allclose(dz.float(), residual.float(), rtol=2.0 ** -7, atol=1e-6)


def test_the_gradient_against_differences():
    """Along random directions, in fp32: the third derivative of log probabilities and entropies of logits of this size stays below 10."""
    gen = torch.Generator(device="cuda").manual_seed(5)
    z = torch.randn(20, 90, generator=gen, device="cuda") * 2
    y = torch.randint(0, 90, (20,), generator=gen, device="cuda", dtype=torch.int32)
    dl, de = torch.randn(20, generator=gen, device="cuda"), torch.randn(20, generator=gen, device="cuda")
    saved = ops.log_probs(z, y, save=True)[4]
    dz = ops.log_probs_backward(dl, de, z, y, saved).double()

    def value(z):
        logprob, entropy, _, _ = ops.log_probs(z, y)
        return float((logprob.double() * dl.double() + entropy.double() * de.double()).sum())
    h = 2.0 ** -7
    for _ in range(5):
        v = torch.randn(20, 90, generator=gen, device="cuda")
        v /= v.abs().max()
        along = (value(z + h * v) - value(z - h * v)) / (2 * h)
        size = float((dl.abs() * 10 + de.abs() * 5).sum())
        assert abs(along - float((dz * v.double()).sum())) < 10 * float((dl.abs() + de.abs()).sum()) * h * h / 6 + 16 * E32 * size / h


def test_equal_calls_give_equal_bits():
    z = torch.randn(900, 50257, device="cuda").bfloat16()
    y = torch.zeros(900, dtype=torch.int32, device="cuda")
    first = ops.log_probs(z, y, top=20, save=True)
    for _ in range(4):
        assert all(torch.equal(a, b) for a, b in zip(ops.log_probs(z, y, top=20, save=True), first))


def test_other_stream_and_graph():
    jobs = [(torch.randn(n, C, device="cuda").to(t), torch.randint(0, C, (n,), device="cuda", dtype=torch.int32)) for n, C, t in
            ((3, 50257, torch.bfloat16), (800, 3000, torch.float16), (40, 10, torch.float32))]

    def all_of(**kw):
        out = []
        for z, y in jobs:
            got = ops.log_probs(z, y, top=4, save=True, **kw)
            ones = torch.ones_like(got[0])
            out += [*got, ops.log_probs_backward(one[len(z)], one[len(z)], z, y, got[4], **kw)] if kw else [*got, ops.log_probs_backward(ones, ones, z, y, got[4])]
        return out
    one = {len(z): torch.ones(len(z), device="cuda") for z, _ in jobs}
    want = all_of()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = all_of(stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = all_of()
    for _ in range(2):
        graph.replay()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_refusals():
    z = torch.randn(4, 30, device="cuda")
    y = torch.zeros(4, dtype=torch.int32, device="cuda")
    saved = ops.log_probs(z, y, save=True)[4]
    f = torch.ones(4, device="cuda")
    bad = [
        lambda: ops.log_probs(z.double(), y), lambda: ops.log_probs(z, y.long()), lambda: ops.log_probs(z, y[:3]), lambda: ops.log_probs(z, y, top=33),
        lambda: ops.log_probs(z, y, top=-1), lambda: ops.log_probs(z[:, :4], y, top=5), lambda: ops.log_probs(z[:, :0], y), lambda: ops.log_probs(z.T, y[:4]),
        lambda: ops.log_probs(z.cpu(), y.cpu()), lambda: ops.log_probs(z[0], y), lambda: ops.log_probs_backward(f[:3], None, z, y, saved),
        lambda: ops.log_probs_backward(f, f.double(), z, y, saved), lambda: ops.log_probs_backward(f, f, z, y, saved[:3]),
        lambda: ops.log_probs_backward(f, f, z, y, saved.half()), lambda: ops.log_probs(z.requires_grad_(), y),
    ]
    for k, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            pytest.fail(f"call {k} was taken")
    assert math.isfinite(float(ops.log_probs(z.detach(), y)[0].sum()))
