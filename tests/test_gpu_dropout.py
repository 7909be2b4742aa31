"""Dropout against the generator's definition, word by word, and its values within their roundings."""
import numpy as np
import pytest
import torch

from paper_2312_08728_b200 import operators as ops
from test_gpu_norm import inside, rows_of
from test_gpu_operators import E32, TINY, U

pytestmark = pytest.mark.gpu

DTYPES = [torch.bfloat16, torch.float16, torch.float32]
NAMES = ["bf16", "fp16", "fp32"]


def philox(c, k):
    """Philox4x32-10 on arrays of 64-bit integers that hold 32-bit words."""
    c = [np.asarray(x, dtype=np.uint64) for x in np.broadcast_arrays(*c)]
    k0, k1 = (np.uint64(x & 0xFFFFFFFF) for x in k)
    low = np.uint64(0xFFFFFFFF)
    for _ in range(10):
        a, b = np.uint64(0xD2511F53) * c[0], np.uint64(0xCD9E8D57) * c[2]
        c = [(b >> np.uint64(32)) ^ c[1] ^ k0, b & low, (a >> np.uint64(32)) ^ c[3] ^ k1, a & low]
        k0, k1 = (k0 + np.uint64(0x9E3779B9)) & low, (k1 + np.uint64(0xBB67AE85)) & low
    return c


def kept(first, count, rate, seed, layer=0, step=0):
    """Whether values first .. first + count - 1 stay."""
    blocks = np.arange(first // 8, (first + count + 7) // 8, dtype=np.uint64)
    words = philox([blocks & np.uint64(0xFFFFFFFF), blocks >> np.uint64(32), step & 0xFFFFFFFF, 0x44524F50 + layer], (seed, seed >> 32))
    numbers = np.stack([h for w in words for h in (w & np.uint64(0xFFFF), w >> np.uint64(16))], axis=1).reshape(-1)
    numbers = numbers[first % 8:first % 8 + count]
    return torch.from_numpy(numbers >= round(rate * 65536)).cuda()


def check(x, rate, seed, residual=None, layer=0, step=None, **kw):
    n, d = x.shape
    y = ops.dropout(x, rate, seed, layer=layer, step=None if step is None else torch.tensor([step], device="cuda"), residual=residual, **kw)
    keep = kept(0, n * d, rate, seed, layer, step or 0).view(n, d)
    factor = 65536.0 / (65536 - round(rate * 65536))
    want = torch.where(keep, x.double() * factor, torch.zeros((), dtype=torch.float64, device="cuda"))
    size = want.abs()
    if residual is not None:
        want, size = want + residual.double(), size + residual.double().abs()
    else:
        assert not y[~keep].any()
    inside(y, want, 4 * E32 * size + U[x.dtype] * want.abs() * (1 + 4 * E32) + U[x.dtype] * 4 * E32 * size + TINY[x.dtype], "y")
    return y, keep


@pytest.mark.parametrize("dtype", DTYPES, ids=NAMES)
@pytest.mark.parametrize("n,d,extra,shift", [(1, 1, 0, 0), (1, 7, 0, 0), (1, 8, 0, 0), (3, 5, 0, 0), (2, 4096, 0, 0), (777, 501, 0, 0), (777, 501, 0, 1), (5, 13, 2, 0), (40, 512, 8, 0),
                                             (40, 512, 3, 1), (100, 3, 1, 0), (33, 1000, 24, 0), (4000, 8, 8, 0), (1, 100_003, 0, 0)])
def test_dropout(n, d, extra, shift, dtype):
    gen = torch.Generator(device="cuda").manual_seed(n + d)
    x, r = rows_of(gen, n, d, dtype, extra, shift), rows_of(gen, n, d, dtype, extra + 1, 0)
    check(x, 0.3, 12345)
    check(x, 0.3, 12345, residual=r)
    check(x, 0.07, -5 & 0xFFFFFFFFFFFFFFFF, residual=rows_of(gen, n, d, dtype), layer=7, step=2 ** 40 + 3)


def test_rates():
    x = torch.ones(400, 1000, device="cuda")
    for rate in (0.0, 2.0 ** -18, 2.0 ** -16, 0.5, 0.9, 65535 / 65536):
        y, keep = check(x, rate, 3)
        dropped = 1 - float(keep.float().mean())
        assert abs(dropped - round(rate * 65536) / 65536) < 5 * (rate * (1 - rate) / 4e5) ** 0.5 + 1e-9
    assert torch.equal(ops.dropout(x, 0.0, 3), x)


def test_a_dropped_value_is_zero_whatever_it_was():
    x = torch.full((64, 64), float("nan"), device="cuda")
    x[::2] = float("inf")
    keep = kept(0, 4096, 0.5, 1).view(64, 64)
    y = ops.dropout(x, 0.5, 1)
    assert not y[~keep].any() and bool((~torch.isfinite(y[keep])).all())
    r = torch.randn(64, 64, device="cuda")
    assert torch.equal(ops.dropout(x, 0.5, 1, residual=r)[~keep], r[~keep])


def test_what_the_mask_depends_on():
    x = torch.ones(100, 512, device="cuda")
    base = ops.dropout(x, 0.5, 10)
    step = torch.zeros(1, dtype=torch.int64, device="cuda")
    assert torch.equal(ops.dropout(x, 0.5, 10, step=step), base) and torch.equal(ops.dropout(x.bfloat16(), 0.5, 10).float(), base)
    wide = torch.ones(100, 700, device="cuda")
    assert torch.equal(ops.dropout(wide[:, 3:515], 0.5, 10), base)                # (strides and boundaries do not matter)
    others = [ops.dropout(x, 0.5, 11), ops.dropout(x, 0.5, 10 + 2 ** 32), ops.dropout(x, 0.5, 10, layer=1), ops.dropout(x, 0.5, 10, step=step + 1), base]
    for i, a in enumerate(others):
        for b in others[:i]:
            assert abs(float(((a > 0) == (b > 0)).float().mean()) - 0.5) < 0.02


def test_the_gradient_is_the_same_call():
    """y is linear in x: the sum of dy y changes by dropout(dy) along any direction, but for roundings."""
    x, dy, v = (torch.randn(50, 77, device="cuda") for _ in range(3))
    dx = ops.dropout(dy, 0.2, 9, layer=2)
    along = (ops.dropout(x + v, 0.2, 9, layer=2).double() * dy.double()).sum() - (ops.dropout(x - v, 0.2, 9, layer=2).double() * dy.double()).sum()
    size = ((x.abs() + v.abs()) * dy.abs()).sum() * 1.25
    assert abs(float(along / 2 - (dx.double() * v.double()).sum())) < 4 * E32 * float(size)


def test_other_stream_and_graphs():
    x, r = torch.randn(300, 200, device="cuda").bfloat16(), torch.randn(300, 200, device="cuda").bfloat16()
    step = torch.zeros(1, dtype=torch.int64, device="cuda")
    want = [ops.dropout(x, 0.4, 8, step=torch.tensor([k], device="cuda"), residual=r) for k in range(3)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = ops.dropout(x, 0.4, 8, step=step, residual=r, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = ops.dropout(x, 0.4, 8, step=step, residual=r)
    for k in range(3):      # a replayed call reads the step anew
        step.fill_(k)
        graph.replay()
        assert torch.equal(got, want[k])


def test_in_place():
    """Through the C call: y may be x, or the residual."""
    from paper_2312_08728_b200 import binding
    L = binding.load_library()
    s = torch.cuda.current_stream().cuda_stream
    for n, d, ld in ((30, 64, 64), (30, 61, 70), (1, 1003, 1003)):
        x, r = torch.randn(n, ld, device="cuda").bfloat16(), torch.randn(n, ld, device="cuda").bfloat16()
        want = ops.dropout(x[:, :d], 0.3, 4, residual=r[:, :d])
        for into in (x.clone(), r.clone()):
            a, b = (into, r) if torch.equal(into, x) else (x, into)
            args = ops._DROPOUT.pack(n, d, ops.TYPE_BF16, 0, 0.3, 4, 0, a.data_ptr(), b.data_ptr(), into.data_ptr(), ld, ld, ld)
            assert L.bmgd_dropout(args, s) == 0
            torch.cuda.synchronize()
            assert torch.equal(into[:, :d], want)
        args = ops._DROPOUT.pack(n, d, ops.TYPE_BF16, 0, 0.3, 4, 0, x.data_ptr(), 0, x.data_ptr() + 2, ld, 0, ld)
        assert L.bmgd_dropout(args, s) == binding.ERR_ARG


def test_refusals():
    x = torch.randn(4, 8, device="cuda")
    step = torch.zeros(1, dtype=torch.int64, device="cuda")
    bad = [
        lambda: ops.dropout(x, 1.0, 0), lambda: ops.dropout(x, -0.1, 0), lambda: ops.dropout(x, float("nan"), 0), lambda: ops.dropout(x, 1 - 2.0 ** -18, 0),
        lambda: ops.dropout(x.double(), 0.1, 0), lambda: ops.dropout(x.cpu(), 0.1, 0), lambda: ops.dropout(x.T, 0.1, 0), lambda: ops.dropout(x, 0.1, 0, layer=-1),
        lambda: ops.dropout(x, 0.1, 0, layer=65536), lambda: ops.dropout(x, 0.1, 0, step=step.int()), lambda: ops.dropout(x, 0.1, 0, step=step.cpu()),
        lambda: ops.dropout(x, 0.1, 0, step=torch.zeros(2, dtype=torch.int64, device="cuda")), lambda: ops.dropout(x, 0.1, 0, residual=x[:3]),
        lambda: ops.dropout(x, 0.1, 0, residual=x.half()), lambda: ops.dropout(x[:, :0], 0.1, 0), lambda: ops.dropout(x.requires_grad_(), 0.1, 0),
    ]
    for k, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            pytest.fail(f"call {k} was taken")
    assert ops.dropout(x.detach()[:0], 0.1, 0).shape == (0, 8)
