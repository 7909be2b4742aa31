"""The product in 8-bit integers against whole numbers in 64 bits.

Bounds: the sum is exact; taking it to fp32, two scales and a bias are four roundings of 2^-24, the result's type half a step more."""
import ctypes

import pytest
import torch

from paper_2312_08728_b200 import binding
from paper_2312_08728_b200 import operators as ops
from test_gpu_norm import inside
from test_gpu_operators import E32, TINY, U

pytestmark = pytest.mark.gpu


def operands(n, d, c, seed=0, extra=0, shift=0, full=False):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def codes(rows):
        flat = torch.randint(-128 if full else -127, 128, (shift + rows * (d + extra),), generator=gen, device="cuda").to(torch.int8)
        return flat[shift:].view(rows, d + extra)[:, :d]
    return codes(n), torch.rand(n, generator=gen, device="cuda") + 0.1, codes(c), torch.randn(c, generator=gen, device="cuda")


def reference(q, qs, w, ws, bias):
    sums = q.double() @ w.double().T                     # whole numbers below 2^31: exact
    y = sums * qs.double()[:, None] * ws.double()
    size = y.abs()
    if bias is not None:
        y, size = y + bias.double(), size + bias.double().abs()
    return y, size


def check(q, qs, w, ws, bias=None, dtype=torch.bfloat16, **kw):
    y = ops.int8_linear(q, qs, w, ws, bias=bias, dtype=dtype, **kw)
    want, size = reference(q, qs, w, ws, bias)
    e = 5 * E32 * size
    assert y.dtype == dtype and y.shape == want.shape
    inside(y, want, e + U[dtype] * (want.abs() + e) + TINY[dtype], "y")
    return y


# one and two tokens; a cluster's split and none; tiles of one CTA; tiles of CTA pairs; sizes that end inside pieces and tiles
SHAPES = [(1, 1, 1), (1, 16, 8), (1, 4096, 1371), (2, 777, 300), (3, 128, 1000), (4, 2000, 2501), (5, 40, 40), (16, 128, 128), (17, 1371, 2501),
          (29, 2048, 264), (64, 96, 4104), (100, 4096, 130), (129, 520, 129), (200, 1000, 1000), (257, 264, 5000), (300, 1024, 6000), (777, 500, 3001),
          (2304, 1040, 2824), (1025, 4112, 2050), (2048, 264, 2048), (1, 1040, 6000), (2, 4112, 2370)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32], ids=["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_product(shape, dtype):
    q, qs, w, ws = operands(*shape, seed=sum(shape))
    ws = ws * (1.0 / (shape[1] ** 0.5 * 5000))           # (fp16 holds the results)
    bias = torch.randn(shape[2], device="cuda")
    check(q, qs, w, ws, bias, dtype)
    check(q, qs, w, ws, None, dtype)


@pytest.mark.parametrize("shape,extra,shift", [((3, 64, 40), 1, 0), ((3, 64, 40), 16, 0), ((1, 500, 77), 12, 0), ((33, 500, 77), 3, 1), ((33, 512, 77), 0, 5),
                                               ((300, 1001, 3000), 0, 0), ((300, 1001, 3000), 7, 2), ((2, 33, 5000), 0, 1)])
def test_strides_and_boundaries(shape, extra, shift):
    check(*operands(*shape, seed=3, extra=extra, shift=shift))


def test_codes_of_the_quantisation():
    """As the operators before it leave them: rows padded to 16 bytes."""
    x, w = torch.randn(70, 333, device="cuda"), torch.randn(333, 100, device="cuda")
    q, qs = ops.quantize_rows(x)
    codes, ws = ops.quantize_weight(w)
    assert q.stride(0) == 336 and codes.stride(0) == 336
    y = check(q, qs, codes, ws, dtype=torch.float32)
    # each code is off by half a scale at most
    half = 0.5 * qs.double()[:, None] * w.double().abs().sum(dim=0) + 0.5 * ws.double() * x.double().abs().sum(dim=1)[:, None] + 0.25 * 333 * qs.double()[:, None] * ws.double()
    assert bool(((y.double() - x.double() @ w.double()).abs() <= half * 1.0001).all())


@pytest.mark.parametrize("n,c", [(1, 40), (4, 40), (20, 40), (300, 20000)])
def test_largest_sums(n, c):
    """131,071 inputs of -128: 2,147,467,264."""
    d = 131071
    q, w = torch.full((n, d), -128, dtype=torch.int8, device="cuda"), torch.full((c, d), -128, dtype=torch.int8, device="cuda")
    w[c // 2] = 127
    y = ops.int8_linear(q, torch.ones(n, device="cuda"), w, torch.ones(c, device="cuda"), dtype=torch.float32)
    want = torch.full((c,), 131071.0 * 16384, device="cuda", dtype=torch.float64)
    want[c // 2] = -131071.0 * 128 * 127
    assert torch.equal(y, want.float().expand(n, c))


def test_a_token_alone_and_among_others():
    """Sums are exact, so every form gives the same bits."""
    q, qs, w, ws = operands(700, 1040, 2000, seed=1, full=True)
    all_of = ops.int8_linear(q, qs, w, ws, dtype=torch.float32)
    for n in (1, 2, 3, 4, 5, 16, 40, 100, 256, 300):
        assert torch.equal(ops.int8_linear(q[:n], qs[:n], w, ws, dtype=torch.float32), all_of[:n]), n


def test_scales_that_are_nan_or_zero():
    q, qs, w, ws = operands(40, 64, 24)
    qs[3], qs[5], ws[7] = float("nan"), 0.0, float("nan")
    for n in (4, 40):
        y = ops.int8_linear(q[:n], qs[:n], w, ws, dtype=torch.float32)
        assert bool(torch.isnan(y[3]).all()) and bool(torch.isnan(y[:, 7]).all()) and int(torch.isnan(y).sum()) == 24 + n - 1
        if n > 5:
            rest = torch.cat((y[5, :7], y[5, 8:]))
            assert not rest.any()


def test_other_stream_and_graph():
    jobs = [operands(n, 1001, 777, seed=n, extra=e) for n, e in ((1, 0), (30, 0), (1, 7), (900, 7))]
    want = [ops.int8_linear(*j) for j in jobs]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = [ops.int8_linear(*j, stream=side) for j in jobs]
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = [ops.int8_linear(*j) for j in jobs]
    for t in got:
        t.zero_()
    for _ in range(2):
        graph.replay()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_calls_at_once_on_several_streams():
    jobs = [operands(n, 1040, 3000, seed=n) for n in (7, 300, 1500, 2)]
    want = [ops.int8_linear(*j) for j in jobs]
    streams = [torch.cuda.Stream() for _ in jobs]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    got = [[ops.int8_linear(*j, stream=s) for j, s in zip(jobs, streams)] for _ in range(5)]
    for s in streams:
        torch.cuda.current_stream().wait_stream(s)
    assert all(torch.equal(a, b) for round_ in got for a, b in zip(round_, want))


# ---------------------------------------------------------------- waits that run out

@pytest.mark.parametrize("shape", [(1, 1, 1), (1, 15, 3), (3, 17, 129), (2, 130, 5), (16, 127, 128), (29, 1371, 2501), (64, 129, 300), (40, 4099, 1000), (100, 1371, 130), (129, 515, 129),
                                   (300, 1000, 1000), (500, 77, 600)], ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("extra,shift", [(0, 1), (1, 0), (2, 2), (3, 3), (16, 7)])
def test_few_tokens_on_any_boundary(shape, extra, shift):
    check(*operands(*shape, seed=5, extra=extra, shift=shift, full=True), dtype=torch.float32)


def test_one_operand_on_any_boundary():
    q, qs, w, ws = operands(33, 1360, 700, seed=6)
    odd = operands(33, 1360, 700, seed=6, extra=3, shift=1)
    y = check(q, qs, w, ws)
    odd[0].copy_(q), odd[2].copy_(w)
    assert torch.equal(check(odd[0], qs, w, ws), y) and torch.equal(check(q, qs, odd[2], ws), y) and torch.equal(check(odd[0], qs, odd[2], ws), y)


def test_nothing_beyond_a_row_counts():
    """What stands in front of, behind and between the rows changes nothing."""
    jobs = [operands(20, 1371, 400, seed=7, extra=5, shift=3) for _ in range(2)]
    for t in (jobs[1][0], jobs[1][2]):
        flat = torch.as_strided(t, (t.storage_offset() + t.shape[0] * t.stride(0),), (1,), 0)
        kept = t.clone()
        flat.fill_(-77)
        t.copy_(kept)
    assert torch.equal(ops.int8_linear(*jobs[0]), ops.int8_linear(*jobs[1]))


def starve(job, fills, dtype=torch.bfloat16, budget_ms=5.0):
    """A product whose kernel fetches `fills` pieces per CTA; the output's memory is zero before."""
    L = binding.load_library()
    q, qs, w, ws = job
    y = torch.zeros(q.shape[0], w.shape[0], dtype=dtype, device="cuda")
    args = ops._QUANTIZED_LINEAR.pack(q.shape[0], q.shape[1], w.shape[0], ops._TYPES[dtype], 0, q.data_ptr(), qs.data_ptr(), w.data_ptr(), ws.data_ptr(), 0,
                                      y.data_ptr(), q.stride(0), w.stride(0), w.shape[0])
    assert L.bmgd_debug_quantized_linear_timeout(args, None, 0, fills, budget_ms, torch.cuda.current_stream().cuda_stream) == 0
    torch.cuda.synchronize()
    return y


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("fills", [0, 1, 8])
@pytest.mark.parametrize("shape", [(3, 2048, 1376), (100, 128, 136), (700, 512, 2700), (2304, 1024, 2816), (2048, 1024, 2048), (3, 2047, 1376), (100, 127, 136)],
                         ids=lambda s: "x".join(map(str, s)))
def test_what_was_not_computed_is_nan(shape, fills, dtype):
    job = operands(*shape, seed=2)
    want = ops.int8_linear(*job, dtype=dtype)
    ops.stream_check()
    got = starve(job, fills, dtype)
    lost = torch.isnan(got)
    assert bool((lost | (got == want)).all())
    assert fills > 0 or bool(lost.all())
    if bool(lost.any()):
        again = ops.int8_linear(*job, dtype=dtype)       # (nobody has asked for the report yet)
        assert torch.equal(again, want)
        with pytest.raises(binding.BmgdError):
            ops.stream_check()
    else:
        assert 128 * fills >= shape[1] or fills == 8     # (everything could be fetched: a piece is 128 values long)
    ops.stream_check()


def test_refusals():
    q, qs, w, ws = operands(4, 32, 8)
    bad = [
        lambda: ops.int8_linear(q.float(), qs, w, ws), lambda: ops.int8_linear(q, qs, w[:, :31], ws), lambda: ops.int8_linear(q, qs[:3], w, ws),
        lambda: ops.int8_linear(q, qs, w, ws[:7]), lambda: ops.int8_linear(q, qs.double(), w, ws), lambda: ops.int8_linear(q, qs, w, ws, bias=ws[:5]),
        lambda: ops.int8_linear(q, qs, w, ws, dtype=torch.float64), lambda: ops.int8_linear(q.cpu(), qs, w, ws), lambda: ops.int8_linear(q, None, w, ws),
        lambda: ops.int8_linear(q, qs, w, None), lambda: ops.int8_linear(q[:, :0], qs, w[:, :0], ws), lambda: ops.int8_linear(q.T, qs, w, ws),
        lambda: ops.int8_linear(q, qs, w.view(torch.uint8), ws), lambda: ops.int8_linear(q, qs.requires_grad_(), w, ws),
    ]
    for k, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            pytest.fail(f"call {k} was taken")
    wide = torch.zeros(1, 131072, dtype=torch.int8, device="cuda")
    with pytest.raises(ValueError):
        ops.int8_linear(wide, torch.ones(1, device="cuda"), wide, torch.ones(1, device="cuda"))
    y = ops.int8_linear(q[:0], qs.detach()[:0], w, ws)
    assert y.shape == (0, 8)
    L, need = binding.load_library(), ctypes.c_int64()
    args = ops._QUANTIZED_LINEAR.pack(4000, 32, 800, 1, 0, q.data_ptr() + 1, qs.data_ptr(), w.data_ptr() + 1, ws.data_ptr(), 0, 1 << 20, 32, 32, 800)
    assert L.bmgd_quantized_linear_workspace_bytes(args, ctypes.byref(need)) == 0 and need.value > 0
    assert L.bmgd_quantized_linear(args, None, 0, None) == binding.ERR_ARG
    assert L.bmgd_quantized_linear(args, 1 << 20, need.value - 1, None) == binding.ERR_CAPACITY
