"""Operands and results side by side in one wide matrix, through the C calls: they share no memory, so they are taken, and give what separate ones give."""
import ctypes

import pytest
import torch

from paper_2312_08728_b200 import binding
from paper_2312_08728_b200 import operators as ops

pytestmark = pytest.mark.gpu

DTYPES = [torch.bfloat16, torch.float16, torch.float32]
NAMES = ["bf16", "fp16", "fp32"]


class Wide:
    """Parts of `n` rows side by side: each a tensor of its own type, `gap` bytes behind the one before."""

    def __init__(self, n, parts, gap=0):
        at, places = 0, []
        for dtype, cols in parts:
            at = -(-at // dtype.itemsize) * dtype.itemsize
            places.append((at, dtype, cols))
            at += cols * dtype.itemsize + gap
        self.pitch = -(-at // 16) * 16
        self.memory = torch.zeros(n * self.pitch, dtype=torch.uint8, device="cuda")
        self.tensors = [torch.as_strided(self.memory.view(t), (n, c), (self.pitch // t.itemsize, 1), p // t.itemsize) for p, t, c in places]


def stream():
    return torch.cuda.current_stream().cuda_stream


@pytest.mark.parametrize("dtype", DTYPES, ids=NAMES)
@pytest.mark.parametrize("n,d", [(5, 64), (70, 501), (9, 4096), (3, 40000)])
def test_norm(n, d, dtype):
    L, code = binding.load_library(), ops._TYPES[dtype]
    x, r, total, y, codes, dy, dx = Wide(n, [(dtype, d)] * 4 + [(torch.int8, d)] + [(dtype, d)] * 2, gap=8).tensors
    for t in (x, r, dy):
        t.copy_(torch.randn(n, d, device="cuda"))
    w = 1 + 0.1 * torch.randn(d, device="cuda")
    want, want_total, rstd = ops.rms_norm(x, w, residual=r, save=True)
    q, scale, _ = ops.rms_norm_int8(x, w, residual=r)
    got_rstd, got_scale = torch.zeros_like(rstd), torch.zeros_like(scale)

    def args(at_y, at_codes, at_scale, at_rstd):
        return ops._RMS_NORM.pack(n, d, code, 0, 0, 1e-6, x.data_ptr(), r.data_ptr(), w.data_ptr(), total.data_ptr(), at_y, at_codes, at_scale, at_rstd, x.stride(0), r.stride(0),
                                  total.stride(0), y.stride(0), codes.stride(0), 0, 0, 0, 0, 0, 0, 0)
    assert L.bmgd_rms_norm_forward(args(y.data_ptr(), 0, 0, got_rstd.data_ptr()), stream()) == 0
    assert torch.equal(y, want) and torch.equal(total, want_total) and torch.equal(got_rstd, rstd)
    total.zero_()
    assert L.bmgd_rms_norm_forward(args(0, codes.data_ptr(), got_scale.data_ptr(), 0), stream()) == 0
    assert torch.equal(codes, q) and torch.equal(total, want_total) and torch.equal(got_scale, scale)
    want_dx, want_dw = ops.rms_norm_backward(dy, total, w, rstd, r)
    dw, need = torch.zeros_like(w), ctypes.c_int64()
    back = ops._RMS_NORM.pack(n, d, code, 0, 0, 0.0, 0, 0, w.data_ptr(), total.data_ptr(), 0, 0, 0, rstd.data_ptr(), 0, 0, total.stride(0), 0, 0, dy.data_ptr(), r.data_ptr(),
                              dx.data_ptr(), dw.data_ptr(), dy.stride(0), r.stride(0), dx.stride(0))
    assert L.bmgd_rms_norm_workspace_bytes(back, ctypes.byref(need)) == 0
    space = torch.empty(need.value, dtype=torch.uint8, device="cuda")
    assert L.bmgd_rms_norm_backward(back, space.data_ptr(), need.value, stream()) == 0
    assert torch.allclose(dx.float(), want_dx.float(), rtol=2.0 ** -7, atol=1e-5) and torch.allclose(dw, want_dw, rtol=1e-5, atol=1e-5)


@pytest.mark.parametrize("dtype", DTYPES, ids=NAMES)
@pytest.mark.parametrize("n,d", [(5, 64), (70, 501), (3, 40000)])
def test_codes(n, d, dtype):
    L, code = binding.load_library(), ops._TYPES[dtype]
    x, gate, codes = Wide(n, [(dtype, d), (dtype, d), (torch.int8, d)], gap=4).tensors
    x.copy_(torch.randn(n, d, device="cuda")), gate.copy_(torch.randn(n, d, device="cuda"))
    q, scale = ops.quantize_rows(x, gate=gate)
    got = torch.zeros_like(scale)
    assert L.bmgd_quantize_rows(ops._QUANTIZE_ROWS.pack(n, d, code, 0, 0, x.data_ptr(), gate.data_ptr(), codes.data_ptr(), got.data_ptr(), x.stride(0), gate.stride(0),
                                                        codes.stride(0)), stream()) == 0
    assert torch.equal(codes, q) and torch.equal(got, scale)
    if n == 70:     # a weight [n, n] beside its codes [n, n]
        w, codes = Wide(n, [(dtype, n), (torch.int8, n)]).tensors
        w.copy_(torch.randn(n, n, device="cuda"))
        q, scale = ops.quantize_weight(w)
        got = torch.zeros_like(scale)
        assert L.bmgd_quantize_weight(w.data_ptr(), w.stride(0), n, n, code, codes.data_ptr(), codes.stride(0), got.data_ptr(), stream()) == 0
        assert torch.equal(codes, q) and torch.equal(got, scale)


@pytest.mark.parametrize("dtype", DTYPES, ids=NAMES)
@pytest.mark.parametrize("n,d,c", [(1, 64, 40), (2, 500, 40), (20, 1371, 264), (300, 520, 3000)])
def test_product(n, d, c, dtype):
    L = binding.load_library()
    q, y = Wide(n, [(torch.int8, d), (dtype, c)], gap=4).tensors
    q.copy_(torch.randint(-127, 128, (n, d), device="cuda"))
    w = torch.randint(-127, 128, (c, d), device="cuda").to(torch.int8)
    qs, ws = torch.rand(n, device="cuda") / d, torch.rand(c, device="cuda") / 100
    want = ops.int8_linear(q, qs, w, ws, dtype=dtype)
    args = ops._QUANTIZED_LINEAR.pack(n, d, c, ops._TYPES[dtype], 0, q.data_ptr(), qs.data_ptr(), w.data_ptr(), ws.data_ptr(), 0, y.data_ptr(), q.stride(0), w.stride(0), y.stride(0))
    need = ctypes.c_int64()
    assert L.bmgd_quantized_linear_workspace_bytes(args, ctypes.byref(need)) == 0
    space = torch.empty(max(need.value, 256), dtype=torch.uint8, device="cuda")
    assert L.bmgd_quantized_linear(args, space.data_ptr(), need.value, stream()) == 0
    assert torch.equal(y, want)


@pytest.mark.parametrize("dtype", DTYPES, ids=NAMES)
@pytest.mark.parametrize("n,C", [(5, 30), (40, 3001), (3, 50257)])
def test_gradient_of_log_probabilities(n, C, dtype):
    z, dz = Wide(n, [(dtype, C), (dtype, C)]).tensors
    z.copy_(torch.randn(n, C, device="cuda"))
    y = torch.randint(0, C, (n,), device="cuda", dtype=torch.int32)
    one = torch.ones(n, device="cuda")
    saved = ops.log_probs(z, y, save=True)[4]
    want = ops.log_probs_backward(one, one, z, y, saved)
    args = ops._LOG_PROBS.pack(n, C, ops._TYPES[dtype], 0, 0, z.data_ptr(), y.data_ptr(), 0, 0, saved.data_ptr(), 0, 0, z.stride(0), one.data_ptr(), one.data_ptr(), dz.data_ptr(),
                               dz.stride(0))
    assert binding.load_library().bmgd_log_probs_backward(args, stream()) == 0
    assert torch.equal(dz, want)


@pytest.mark.parametrize("dtype", DTYPES, ids=NAMES)
@pytest.mark.parametrize("n,d", [(5, 64), (70, 501)])
def test_dropout(n, d, dtype):
    x, r, y = Wide(n, [(dtype, d)] * 3).tensors
    x.copy_(torch.randn(n, d, device="cuda")), r.copy_(torch.randn(n, d, device="cuda"))
    want = ops.dropout(x, 0.3, 9, residual=r)
    args = ops._DROPOUT.pack(n, d, ops._TYPES[dtype], 0, 0.3, 9, 0, x.data_ptr(), r.data_ptr(), y.data_ptr(), x.stride(0), r.stride(0), y.stride(0))
    assert binding.load_library().bmgd_dropout(args, stream()) == 0
    assert torch.equal(y, want)
