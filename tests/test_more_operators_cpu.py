"""What the norm, the products in 8 bits, the log probabilities and dropout refuse, before any pointer reaches a kernel.  No GPU needed."""
import ctypes

import pytest
import torch

from paper_2312_08728_b200 import binding, operators as ops

L = binding.load_library()
PTR = 1 << 20  # an aligned address that no call here gets as far as reading
FAR = 1 << 30


def norm(**kw):
    v = dict(rows=4, width=64, type=ops.TYPE_BF16, weight_type=ops.TYPE_F32, reserved=0, eps=1e-6, x=PTR, residual=0, weight=PTR, total=0, y=FAR, codes=0,
             scale=0, rstd=0, ld_x=64, ld_residual=64, ld_total=64, ld_y=64, ld_codes=64, dy=0, dtotal=0, dx=0, dweight=0, ld_dy=64, ld_dtotal=64, ld_dx=64)
    assert set(kw) <= set(v)
    v.update(kw)
    return ops._RMS_NORM.pack(*v.values())


BACK = dict(x=0, y=0, total=PTR, rstd=PTR, dy=2 * PTR, dx=FAR, dweight=3 * PTR)


def test_structs_match_the_header():
    assert ops._QUANTIZE_ROWS.size == 80 and ops._DROPOUT.size == 96
    assert ops._RMS_NORM.size == 192 and ops._QUANTIZED_LINEAR.size == 96 and ops._LOG_PROBS.size == 120


@pytest.mark.parametrize("kw", [
    dict(rows=-1), dict(rows=2 ** 31), dict(width=0), dict(width=2 ** 24 + 1), dict(type=3), dict(type=-1), dict(weight_type=ops.TYPE_F16), dict(reserved=1),
    dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(x=0), dict(x=PTR + 1), dict(y=FAR + 1), dict(weight=PTR + 2), dict(ld_x=63),
    dict(ld_y=63), dict(y=0), dict(codes=FAR), dict(y=0, codes=FAR), dict(scale=PTR), dict(y=0, codes=FAR, scale=PTR, ld_codes=63), dict(residual=2 * PTR),
    dict(total=2 * PTR), dict(residual=2 * PTR, total=3 * PTR, ld_residual=63), dict(residual=2 * PTR, total=3 * PTR, ld_total=63), dict(rstd=PTR + 2),
    dict(y=PTR), dict(y=PTR + 64), dict(residual=2 * PTR, total=2 * PTR), dict(residual=2 * PTR, total=PTR), dict(residual=2 * PTR, total=FAR + 128),
    dict(y=0, codes=PTR + 16, scale=FAR), dict(residual=2 * PTR + 1, total=3 * PTR),
])
def test_norm_forward(kw):
    assert L.bmgd_rms_norm_forward(norm(**kw), None) == binding.ERR_ARG


@pytest.mark.parametrize("kw", [
    dict(rows=-1), dict(total=0), dict(dy=0), dict(dx=0), dict(rstd=0), dict(dweight=0), dict(weight=0), dict(ld_total=63), dict(ld_dy=63), dict(ld_dx=63),
    dict(dtotal=4 * PTR, ld_dtotal=63), dict(dx=PTR), dict(dx=2 * PTR + 64), dict(dtotal=FAR + 64), dict(dweight=3 * PTR + 2), dict(rstd=PTR + 1),
])
def test_norm_backward(kw):
    assert L.bmgd_rms_norm_backward(norm(**{**BACK, **kw}), PTR, 1 << 40, None) == binding.ERR_ARG


def test_norm_workspace():
    need = ctypes.c_int64()
    args = norm(**BACK)
    assert L.bmgd_rms_norm_workspace_bytes(args, ctypes.byref(need)) == 0 and need.value >= 64 * 4
    assert L.bmgd_rms_norm_backward(args, None, 1 << 40, None) == binding.ERR_ARG
    assert L.bmgd_rms_norm_backward(args, PTR + 128, 1 << 40, None) == binding.ERR_ARG
    assert L.bmgd_rms_norm_backward(args, PTR, need.value - 1, None) == binding.ERR_CAPACITY
    assert L.bmgd_rms_norm_workspace_bytes(args, None) == binding.ERR_ARG and L.bmgd_rms_norm_workspace_bytes(None, ctypes.byref(need)) == binding.ERR_ARG
    assert L.bmgd_rms_norm_workspace_bytes(norm(**{**BACK, "weight": 0, "dweight": 0}), ctypes.byref(need)) == 0 and need.value == 0
    for width in (1, 64, 501, 4096, 20000, 100_000):
        for rows in (1, 7, 100_000):
            assert L.bmgd_rms_norm_workspace_bytes(norm(**{**BACK, "rows": rows, "width": width}), ctypes.byref(need)) == 0
            assert width * 4 <= need.value <= 800 * (width + 64) * 4
    assert L.bmgd_rms_norm_forward(norm(rows=0, x=0, y=0), None) == 0


@pytest.mark.parametrize("kw", [
    dict(rows=-1), dict(rows=2 ** 31), dict(width=0), dict(width=2 ** 24 + 1), dict(type=3), dict(activation=4), dict(activation=-1), dict(reserved=1), dict(x=0), dict(codes=0),
    dict(scale=0), dict(ld_x=63), dict(ld_codes=63), dict(gate=2 * PTR, ld_gate=63), dict(x=PTR + 1), dict(gate=2 * PTR + 1), dict(scale=PTR + 2),
    dict(codes=PTR + 10), dict(gate=FAR + 5),
])
def test_quantize_rows(kw):
    v = dict(rows=4, width=64, type=ops.TYPE_BF16, activation=0, reserved=0, x=PTR, gate=0, codes=FAR, scale=3 * PTR, ld_x=64, ld_gate=64, ld_codes=64)
    assert set(kw) <= set(v)
    v.update(kw)
    assert L.bmgd_quantize_rows(ops._QUANTIZE_ROWS.pack(*v.values()), None) == binding.ERR_ARG
    v.update(rows=0)
    if not set(kw) & {"rows", "width", "type", "activation", "reserved"}:
        assert L.bmgd_quantize_rows(ops._QUANTIZE_ROWS.pack(*v.values()), None) == 0
    assert L.bmgd_quantize_rows(None, None) == binding.ERR_ARG


@pytest.mark.parametrize("kw", [
    dict(inputs=0), dict(outputs=0), dict(inputs=2 ** 24 + 1), dict(type=3), dict(w=None), dict(codes=None), dict(scale=None), dict(ld_w=31), dict(ld_codes=63),
    dict(w=PTR + 1), dict(scale=PTR + 2), dict(codes=PTR + 100),
])
def test_quantize_weight(kw):
    v = dict(w=PTR, ld_w=32, inputs=64, outputs=32, type=ops.TYPE_BF16, codes=FAR, ld_codes=64, scale=3 * PTR)
    v.update(kw)
    assert L.bmgd_quantize_weight(*v.values(), None) == binding.ERR_ARG


def linear(**kw):
    v = dict(rows=4, inputs=64, outputs=32, type=ops.TYPE_BF16, reserved=0, codes=PTR, scale=PTR, weight=2 * PTR, weight_scale=PTR, bias=0, y=FAR, ld_codes=64, ld_weight=64,
             ld_y=32)
    assert set(kw) <= set(v)
    v.update(kw)
    return ops._QUANTIZED_LINEAR.pack(*v.values())


@pytest.mark.parametrize("kw", [
    dict(rows=-1), dict(rows=2 ** 31), dict(inputs=0), dict(inputs=131072, ld_codes=131072, ld_weight=131072), dict(outputs=0), dict(outputs=2 ** 24 + 1, ld_y=2 ** 25), dict(type=3), dict(reserved=1),
    dict(codes=0), dict(scale=0), dict(weight=0), dict(weight_scale=0), dict(y=0), dict(ld_codes=63), dict(ld_weight=63), dict(ld_y=31), dict(scale=PTR + 2),
    dict(weight_scale=PTR + 1), dict(bias=PTR + 2), dict(y=FAR + 1), dict(type=ops.TYPE_F32, y=FAR + 2),
    dict(y=PTR), dict(y=PTR + 200), dict(y=2 * PTR + 1024), dict(y=2 * PTR - 100),
])
def test_quantized_linear(kw):
    assert L.bmgd_quantized_linear(linear(**kw), PTR, 1 << 40, None) == binding.ERR_ARG


def test_quantized_linear_workspace():
    need = ctypes.c_int64(-1)

    def bytes_of(**kw):
        assert L.bmgd_quantized_linear_workspace_bytes(linear(**kw), ctypes.byref(need)) == 0
        return need.value
    many = dict(rows=2000, outputs=1000, ld_y=1000)      # (few tokens, or few tiles, are read on any boundary)
    assert bytes_of() == 0 and bytes_of(rows=500) == 0 and bytes_of(ld_codes=65, ld_weight=65) == 0 and bytes_of(**many) == 0
    assert bytes_of(**many, ld_codes=65) >= 2000 * 64 and bytes_of(**many, ld_weight=65) >= 1000 * 64 and bytes_of(**many, weight=2 * PTR + 1) >= 1000 * 64
    assert bytes_of(**many, inputs=63, ld_codes=63, ld_weight=63) >= 3000 * 64
    odd = linear(**many, ld_codes=65)
    assert L.bmgd_quantized_linear_workspace_bytes(odd, ctypes.byref(need)) == 0
    assert L.bmgd_quantized_linear(odd, None, 1 << 40, None) == binding.ERR_ARG
    assert L.bmgd_quantized_linear(odd, PTR + 16, 1 << 40, None) == binding.ERR_ARG
    assert L.bmgd_quantized_linear(odd, PTR, need.value - 1, None) == binding.ERR_CAPACITY
    assert L.bmgd_quantized_linear(linear(rows=0), None, 0, None) == 0
    assert L.bmgd_quantized_linear(None, None, 0, None) == binding.ERR_ARG and L.bmgd_quantized_linear_workspace_bytes(linear(), None) == binding.ERR_ARG
    for fills, budget in ((-1, 1.0), (0, 0.0), (0, -1.0), (0, 2000.0), (0, float("nan"))):
        assert L.bmgd_debug_quantized_linear_timeout(linear(), None, 0, fills, budget, None) == binding.ERR_ARG


def score(**kw):
    v = dict(rows=4, C=30, type=ops.TYPE_BF16, top=0, reserved=0, logits=PTR, y=PTR, logprob=FAR, entropy=FAR, saved=FAR, top_class=0, top_logprob=0, ld_logits=30,
             dlogprob=PTR, dentropy=PTR, dlogits=FAR, ld_dlogits=30)
    assert set(kw) <= set(v)
    v.update(kw)
    return ops._LOG_PROBS.pack(*v.values())


BAD_SCORES = [dict(rows=-1), dict(rows=2 ** 31), dict(C=0), dict(C=2 ** 30 + 1), dict(type=3), dict(top=-1), dict(top=33), dict(C=4, top=5), dict(reserved=1), dict(logits=0),
              dict(logits=PTR + 1), dict(ld_logits=29), dict(y=PTR + 2), dict(logprob=PTR + 1), dict(entropy=PTR + 2), dict(saved=FAR + 1)]


@pytest.mark.parametrize("kw", BAD_SCORES + [dict(top=3), dict(top=3, top_class=FAR), dict(top=3, top_class=FAR, top_logprob=FAR + 2)])
def test_log_probs(kw):
    assert L.bmgd_log_probs(score(**kw), None) == binding.ERR_ARG


@pytest.mark.parametrize("kw", BAD_SCORES + [dict(saved=0), dict(dlogits=0), dict(dlogits=FAR + 1), dict(ld_dlogits=29), dict(dlogprob=PTR + 2), dict(dentropy=PTR + 1),
                                             dict(dlogits=PTR + 2), dict(dlogits=PTR, ld_dlogits=31), dict(dlogits=PTR - 60)])
def test_log_probs_backward(kw):
    assert L.bmgd_log_probs_backward(score(**kw), None) == binding.ERR_ARG


def test_log_probs_of_nothing():
    assert L.bmgd_log_probs(score(rows=0, logits=0), None) == 0 and L.bmgd_log_probs_backward(score(rows=0, logits=0), None) == 0
    assert L.bmgd_log_probs(None, None) == binding.ERR_ARG and L.bmgd_log_probs_backward(None, None) == binding.ERR_ARG


@pytest.mark.parametrize("kw", [
    dict(rows=-1), dict(rows=2 ** 31), dict(width=0), dict(width=2 ** 40 + 1), dict(type=3), dict(rate=1.0), dict(rate=-0.1), dict(rate=float("nan")), dict(rate=1 - 2.0 ** -18),
    dict(layer=-1), dict(layer=65536), dict(x=0), dict(y=0), dict(ld_x=63), dict(ld_y=63), dict(residual=2 * PTR, ld_residual=63), dict(x=PTR + 1), dict(y=FAR + 1),
    dict(residual=2 * PTR + 1), dict(step=PTR + 4), dict(y=PTR + 2), dict(y=PTR, ld_y=65), dict(residual=FAR + 2), dict(rows=2 ** 30, width=2 ** 31, ld_x=2 ** 31, ld_y=2 ** 31),
])
def test_dropout(kw):
    v = dict(rows=4, width=64, type=ops.TYPE_BF16, layer=0, rate=0.1, seed=1, step=0, x=PTR, residual=0, y=FAR, ld_x=64, ld_residual=64, ld_y=64)
    assert set(kw) <= set(v)
    v.update(kw)
    assert L.bmgd_dropout(ops._DROPOUT.pack(*v.values()), None) == binding.ERR_ARG


def test_dropout_of_nothing():
    assert L.bmgd_dropout(ops._DROPOUT.pack(0, 64, ops.TYPE_BF16, 0, 0.1, 1, 0, 0, 0, 0, 64, 64, 64), None) == 0
    assert L.bmgd_dropout(None, None) == binding.ERR_ARG


@pytest.mark.parametrize("call", [
    lambda x: ops.rms_norm(x), lambda x: ops.rms_norm_int8(x), lambda x: ops.rms_norm_backward(x, x, None, x[:, 0]), lambda x: ops.quantize_rows(x),
    lambda x: ops.quantize_weight(x), lambda x: ops.int8_linear(x.to(torch.int8), x[:, 0], x.to(torch.int8), x[:, 0]), lambda x: ops.log_probs(x),
    lambda x: ops.log_probs_backward(None, None, x, None, x), lambda x: ops.dropout(x, 0.1, 0),
])
def test_there_is_no_cpu_path(call):
    with pytest.raises(ValueError, match="no CPU path"):
        call(torch.zeros(4, 4))
