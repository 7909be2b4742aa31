"""Small results that would be written over what is read, or over one another, are refused like large ones.  No pointer is followed; no GPU needed."""
import pytest

from paper_2312_08728_b200 import binding, operators as ops
from test_more_operators_cpu import BACK, FAR, PTR, L, linear, norm, score

ONE, TWO = 5 * PTR, 6 * PTR


@pytest.mark.parametrize("kw", [
    dict(rstd=PTR), dict(rstd=PTR + 4 * 128 - 4), dict(rstd=FAR + 64), dict(rstd=3 * PTR, residual=2 * PTR, total=3 * PTR), dict(rstd=2 * PTR, residual=2 * PTR, total=3 * PTR),
    dict(weight=FAR), dict(weight=FAR - 64 * 4 + 4), dict(weight=ONE, rstd=ONE + 64 * 4 - 4), dict(y=0, codes=FAR, scale=FAR + 3 * 64 + 60), dict(y=0, codes=FAR, scale=PTR),
    dict(y=0, codes=FAR, scale=ONE, rstd=ONE + 12), dict(y=0, codes=FAR, scale=ONE, weight=ONE), dict(weight=TWO, weight_type=ops.TYPE_BF16, y=TWO + 64 * 2 - 2),
])
def test_norm_forward(kw):
    assert L.bmgd_rms_norm_forward(norm(**kw), None) == binding.ERR_ARG


@pytest.mark.parametrize("kw", [
    dict(dweight=PTR), dict(dweight=2 * PTR + 4), dict(dweight=FAR), dict(dweight=FAR - 252), dict(dweight=ONE, rstd=ONE), dict(dweight=ONE, weight=ONE + 252), dict(dx=ONE, rstd=ONE + 8),
    dict(dx=ONE, weight=ONE + 4 * 128 - 4), dict(dtotal=TWO, dweight=TWO),
])
def test_norm_backward(kw):
    assert L.bmgd_rms_norm_backward(norm(**{**BACK, **kw}), 9 * PTR, 1 << 20, None) == binding.ERR_ARG


@pytest.mark.parametrize("kw", [dict(scale=PTR), dict(scale=FAR + 252), dict(gate=ONE, scale=ONE + 4 * 128 - 4), dict(scale=PTR - 12)])
def test_quantize_rows(kw):
    v = dict(rows=4, width=64, type=ops.TYPE_BF16, activation=0, reserved=0, x=PTR, gate=0, codes=FAR, scale=3 * PTR, ld_x=64, ld_gate=64, ld_codes=64)
    v.update(kw)
    assert L.bmgd_quantize_rows(ops._QUANTIZE_ROWS.pack(*v.values()), None) == binding.ERR_ARG


@pytest.mark.parametrize("scale", [PTR, PTR + 64 * 64 - 4, FAR + 32 * 64 - 4, FAR - 32 * 4 + 4])
def test_quantize_weight(scale):
    assert L.bmgd_quantize_weight(PTR, 32, 64, 32, ops.TYPE_BF16, FAR, 64, scale, None) == binding.ERR_ARG


@pytest.mark.parametrize("kw", [dict(scale=FAR), dict(weight_scale=FAR + 4 * 64 - 4), dict(bias=FAR - 124), dict(bias=FAR + 100), dict(y=ONE, scale=ONE - 12)])
def test_quantized_linear(kw):
    assert L.bmgd_quantized_linear(linear(**kw), 9 * PTR, 1 << 20, None) == binding.ERR_ARG


APART = dict(logprob=ONE, entropy=ONE + 16, saved=TWO, top_class=7 * PTR, top_logprob=8 * PTR, top=3, y=2 * PTR)


@pytest.mark.parametrize("kw", [
    dict(entropy=ONE + 12), dict(saved=ONE - 44), dict(logprob=TWO + 44), dict(top_class=8 * PTR + 44), dict(top_logprob=TWO + 40), dict(logprob=PTR), dict(entropy=PTR + 236),
    dict(saved=PTR + 100), dict(logprob=2 * PTR), dict(top_class=2 * PTR + 12), dict(top_logprob=PTR + 4), dict(top_class=ONE),
])
def test_log_probs(kw):
    assert L.bmgd_log_probs(score(**{**APART, **kw}), None) == binding.ERR_ARG


@pytest.mark.parametrize("kw", [dict(y=FAR), dict(saved=FAR + 236), dict(dlogprob=FAR + 100), dict(dentropy=FAR - 12), dict(dlogits=PTR, y=PTR + 8), dict(dlogits=PTR, dentropy=PTR + 236)])
def test_log_probs_backward(kw):
    v = dict(saved=TWO, y=ONE, dlogprob=7 * PTR, dentropy=8 * PTR)
    assert L.bmgd_log_probs_backward(score(**{**v, **kw}), None) == binding.ERR_ARG


@pytest.mark.parametrize("step", [FAR, FAR + 504])
def test_dropout(step):
    assert L.bmgd_dropout(ops._DROPOUT.pack(4, 64, ops.TYPE_BF16, 0, 0.1, 1, step, PTR, 0, FAR, 64, 64, 64), None) == binding.ERR_ARG
