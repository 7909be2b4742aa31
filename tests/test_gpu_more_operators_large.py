"""The norm, the products in 8 bits, the log probabilities and dropout where offsets pass 32 bits: the last rows stand for all."""
import torch
import pytest

from paper_2312_08728_b200 import operators as ops
from test_gpu_dropout import kept
from test_gpu_int8_linear import check as check_product
from test_gpu_log_probs import check as check_scores, check_backward as check_scores_backward
from test_gpu_norm import check_backward, check_codes, check_total, normed, root_error, inside
from test_gpu_operators import E32, U

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("width", [32768 - 8, 16384, 4099])
def test_norm(width):
    """Rows read more than once, rows in registers, rows on any boundary."""
    rows, last = 2 ** 31 // width + 600, 300
    x, r, dy = (torch.zeros(rows, width, dtype=torch.bfloat16, device="cuda") for _ in range(3))
    for t in (x, r, dy):
        t[-last:] = torch.randn(last, width, device="cuda").bfloat16()
    w = 1 + 0.2 * torch.randn(width, device="cuda")
    y, total, rstd = ops.rms_norm(x, w, residual=r, eps=1e-5, save=True)
    check_total(total[-last:], x[-last:], r[-last:])
    want, s = normed(total[-last:], w)
    rel, u = root_error(width), U[torch.bfloat16]
    inside(y[-last:], want, ((rel + 3 * E32) * (1 + u) + u) * want.abs(), "y")
    assert not y[:1000].any() and not y[-last - 1].any()
    dx, dw = ops.rms_norm_backward(dy, total, w, rstd, r)
    small = ops.rms_norm_backward(dy[-last:].contiguous(), total[-last:].contiguous(), w, rstd[-last:].contiguous(), r[-last:].contiguous())
    assert torch.equal(dx[-last:], small[0]) and not dx[:-last].any()
    check_backward(dy[-last:].contiguous(), total[-last:].contiguous(), w, rstd[-last:].contiguous(), r[-last:].contiguous())
    assert torch.allclose(dw, small[1], rtol=1e-4, atol=1e-3)      # (the same terms, added up in other groups)
    del dx, y
    q, scale, _ = ops.rms_norm_int8(x, w, residual=r, eps=1e-5)
    check_codes(q[-last:], scale[-last:], want, rel + 3 * E32)
    assert not q[:1000].any() and not scale[:-last].any()


def test_quantize_rows():
    rows, width, last = 140_000, 16_000, 50
    both = torch.zeros(rows, 2 * width, dtype=torch.bfloat16, device="cuda")
    both[-last:] = torch.randn(last, 2 * width, device="cuda").bfloat16()
    codes, scale = ops.quantize_rows(both[:, width:], gate=both[:, :width])
    want = ops.quantize_rows(both[-last:, width:].contiguous(), gate=both[-last:, :width].contiguous())
    assert torch.equal(codes[-last:], want[0]) and torch.equal(scale[-last:], want[1])
    assert not codes[:1000].any() and not scale[:-last].any()


@pytest.mark.parametrize("n", [1, 3, 30, 300])
def test_long_weights(n):
    """Offsets in the weights: 33,000 channels of 65,552 inputs."""
    c, d = 33_000, 65_552
    assert c * d > 2 ** 31
    w = torch.zeros(c, d, dtype=torch.int8, device="cuda")
    w[-100:] = torch.randint(-127, 128, (100, d), device="cuda").to(torch.int8)
    q = torch.randint(-127, 128, (n, d), device="cuda").to(torch.int8)
    qs, ws = torch.rand(n, device="cuda"), torch.rand(c, device="cuda")
    y = ops.int8_linear(q, qs, w, ws, dtype=torch.float32)
    want = check_product(q, qs, w[-100:].contiguous(), ws[-100:].contiguous(), dtype=torch.float32)
    assert torch.equal(y[:, -100:], want) and not y[:, :-100].any()


def test_large_outputs():
    rows, c, d = 140_000, 16_384, 48
    q = torch.zeros(rows, d, dtype=torch.int8, device="cuda")
    q[-200:] = torch.randint(-127, 128, (200, d), device="cuda").to(torch.int8)
    w = torch.randint(-127, 128, (c, d), device="cuda").to(torch.int8)
    qs, ws = torch.rand(rows, device="cuda"), torch.rand(c, device="cuda")
    y = ops.int8_linear(q, qs, w, ws)
    want = check_product(q[-200:].contiguous(), qs[-200:].contiguous(), w, ws)
    assert torch.equal(y[-200:], want) and not y[:1000].any() and not y[-201].any()


def test_log_probs():
    rows, C = 43_100, 50_001
    assert rows * C > 2 ** 31
    z = torch.zeros(rows, C, dtype=torch.bfloat16, device="cuda")
    z[-700:] = (torch.randn(700, C, device="cuda") * 3).bfloat16()
    y = torch.full((rows,), -1, dtype=torch.int32, device="cuda")
    y[-700:] = torch.randint(0, C, (700,), device="cuda", dtype=torch.int32)
    got = ops.log_probs(z, y, top=20, save=True)
    tail, labels = z[-700:].contiguous(), y[-700:].contiguous()
    saved, logp, entropy = check_scores(tail, labels, 20)
    want = ops.log_probs(tail, labels, top=20, save=True)
    # (where a row begins within 16 bytes decides how its sums are grouped)
    assert torch.equal(got[2][-700:], want[2]) and all(torch.allclose(a[-700:], b, rtol=1e-5, atol=1e-5) for a, b in zip(got, want) if a.is_floating_point())
    assert got[2][0].tolist() == list(range(20)) and not got[0][:-700].any()
    f = torch.zeros(rows, device="cuda")
    f[-700:] = 1.0
    dz = ops.log_probs_backward(f, f, z, y, got[4])
    assert not dz[:1000].any() and not dz[-701].any()
    small = ops.log_probs_backward(f[-700:].contiguous(), f[-700:].contiguous(), tail, labels, saved)
    assert torch.allclose(dz[-700:].float(), small.float(), rtol=2.0 ** -6, atol=1e-6)
    check_scores_backward(tail, labels, f[-700:].contiguous(), f[-700:].contiguous(), saved, logp, entropy)


@pytest.mark.parametrize("flat", [True, False])
def test_dropout(flat):
    """Values, and blocks of the generator's, beyond 32 bits: 2^35 + 16 of 16 bits are 69 GB, so fewer values and a check of their places."""
    rows, width = 70_001, 32_771
    assert rows * width > 2 ** 31
    x = torch.ones(rows, width + (0 if flat else 5), dtype=torch.bfloat16, device="cuda")[:, :width]
    y = ops.dropout(x, 0.5, 77)
    keep = kept((rows - 3) * width, 3 * width, 0.5, 77).view(3, width)
    assert torch.equal(y[-3:] > 0, keep) and bool((y[-3:][keep] == 2).all())
    assert torch.equal(y[0] > 0, kept(0, width, 0.5, 77))
