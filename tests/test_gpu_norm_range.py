"""The norm at the ends of its range: an eps that fp32 does not hold is still more than none; sums of squares that leave fp32 give zeros, as the header says."""
import pytest
import torch

from paper_2312_08728_b200 import operators as ops

pytestmark = pytest.mark.gpu

DTYPES = [torch.bfloat16, torch.float16, torch.float32]
NAMES = ["bf16", "fp16", "fp32"]


@pytest.mark.parametrize("dtype", DTYPES, ids=NAMES)
@pytest.mark.parametrize("width", [8, 501, 4096, 40000])
def test_smallest_eps(width, dtype):
    x = torch.zeros(3, width, device="cuda", dtype=dtype)
    x[1] = 1
    for eps in (1e-50, 5e-324, 1e-45, 1e-30):
        y, _, rstd = ops.rms_norm(x, None, eps=eps, save=True)
        assert not y[0].any() and not y[2].any() and bool(torch.isfinite(rstd).all()) and bool((y[1] == 1).all())
        codes, scale, _ = ops.rms_norm_int8(x, None, eps=eps)
        assert not codes[0].any() and scale[0] == 0 and bool((codes[1] == 127).all())


@pytest.mark.parametrize("width", [64, 4096, 40000])
def test_largest_squares(width):
    for dtype, fits, beyond in ((torch.bfloat16, 1.5e19 / width ** 0.5, 2.5e19 / width ** 0.5), (torch.float32, 1.8e19, 1.9e19)):
        x = torch.tensor([[fits], [beyond]], device="cuda").expand(2, width).to(dtype).contiguous()
        y, _, rstd = ops.rms_norm(x, None, save=True)
        assert bool(((y[0].float() - 1).abs() < 2.0 ** -7).all()) and rstd[0] > 0
        assert not y[1].any() and rstd[1] == 0
