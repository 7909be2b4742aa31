"""The gradient of log probabilities in the logits' own memory, through the C call: the same bits as beside them."""
import pytest
import torch

from paper_2312_08728_b200 import binding
from paper_2312_08728_b200 import operators as ops
from test_gpu_norm import rows_of

pytestmark = pytest.mark.gpu


def backward(z, y, saved, dl, de, out):
    args = ops._LOG_PROBS.pack(*z.shape, ops._TYPES[z.dtype], 0, 0, z.data_ptr(), y.data_ptr(), 0, 0, saved.data_ptr(), 0, 0, z.stride(0), dl.data_ptr(), de.data_ptr(),
                               out.data_ptr(), out.stride(0))
    return binding.load_library().bmgd_log_probs_backward(args, torch.cuda.current_stream().cuda_stream)


# a warp to a row, 256 threads to a row, several blocks of 256 to a row, 512 threads
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32], ids=["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("rows,C", [(7, 10), (50, 900), (700, 5001), (9, 50257), (3, 131072), (650, 40007)])
@pytest.mark.parametrize("extra,shift", [(0, 0), (3, 1)])
def test_gradient_in_place(rows, C, extra, shift, dtype):
    gen = torch.Generator(device="cuda").manual_seed(C)
    z = rows_of(gen, rows, C, dtype, extra, shift, scale=3.0)
    y = torch.randint(0, C, (rows,), generator=gen, device="cuda", dtype=torch.int32)
    z[0] = -float("inf")
    z[1, C // 2] = float("nan")
    y[2] = -1
    dl, de = torch.randn(rows, generator=gen, device="cuda"), torch.randn(rows, generator=gen, device="cuda")
    saved = ops.log_probs(z, y, save=True)[4]
    apart = torch.empty_strided(z.shape, z.stride(), dtype=dtype, device="cuda")
    assert backward(z, y, saved, dl, de, apart) == 0
    assert not apart[0].any() and bool(torch.isnan(apart[1]).all())
    whole = torch.as_strided(z, (rows * z.stride(0) - extra,), (1,))       # what stands between the rows is left as it was
    between = whole.clone()
    assert backward(z, y, saved, dl, de, z) == 0
    bits = torch.int32 if dtype is torch.float32 else torch.int16
    assert torch.equal(z.contiguous().view(bits), apart.contiguous().view(bits))
    torch.as_strided(between, z.shape, z.stride()).copy_(z)
    assert torch.equal(whole.view(bits), between.view(bits))
