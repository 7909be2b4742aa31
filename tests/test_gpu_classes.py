"""Alternatives of rows with some hundred classes: fewer pieces of 16 bytes than 32, so that few parts of the row have a maximum, and more classes than there are places
for candidates."""
import pytest
import torch

from test_gpu_log_probs import check, check_backward
from test_gpu_norm import rows_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32], ids=["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("C", [127, 159, 160, 161, 176, 200, 255, 256, 257])
def test_some_hundred_classes(C, dtype):
    gen = torch.Generator(device="cuda").manual_seed(C)
    for rows, extra in ((3, 0), (700, 0), (60, 3)):
        z = rows_of(gen, rows, C, dtype, extra, scale=3.0)
        y = torch.randint(0, C, (rows,), generator=gen, device="cuda", dtype=torch.int32)
        for top in (5, 20, 21, 32):
            saved, logp, entropy = check(z, y, top)
        check_backward(z, y, torch.randn(rows, generator=gen, device="cuda"), torch.randn(rows, generator=gen, device="cuda"), saved, logp, entropy)
