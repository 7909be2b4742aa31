"""The operators where offsets pass 32 bits: the last rows, or values, against their definitions."""
import pytest
import torch

from paper_2312_08728_b200 import operators as ops
from test_gpu_operators import Block, check_residual

pytestmark = pytest.mark.gpu


def test_gated_block():
    """140,000 rows by 16,384 hidden units: 2.3e9 values.  The last rows stand for all (their inputs differ from the others'), and
    the weights' gradients, with the gradient of Y zero but for the last rows, are theirs alone."""
    rows, d, f, c, last = 140_000, 40, 16_384, 24, 300
    b = Block(rows, d, f, c, torch.bfloat16, ops.ACT_SILU, seed=2)
    b.dy[:-last] = 0
    got = b.run()
    tail = Block.__new__(Block)
    tail.x, tail.dy, tail.wg, tail.wu, tail.wd, tail.act, tail.dtype = b.x[-last:], b.dy[-last:], b.wg, b.wu, b.wd, b.act, b.dtype
    assert not got["dx"][:-last].any()
    got["y"], got["dx"] = got["y"][-last:], got["dx"][-last:]
    tail.check(got)


def test_residual():
    rows, C = 43_100, 50_001
    assert rows * C > 2 ** 31
    z = torch.zeros(rows, C, dtype=torch.bfloat16, device="cuda")
    z[-5:] = torch.randn(5, C, device="cuda").bfloat16() * 3
    y = torch.full((rows,), -1, dtype=torch.int32, device="cuda")
    y[-5:] = torch.randint(0, C, (5,), device="cuda", dtype=torch.int32)
    residual, loss = ops.softmax_residual(z, y, scale=1.0)
    assert not loss[:-5].any() and not residual[-6].any() and not residual[0].any()
    want, want_loss = check_residual(z[-5:].contiguous(), y[-5:].contiguous(), scale=1.0)
    # (the small call may take another form of the kernel: both are within the bound that check_residual tests)
    assert torch.allclose(residual[-5:].float(), want.float(), rtol=2.0 ** -7, atol=1e-7) and torch.allclose(loss[-5:], want_loss, rtol=1e-5)


@pytest.mark.parametrize("bits", [8, 32])
def test_adamw(bits):
    n, last = 2 ** 31 + 1000, 5000
    p = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    g = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    p[-last:] = torch.randn(last, device="cuda").bfloat16()
    g[-last:] = torch.randn(last, device="cuda").bfloat16()
    s = ops.adamw_state([p], bits)
    before = p[-last:].double()
    ops.adamw_step([p], [g], lr=1e-2, weight_decay=0.1, max_norm=1e9, seed=1, **s)
    # the first update: m / sqrt(v) is the gradient's sign
    want = before * (1 - 1e-3) - 1e-2 * torch.sign(g[-last:].double())
    assert bool(((p[-last:].double() - want).abs() <= 2.0 ** -7 * want.abs() + 1e-5).all())
    assert not p[:1000].any() and not p[-last - 1000:-last].any() and not s["m"][0].view(torch.uint8)[:1000].any()
    assert s["control"].tolist()[:3] == [1, 0, 0]
    norm = float(g[-last:].double().square().sum().sqrt())
    assert abs(s["control"][3:].view(torch.float64).item() / norm - 1) < 1e-12
