"""Waits of the gated block's kernels that run out of time: what the caller sees, and that nobody else does.

Nothing is hung: the kernels are told to fetch only part of their operands, and give up waiting for the rest after a few
milliseconds."""
import ctypes

import pytest
import torch

from paper_2312_08728_b200 import binding
from paper_2312_08728_b200 import operators as ops
from test_gpu_operators import Block

pytestmark = pytest.mark.gpu

# the form for few rows (split over a cluster and not), tiles of one CTA, tiles of CTA pairs
SHAPES = [(3, 512, 1376, 512), (100, 64, 136, 40), (700, 256, 264, 136), (2304, 1024, 2816, 1024)]


def starve(b, fills, budget_ms=5.0):
    """Both passes of a block whose kernels fetch `fills` pieces per CTA; the outputs' memory is zero before."""
    L = binding.load_library()
    w = (b.wg, b.wu, b.wd)
    shared, (n, d, f, c), _ = ops._ffn_args(b.x, *w, b.act)
    width = (f + 7) // 8 * 8
    out = {"y": b.x.new_zeros(n, c), "dx": b.x.new_zeros(n, d), "dw_gate": b.x.new_zeros(d, f), "dw_up": b.x.new_zeros(d, f), "dw_down": b.x.new_zeros(f, c)}
    saved = b.x.new_zeros(n, 5 * width)
    kept = ops._saved_args(saved, n, width)
    forward = ops._GATED_FFN.pack(*shared, out["y"].data_ptr(), c, *kept, 0, 0, 0, 0, 0, 0)
    _, good = ops.gated_ffn(b.x, *w, b.act, save=True)  # the backward pass is starved by itself
    backward = ops._GATED_FFN.pack(*shared, 0, 0, *ops._saved_args(good, n, width), b.dy.data_ptr(), b.dy.stride(0),
                                   *(out[k].data_ptr() for k in ("dx", "dw_gate", "dw_up", "dw_down")))
    for which, args in ((0, forward), (1, backward)):
        need = ctypes.c_int64()
        assert L.bmgd_gated_ffn_workspace_bytes(args, which, ctypes.byref(need)) == 0
        space = torch.empty(max(need.value, 1), dtype=torch.uint8, device="cuda")
        assert L.bmgd_debug_gated_ffn_timeout(args, which, space.data_ptr(), need.value, fills, budget_ms, torch.cuda.current_stream().cuda_stream) == 0
        torch.cuda.synchronize()
    return out


@pytest.mark.parametrize("dtype,act", [(torch.bfloat16, ops.ACT_SILU), (torch.float16, ops.ACT_RELU)], ids=["bf16-silu", "fp16-relu"])
@pytest.mark.parametrize("fills", [0, 1, 8])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_what_was_not_computed_is_nan(shape, fills, dtype, act):
    """No output keeps what its memory held, or holds a part of a sum: each is right or NaN."""
    b = Block(*shape, dtype, act, seed=2)
    want = b.run()
    got = starve(b, fills)
    for k in want:
        lost = torch.isnan(got[k])
        assert bool((lost | (got[k] == want[k])).all()), k
        assert fills > 0 or bool(lost.all()), k
    if not any(bool(torch.isnan(got[k]).any()) for k in want):
        assert fills == 8                      # everything could be fetched
        ops.stream_check()
    else:
        with pytest.raises(binding.BmgdError):
            ops.stream_check()


@pytest.mark.parametrize("fills", [0, 1, 2])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_a_wait_that_runs_out_touches_no_other_call(shape, fills):
    b = Block(*shape, torch.bfloat16, ops.ACT_SILU, seed=1)
    want = b.run()
    ops.stream_check()
    starve(b, fills)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for got in (b.run(), b.run(stream=side)):  # nobody has asked for the report yet
        torch.cuda.synchronize()
        for k in want:
            assert torch.equal(got[k], want[k]), k
    with pytest.raises(binding.BmgdError):
        ops.stream_check()
    ops.stream_check()                         # reported once


def test_every_wait_that_runs_out_is_reported():
    b = Block(3, 64, 64, 8, torch.bfloat16, ops.ACT_SILU)
    for _ in range(3):
        starve(b, 0, 1.0)
        with pytest.raises(binding.BmgdError):
            ops.stream_check(torch.cuda.Stream())  # any stream of the device
        ops.stream_check()


def test_refusals():
    L = binding.load_library()
    b = Block(3, 64, 64, 8, torch.bfloat16, ops.ACT_SILU)
    shared, (n, _, _, c), _ = ops._ffn_args(b.x, b.wg, b.wu, b.wd, b.act)
    args = ops._GATED_FFN.pack(*shared, torch.empty(n, c, device="cuda", dtype=torch.bfloat16).data_ptr(), c, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0)
    for fills, budget in ((-1, 1.0), (0, 0.0), (0, -1.0), (0, 2000.0), (0, float("nan"))):
        assert L.bmgd_debug_gated_ffn_timeout(args, 0, None, 0, fills, budget, None) == -1
