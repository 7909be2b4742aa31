"""What a product in 8 bits whose waits run out has computed, shape by shape: a limited number of fetches per block reaches a whole tile, a part of one, or the first
of a block's tiles only."""
import pytest
import torch

from paper_2312_08728_b200 import binding
from paper_2312_08728_b200 import operators as ops
from test_gpu_int8_linear import operands, starve

pytestmark = pytest.mark.gpu

ALL, NONE, LATER = "all of it", "nothing", "what comes after the first tiles"
# what is lost with 1 fetch of 128 inputs and with 8: contractions of 16 steps over at most 8 blocks, of one step, of 4 and 8 steps by one block for each tile, and
# of 8 steps with more tiles than blocks (135 of 256 x 192 for 74 pairs at most)
SHAPES = [((3, 2048, 1376), ALL, NONE), ((100, 128, 136), NONE, NONE), ((700, 512, 2700), ALL, NONE), ((2304, 1024, 2816), ALL, LATER), ((2048, 1024, 2048), ALL, NONE),
          ((3, 2047, 1376), ALL, NONE), ((100, 127, 136), NONE, NONE)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("shape,one,eight", SHAPES, ids=lambda s: "x".join(map(str, s)) if isinstance(s, tuple) else "")
def test_what_is_lost(shape, one, eight, dtype):
    job = operands(*shape, seed=4)
    want = ops.int8_linear(*job, dtype=dtype)
    ops.stream_check()
    for fills, lost in ((0, ALL), (1, one), (8, eight)):
        got = starve(job, fills, dtype)
        nan = torch.isnan(got)
        assert torch.equal(got[~nan], want[~nan])
        if lost == NONE:
            assert not nan.any()
            ops.stream_check()
            continue
        with pytest.raises(binding.BmgdError):
            ops.stream_check()
        if lost == ALL:
            assert bool(nan.all())
            continue
        # the first tiles stand, one to a pair of blocks, as whole tiles; those after them are gone
        pairs = torch.cuda.get_device_properties(0).multi_processor_count // 2
        tiles_m, tiles_n = -(-shape[0] // 256), -(-shape[2] // 192)
        whole = torch.zeros(tiles_m * 256, tiles_n * 192, dtype=torch.bool, device="cuda")
        whole[:shape[0], :shape[2]] = ~nan
        inner = torch.zeros_like(whole)
        inner[:shape[0], :shape[2]] = True
        tile = lambda t: t.view(tiles_m, 256, tiles_n, 192).permute(0, 2, 1, 3).reshape(tiles_m * tiles_n, -1)
        stands, cells = tile(whole).sum(dim=1), tile(inner).sum(dim=1)
        assert bool(((stands == 0) | (stands == cells)).all())
        assert int((stands > 0).sum()) == min(pairs, tiles_m * tiles_n) < tiles_m * tiles_n and int(stands[0]) == 256 * 192
    ops.stream_check()
