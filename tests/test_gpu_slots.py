"""Buffer slots of the step kernels' handle: copies into one slot are ordered."""
import numpy as np
import pytest
import torch

from paper_2312_08728_b200.inputs import DTYPE_F32, LOSS_LINEAR

pytestmark = pytest.mark.gpu


def test_a_slot_loaded_again_on_another_stream():
    """Three loads without a round in between, on three streams, the first of them held up: the third, into the same slot, is
    behind it, and what is trained on is what was loaded last."""
    from paper_2312_08728_b200.binding import Bmgd
    rows, p = 512, 24
    gen = torch.Generator().manual_seed(0)
    parts = [(torch.randn(rows, p, generator=gen).pin_memory(), torch.randn(rows, generator=gen).pin_memory()) for _ in range(3)]
    with Bmgd(2 * rows, p, 2, loss=LOSS_LINEAR, dtype=DTYPE_F32) as h:
        streams = [torch.cuda.Stream() for _ in range(3)]
        torch.cuda.synchronize()
        with torch.cuda.stream(streams[0]):
            torch.cuda._sleep(100_000_000)
        slots = [h.load_buffer(*part, stream=s) for part, s in zip(parts, streams)]
        assert slots == [0, 1, 0]
        torch.cuda.synchronize()
        h.run_rounds(0, 2, 64, 0.05, 7)
        got = h.get_theta()
    with Bmgd(2 * rows, p, 2, loss=LOSS_LINEAR, dtype=DTYPE_F32) as h:
        h.run_rounds_resident(parts[2][0].cuda(), parts[2][1].cuda(), 2, 64, 0.05, 7)
        want = h.get_theta()
    assert np.array_equal(got, want)
