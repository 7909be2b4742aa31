"""What autograd is told of the operators: they record no graph, and an update in place is seen by graphs that saved the tensor."""
import pytest
import torch

from paper_2312_08728_b200 import operators as ops

pytestmark = pytest.mark.gpu

BF = dict(dtype=torch.bfloat16, device="cuda")


@pytest.mark.parametrize("which", range(4))
def test_the_block_refuses_to_drop_a_graph(which):
    tensors = [torch.randn(s, **BF) for s in ((5, 16), (16, 24), (16, 24), (24, 8))]
    want = ops.gated_ffn(*tensors)
    tensors[which].requires_grad_()
    with pytest.raises(ValueError, match="autograd"):
        ops.gated_ffn(*tensors)
    with torch.no_grad():
        y, saved = ops.gated_ffn(*tensors, save=True)
    assert torch.equal(y, want)
    grads = ops.gated_ffn_backward(torch.ones_like(y), *tensors, saved)  # explicit gradients, in either mode
    assert not any(g.requires_grad for g in grads)
