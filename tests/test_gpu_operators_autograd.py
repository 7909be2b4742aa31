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


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("master", [False, True])
def test_a_graph_that_saved_a_weight_sees_its_update(bits, master):
    w = torch.randn(16, 16, **BF, requires_grad=True)
    copies = [w.detach().float().requires_grad_()] if master else None
    x = torch.randn(4, 16, **BF, requires_grad=True)
    loss = (x @ w).sum() + ((x.float() @ copies[0]).sum() if master else 0)
    grad, state = torch.randn(16, 16, **BF), ops.adamw_state([w], bits)
    versions = w._version, copies[0]._version if master else None
    ops.adamw_step([w], [grad], lr=1e-2, masters=copies, **state)
    assert w._version > versions[0] and (not master or copies[0]._version > versions[1])
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()
    (x @ w).sum().backward()                   # a graph of the new weight


def test_weights_made_in_inference_mode_are_updated():
    with torch.inference_mode():
        w = torch.zeros(300, device="cuda")
        state = ops.adamw_state([w])
    ops.adamw_step([w], [torch.ones(300, device="cuda")], lr=1e-2, **state)
    assert torch.allclose(w, torch.full_like(w, -1e-2), atol=1e-6)
