"""Tensors that carry a tangent of forward-mode differentiation are refused where the result would have none.  No GPU needed."""
import pytest
import torch
from torch.autograd import forward_ad

from paper_2312_08728_b200 import operators as ops


def test_dual_tensors():
    x = torch.randn(3, 4)
    ops._no_graph("f", x, None)
    with forward_ad.dual_level():
        ops._no_graph("f", x, None)
        dual = forward_ad.make_dual(x, torch.ones_like(x))
        for context in (torch.enable_grad(), torch.no_grad()):
            with context:
                for tensors in ((dual,), (x, None, dual), (dual[1:],)):
                    with pytest.raises(ValueError, match="graph"):
                        ops._no_graph("f", *tensors)
        ops._no_graph("f", forward_ad.unpack_dual(dual).primal)
    ops._no_graph("f", x)


def test_gradients():
    x = torch.randn(3, 4, requires_grad=True)
    with pytest.raises(ValueError, match="graph"):
        ops._no_graph("f", None, x)
    with torch.no_grad():
        ops._no_graph("f", x)
    ops._no_graph("f", x.detach())
