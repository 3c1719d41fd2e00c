"""What holds for the layers over the training operators beside their gradients."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def block():
    from paper_2601_07876_b200 import block
    return block


def layers(block):
    """Each layer and the block of both, and the width that it takes."""
    return [(block.NormLinear8(64, 96), 64), (block.ActLinear8(96, 64), 96), (block.MlpBlock8(64, 96), 64)]


# ---- second derivatives -------------------------------------------------------------
def test_second_derivatives_are_refused(block):
    """A part of them would be missing, the operators' share."""
    for layer, width in layers(block):
        x = torch.randn(20, width, device="cuda", requires_grad=True)
        grad, = torch.autograd.grad(layer(x).square().sum(), x, create_graph=True)
        with pytest.raises(RuntimeError, match="once_differentiable"):
            grad.square().sum().backward()
