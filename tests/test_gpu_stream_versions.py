"""What the stream's operators write in place is known to autograd: no backward pass takes the new values for those of
its forward pass."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ops():
    from paper_2601_07876_b200 import ops
    return ops


def test_no_backward_pass_through_weights_that_were_stepped_since():
    from paper_2601_07876_b200.block import RmsLinear8
    from paper_2601_07876_b200.optim import Muon
    torch.manual_seed(1)
    layer = RmsLinear8(96, 130)
    opt = Muon([layer.weight], lr=0.1)
    x = torch.randn(20, 96, device="cuda", requires_grad=True)
    loss = layer(x)[0].square().sum()
    loss.backward(retain_graph=True)
    want = x.grad.clone()
    x.grad = None
    loss.backward(retain_graph=True)                    # (nothing has been stepped yet)
    assert torch.equal(x.grad, want)
    opt.step()
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()
    layer(x)[0].square().sum().backward()               # and a new forward pass is as ever


def test_versions(ops):
    theta, m, g = torch.randn(3, 40, 50, device="cuda").unbind()
    theta, m = theta.clone(), m.clone()
    before = [t._version for t in (theta, m, g)]
    ops.orthogonal_step([theta], [g], [m], [0.1])
    assert theta._version > before[0] and m._version > before[1] and g._version == before[2]
    out, dout, ids = torch.zeros(5, 8, device="cuda"), torch.ones(2, 8, device="cuda"), torch.tensor([1, 2], device="cuda")
    before = out._version
    assert ops.embedding_grad(dout, ids, 5, out=out) is not None and out._version > before
    before = out._version
    ops.embedding_grad(dout, ids, 5)
    assert out._version == before and dout._version == 0


def test_tensors_of_inference_have_no_versions(ops):
    with torch.inference_mode():
        theta, g = torch.zeros(8, 9, device="cuda"), torch.ones(8, 9, device="cuda")
        m = torch.zeros_like(theta)
        ops.orthogonal_step([theta], [g], [m], [0.1])
    ops.orthogonal_step([theta], [g], [m], [0.1])
    assert torch.isfinite(theta).all() and theta.any()
