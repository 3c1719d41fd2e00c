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


# ---- memory ---------------------------------------------------------------------------
def allocated():
    torch.cuda.synchronize()
    return torch.cuda.memory_allocated()


def test_what_is_kept_goes_with_the_backward_pass(block):
    """With the outputs still referenced, as a training loop's loss and prediction are.  What stays beside them is
    rounding of the allocator's: less than a 20th of what was kept."""
    rows = 4096
    for layer, width in ((block.NormLinear8(768, 2304), 768), (block.ActLinear8(2304, 768), 2304),
                         (block.MlpBlock8(768, 2304), 768)):
        for p in layer.parameters():
            p.grad = torch.zeros_like(p)
        x = torch.randn(rows, width, device="cuda").to(torch.bfloat16).requires_grad_()
        x.grad, dy = torch.zeros_like(x), None
        for _ in range(2):                  # (the first time round libraries take memory of their own)
            y = None
            before = allocated()
            y = layer(x)
            kept = allocated() - before - y.numel() * 2
            if dy is None:
                dy = torch.ones_like(y)
                before += dy.numel() * 2
            y.backward(dy)
            after = allocated() - before - y.numel() * 2
        assert kept > rows * width and after < kept / 20, (kept, after)


def test_saved_tensor_hooks_see_what_is_kept(block):
    """Kept on the host between the passes: the same gradients, and next to nothing on the device meanwhile."""
    torch.manual_seed(0)
    for layer, width in layers(block):
        x = torch.randn(2000, width, device="cuda", requires_grad=True)
        wrt = [x, *layer.parameters()]
        y = layer(x)
        want = torch.autograd.grad(y, wrt, torch.ones_like(y))
        sizes = []

        def pack(t):
            sizes.append(t.numel() * t.element_size())
            return t.cpu()
        with torch.autograd.graph.saved_tensors_hooks(pack, lambda t: t.cuda()):
            y = layer(x)
        assert sum(sizes) >= 2000 * width * 33 // 32
        for a, b in zip(torch.autograd.grad(y, wrt, torch.ones_like(y)), want):
            assert torch.equal(a, b)


def test_backward_twice(block):
    for layer, width in layers(block):
        x = torch.randn(50, width, device="cuda", requires_grad=True)
        wrt = [x, *layer.parameters()]
        y = layer(x)
        first = torch.autograd.grad(y, wrt, torch.ones_like(y), retain_graph=True)
        second = torch.autograd.grad(y, wrt, torch.ones_like(y))
        assert all(torch.equal(a, b) for a, b in zip(first, second))
        with pytest.raises(RuntimeError, match="second time"):
            torch.autograd.grad(y, wrt, torch.ones_like(y))
