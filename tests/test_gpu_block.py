"""The layers over the training operators: gradients against autograd in 64 bits, training with NOVAK beside
the same blocks by torch's operators, and what is kept between the passes."""
import os
import sys

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def block():
    from paper_2601_07876_b200 import block
    return block


def reference(b, x, dy, kind):
    """Gradients of the block in 64 bits, from unrounded activations."""
    f = {"gelu": torch.nn.functional.gelu, "silu": torch.nn.functional.silu,
         "gelu_tanh": lambda t: torch.nn.functional.gelu(t, approximate="tanh")}[kind]
    p = {n: t.detach().double().requires_grad_() for n, t in b.named_parameters()}
    x = x.detach().double().requires_grad_()
    h = torch.nn.functional.layer_norm(x, x.shape[-1:], p["up.gamma"], p["up.beta"], b.up.eps)
    u = torch.nn.functional.linear(h, p["up.weight"], p["up.bias"])
    y = x + torch.nn.functional.linear(f(u), p["down.weight"], p["down.bias"])
    y.backward(dy.double())
    return y.detach(), x.grad, {n: t.grad for n, t in p.items()}


def far(a, b):
    return float((a.double() - b).norm() / b.norm())


@pytest.mark.parametrize("kind", ["gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("shape,width,hidden", [((300,), 192, 416), ((4, 50), 200, 333), ((1,), 64, 96)])
def test_gradients(block, shape, width, hidden, kind):
    """A kept value is off by at most half a scale, a 128th of its block's largest: an independent error of
    under 1.1 % of the block's deviation (largest of 32 normal values: 2.4 deviations on average), which enters
    each gradient once or twice; the products by themselves are fp32.  Held to 3 % in the norm."""
    torch.manual_seed(3)
    b = block.MlpBlock8(width, hidden, kind)
    with torch.no_grad():
        b.up.gamma.normal_(1.0, 0.1)
        b.up.beta.normal_(0.0, 0.1)
        b.down.bias.normal_(0.0, 0.1)
    x = torch.randn(*shape, width, device="cuda", requires_grad=True)
    dy = torch.randn(*shape, width, device="cuda")
    y = b(x)
    y.backward(dy)
    ry, rx, rp = reference(b, x, dy, kind)
    assert far(y.detach(), ry) < 1e-3            # (the products may run in fewer bits; nothing in 8)
    assert far(x.grad, rx) < 0.03
    for n, p in b.named_parameters():
        assert p.grad.dtype == torch.float32 and p.grad.shape == p.shape
        assert far(p.grad, rp[n]) < 0.03, n


def test_no_gradient_where_none_is_wanted(block):
    b = block.MlpBlock8(64, 96)
    x = torch.randn(20, 64, device="cuda")
    b.up.weight.requires_grad_(False)
    b(x).sum().backward()                        # (a broadcast gradient: not contiguous)
    assert b.up.weight.grad is None and b.up.gamma.grad is not None and b.down.weight.grad is not None


def test_kept_bytes(block):
    rows, width, hidden = 4096, 768, 2304
    b = block.MlpBlock8(width, hidden)
    x = torch.randn(rows, width, device="cuda").to(torch.bfloat16).requires_grad_()
    b(x)
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    y = b(x)
    kept = torch.cuda.memory_allocated() - before - y.numel() * 2
    # xhat, u, a in 8 bits, rstd and mean; the allocator rounds up
    want = rows * (width + 2 * hidden) * 33 // 32 + 8 * rows
    assert want <= kept <= want + 8 * 2 ** 21
    del y


def test_training_beside_torch():
    """40 steps of both from one start: the loss falls, and the 8-bit run ends within 2 % of the other's."""
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import train_mlp_8bit as example
    result = example.run(steps=40, width=256, hidden=768, tokens=4096, depth=2)
    (ours, kept), (plain, kept_plain) = result["8 bits"], result["torch bf16"]
    assert abs(ours[0] / plain[0] - 1) < 0.01
    assert ours[-1] < ours[0] and plain[-1] < plain[0] and abs(ours[-1] / plain[-1] - 1) < 0.02
    assert kept < 0.6 * kept_plain
