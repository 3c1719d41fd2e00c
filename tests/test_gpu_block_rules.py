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


def test_nothing_is_kept_but_the_8_bit_forms(block):
    """The allocator counts at most 1 MiB more for each of the four tensors that are kept; the norm's output or the
    hidden layer, kept in bf16 as well, would be 25 or 75 MB."""
    rows, width, hidden = 16384, 768, 2304
    b = block.MlpBlock8(width, hidden)
    x = torch.randn(rows, width, device="cuda").to(torch.bfloat16).requires_grad_()
    b(x)
    before = allocated()
    y = b(x)
    kept = allocated() - before - y.numel() * 2
    forms = rows * (width + 2 * hidden) * 33 // 32
    assert forms <= kept <= forms + 8 * rows + 5 * 2 ** 20, (kept, forms)


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


# ---- what no gradient needs ---------------------------------------------------------
@pytest.fixture
def calls(block, monkeypatch):
    """(operator, forms asked for) of each call that leaves forms, and the others' names."""
    made = []
    inner = {name: getattr(block.ops, name) for name in ("layer_norm", "activation", "linear_weight_grad")}

    def layer_norm(x, w, b, eps=1e-5, checkpoint=False):
        made.append(("layer_norm", checkpoint))
        return inner["layer_norm"](x, w, b, eps, checkpoint)

    def activation(u, kind="gelu", save_input=True, save_output=False):
        made.append(("activation", save_input, save_output))
        return inner["activation"](u, kind, save_input, save_output)

    def linear_weight_grad(*args, **kw):
        made.append(("linear_weight_grad",))
        return inner["linear_weight_grad"](*args, **kw)
    for f in (layer_norm, activation, linear_weight_grad):
        monkeypatch.setattr(block.ops, f.__name__, f)
    return made


def test_evaluation_keeps_nothing(block, calls):
    b = block.MlpBlock8(64, 96)
    x = torch.randn(20, 64, device="cuda")
    want = b(x).detach()
    assert calls == [("layer_norm", True), ("activation", True, True)]
    nothing = [("layer_norm", False), ("activation", False, False)]
    for context in (torch.no_grad(), torch.inference_mode()):
        calls.clear()
        with context:
            y = b(x)
        assert calls == nothing and torch.equal(y, want) and not y.requires_grad
    for p in b.parameters():
        p.requires_grad_(False)
    calls.clear()
    assert torch.equal(b(x), want) and calls == nothing


def test_frozen_parameters_keep_what_the_others_need(block, calls):
    b = block.MlpBlock8(64, 96)
    x, dy = torch.randn(20, 64, device="cuda", requires_grad=True), torch.randn(20, 64, device="cuda")
    parameters = dict(b.named_parameters(), x=x)
    want = dict(zip(parameters, torch.autograd.grad(b(x), list(parameters.values()), dy)))
    # trained alone: the forms of the norm and of the activation's input and output, whole weight gradients formed
    for names, norm, act, grads in ((["down.bias"], False, (False, False), 0), (["down.weight"], False, (False, True), 1),
                                    (["up.bias"], False, (True, False), 0), (["up.weight"], True, (True, False), 1),
                                    (["x"], True, (True, False), 0), (["up.gamma", "up.beta"], True, (True, False), 0),
                                    (["up.weight", "down.weight"], True, (True, True), 2)):
        for n, p in parameters.items():
            p.requires_grad_(n in names)
        calls.clear()
        got = torch.autograd.grad(b(x), [parameters[n] for n in names], dy)
        assert [c for c in calls if c[0] == "layer_norm"] == [("layer_norm", norm)], names
        assert [c for c in calls if c[0] == "activation"] == [("activation", *act)], names
        assert sum(c[0] == "linear_weight_grad" for c in calls) == grads, names
        for n, g in zip(names, got):
            # (a bias's gradient alone is the same sum in another order)
            bound = 20 * 2.0 ** -24 * dy.abs().sum() if n.endswith("bias") else 0.0
            assert (g - want[n]).abs().max() <= bound, n


def test_a_bias_alone_of_one_row_and_of_none(block, calls):
    layer = block.ActLinear8(64, 96)
    layer.weight.requires_grad_(False)
    one, = torch.autograd.grad(layer(torch.randn(64, device="cuda")), [layer.bias], torch.arange(96.0, device="cuda"))
    assert torch.equal(one, torch.arange(96.0, device="cuda"))
    none, = torch.autograd.grad(layer(torch.empty(0, 64, device="cuda")), [layer.bias], torch.empty(0, 96, device="cuda"))
    assert torch.equal(none, torch.zeros(96, device="cuda"))


# ---- what the backward pass could not take up ------------------------------------------
def test_a_norm_without_bias(block):
    """As one whose bias is zeros, to the bit."""
    x = torch.randn(300, 64, device="cuda", requires_grad=True)
    gamma = torch.randn(64, device="cuda", requires_grad=True)
    weight = torch.randn(96, 64, device="cuda", requires_grad=True)
    results = []
    for beta in (None, torch.zeros(64, device="cuda")):
        y = block.norm_linear(x, gamma, beta, weight)
        results.append((y, *torch.autograd.grad(y, [x, gamma, weight], torch.ones_like(y))))
    assert all(torch.equal(a, b) for a, b in zip(*results))
    kept = block.ops.act8_pack(x.detach())
    dy, w = torch.randn(300, 96, device="cuda"), gamma.detach()
    without = block.ops.linear_weight_grad(dy, kept, affine=(w, None))
    assert all(torch.equal(a, b) for a, b in zip(without, block.ops.linear_weight_grad(dy, kept, affine=(w, 0 * w))))


@pytest.mark.parametrize("dtype", [torch.float16, torch.float64])
def test_types_that_the_backward_pass_does_not_take_are_refused_before_it(block, dtype):
    for layer, width in layers(block):
        if hasattr(layer, "weight"):
            layer.weight.data = layer.weight.data.to(dtype)
        else:
            layer.down.weight.data = layer.down.weight.data.to(dtype)
        x = torch.randn(20, width, device="cuda")
        with pytest.raises(TypeError, match="weight"):
            layer(x)
        with torch.no_grad():
            assert layer(x).dtype == torch.float32


def test_autocast(block):
    """bf16: taken; fp16: refused, and not only by the backward pass."""
    for layer, width in layers(block):
        x = torch.randn(20, width, device="cuda", requires_grad=True)
        with torch.autocast("cuda", torch.float16), pytest.raises(TypeError, match="autocast"):
            layer(x)
        with torch.autocast("cuda", torch.bfloat16):
            y = layer(x)
        y.float().sum().backward()
        assert x.grad.dtype == torch.float32 and torch.isfinite(x.grad).all()
