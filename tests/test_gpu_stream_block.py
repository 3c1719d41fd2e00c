"""The layers over the norm with the residual's addition and over the embedding, and the optimizer over the
orthogonalised step: gradients against autograd in 64 bits, memory, graphs, and a run of all of them together."""
import copy
import math
import os
import sys

import pytest
import torch

import stream_reference as S
from test_gpu_block import far

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.gpu
F = torch.nn.functional


@pytest.fixture(scope="module")
def block():
    from paper_2601_07876_b200 import block
    return block


def f64(t):
    return t.detach().double().requires_grad_()


@pytest.mark.parametrize("shape,width,out", [((300,), 192, 416), ((4, 50), 200, 333), ((1,), 64, 96)])
@pytest.mark.parametrize("with_residual,with_bias", [(True, False), (True, True), (False, True)])
def test_gradients_of_the_norm_and_linear(block, shape, width, out, with_residual, with_bias):
    """A kept value is off by at most half a scale: under 1.1 % of its block's deviation, which enters each gradient
    once or twice (3 % in the norm, as for the layer norm's layer); the stream's own gradient is exact."""
    torch.manual_seed(5)
    layer = block.RmsLinear8(width, out, bias=with_bias)
    with torch.no_grad():
        layer.gamma.normal_(1.0, 0.1)
    x = torch.randn(*shape, width, device="cuda", requires_grad=True)
    r = torch.randn(*shape, width, device="cuda", requires_grad=True) if with_residual else None
    dy, dh = torch.randn(*shape, out, device="cuda"), torch.randn(*shape, width, device="cuda")
    y, h = layer(x, r)
    ((y * dy).sum() + (h * dh).sum()).backward()
    p = {n: f64(t) for n, t in layer.named_parameters()}
    xd, rd = f64(x), None if r is None else f64(r)
    hd = xd if rd is None else xd + rd
    yd = F.linear(F.rms_norm(hd, (width,), p["gamma"], layer.eps), p["weight"], p.get("bias"))
    ((yd * dy.double()).sum() + (hd * dh.double()).sum()).backward()
    assert far(y.detach(), yd.detach()) < 1e-3 and far(h.detach(), hd.detach()) < 1e-6
    assert far(x.grad, xd.grad) < 0.03 and (r is None or torch.equal(r.grad, x.grad))
    for n, t in layer.named_parameters():
        assert t.grad.dtype == torch.float32 and far(t.grad, p[n].grad) < 0.03, n


def test_only_one_of_the_two_outputs_is_used(block):
    layer = block.RmsLinear8(64, 96)
    x, r = (torch.randn(20, 64, device="cuda", requires_grad=True) for _ in range(2))
    layer(x, r)[1].sum().backward()
    assert torch.equal(x.grad, torch.ones_like(x)) and torch.equal(r.grad, x.grad) and layer.weight.grad is None
    x.grad = r.grad = None
    layer(x, r)[0].sum().backward()
    assert torch.equal(x.grad, r.grad) and layer.weight.grad is not None


def test_nothing_is_kept_where_nothing_is_wanted(block):
    layer = block.RmsLinear8(64, 96, bias=True)
    x = torch.randn(20, 64, device="cuda")
    with torch.no_grad():
        y, h = layer(x, x)
    assert not y.requires_grad and torch.equal(h, x + x)
    for p in (layer.gamma, layer.weight):
        p.requires_grad_(False)
    y, h = layer(x, x)
    y.sum().backward()
    assert layer.bias.grad is not None and layer.weight.grad is None and layer.gamma.grad is None
    want = layer(x, None)[0]
    assert torch.equal(want.detach(), layer(x * 1.0, None)[0].detach())


def test_second_derivatives_are_refused(block):
    layer = block.RmsLinear8(64, 96)
    x = torch.randn(20, 64, device="cuda", requires_grad=True)
    for r in (x * 2, None):
        g, = torch.autograd.grad(layer(x, r)[0].sum(), x, create_graph=True)
        with pytest.raises(RuntimeError):
            g.sum().backward()


@pytest.mark.parametrize("scale,dtype", [(1.0, torch.float32), (math.sqrt(48), torch.bfloat16)])
def test_embedding_layer(block, scale, dtype):
    layer = block.Embedding(40, 48, scale=scale, dtype=dtype)
    ids = torch.tensor([[3, 7, -1, 3], [39, 40, 3, 0]], device="cuda")
    out = layer(ids)
    assert out.shape == (2, 4, 48) and torch.equal(out.cpu(), S.embedding(ids, layer.weight.detach(), scale, dtype))
    dout = torch.randn(2, 4, 48, device="cuda").to(dtype)
    out.backward(dout)
    want, size, count = S.embedding_grad(dout, ids, 40, scale)
    assert (layer.weight.grad.cpu().double() - want).abs().le(S.embedding_grad_bound(want, size, count, torch.float32)).all()


def test_a_block_stays_small(block):
    """Beside its parameters a block keeps xhat, u and f(u) in 8 bits and rstd; the stream is the next one's input."""
    rows, width, hidden = 4096, 768, 2304
    b = block.RmsMlpBlock8(width, hidden)
    delta = torch.randn(rows, width, device="cuda").to(torch.bfloat16).requires_grad_()
    stream = torch.randn(rows, width, device="cuda").to(torch.bfloat16)
    b(delta, stream)
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    out, h = b(delta, stream)
    kept = torch.cuda.memory_allocated() - before - (out.numel() + h.numel()) * 2
    want = rows * (width + 2 * hidden) * 33 // 32 + 4 * rows
    assert want <= kept <= want + 8 * 2 ** 21


# ---- the optimizer --------------------------------------------------------------
@pytest.mark.parametrize("scale", ["spectral", "rms"])
def test_muon_steps(scale):
    """Against the step written out in 64 bits.  X's tolerance, times the step, is what theta may be off by."""
    from paper_2601_07876_b200.optim import Muon
    torch.manual_seed(1)
    shapes = [(60, 100), (130, 40), (3, 20, 30)]
    params = [torch.nn.Parameter(0.1 * torch.randn(*s, device="cuda")) for s in shapes]
    idle = torch.nn.Parameter(torch.randn(4, 4, device="cuda"))
    before = idle.detach().clone()
    opt = Muon([*params, idle], lr=0.05, momentum=0.9, weight_decay=0.1, scale=scale)
    ref = [(p.detach().cpu().double(), torch.zeros(p.shape, dtype=torch.float64)) for p in params]
    off = [0.0] * 3
    for k in range(3):
        for i, p in enumerate(params):
            p.grad = torch.randn_like(p)
            t, m = ref[i]
            g = p.grad.cpu().double()
            m = 0.9 * m + g
            u = (g + 0.9 * m).reshape(-1, *p.shape[-2:])
            r, c = p.shape[-2:]
            step = 0.05 * (math.sqrt(max(1, r / c)) if scale == "spectral" else 0.2 * math.sqrt(max(r, c)))
            x = torch.stack([S.orthogonalized(a) for a in u]).reshape(p.shape)
            ref[i] = (t * (1 - 0.05 * 0.1) - step * x, m)
            off[i] += step * S.orthogonal_tolerance(r, c) * float(x.norm())
        opt.step()
    for p, (t, m), limit in zip(params, ref, off):
        assert float((p.detach().cpu().double() - t).norm()) <= limit + 1e-6 * float(t.norm())
        assert torch.allclose(opt.state[p]["momentum"].cpu().double(), m, rtol=1e-5, atol=1e-6)
    assert torch.equal(idle.detach(), before)


def test_muon_checkpoints_groups_and_refusals():
    from paper_2601_07876_b200.optim import Muon
    torch.manual_seed(2)
    a, b = (torch.nn.Parameter(torch.randn(40, 50, device="cuda")) for _ in range(2))
    opt = Muon([dict(params=[a], lr=0.1), dict(params=[b], lr=0.01, nesterov=False)])
    a.grad, b.grad = torch.randn_like(a), torch.randn_like(b).to(torch.float32)
    opt.step()
    saved, kept = copy.deepcopy(opt.state_dict()), (a.detach().clone(), b.detach().clone())
    opt.step()
    after = (a.detach().clone(), b.detach().clone())
    with torch.no_grad():
        a.copy_(kept[0])
        b.copy_(kept[1])
    again = Muon([dict(params=[a]), dict(params=[b])])
    again.load_state_dict(saved)
    again.step()
    assert torch.equal(a.detach(), after[0]) and torch.equal(b.detach(), after[1])
    for bad in (lambda: Muon([torch.nn.Parameter(torch.randn(5, device="cuda"))]), lambda: Muon([a], scale="adam"),
                lambda: Muon([torch.nn.Parameter(torch.randn(5, 5, device="cuda").bfloat16())])):
        with pytest.raises(ValueError):
            bad()


# ---- all of them together -------------------------------------------------------
def model_and_reference():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import train_lm_8bit as example
    torch.manual_seed(0)
    model = example.Model(vocab=300, width=128, hidden=256, depth=2)
    gen = torch.Generator(device="cuda").manual_seed(3)
    after = torch.randint(300, (300, 4), generator=gen, device="cuda")
    return example, model, *example.batch(gen, 512, 300, after)


def reference_loss(model, ids, target):
    """The example's model by torch's operators in 64 bits."""
    p = {n: f64(t) for n, t in model.named_parameters()}
    w = p["embed.weight"]
    delta = torch.where((ids >= 0)[:, None], w[ids.clamp(min=0)] * model.embed.scale, torch.zeros(1, dtype=torch.float64, device="cuda"))
    stream = None
    for i, b in enumerate(model.blocks):
        stream = delta if stream is None else stream + delta
        u = F.linear(F.rms_norm(stream, stream.shape[-1:], p[f"blocks.{i}.up.gamma"], b.up.eps), p[f"blocks.{i}.up.weight"])
        delta = F.linear(F.silu(u), p[f"blocks.{i}.down.weight"], p[f"blocks.{i}.down.bias"])
    out = F.linear(F.rms_norm(stream + delta, stream.shape[-1:], p["out.gamma"], model.out.eps), w)
    loss = F.cross_entropy(out, target)
    loss.backward()
    return float(loss.detach()), {n: t.grad for n, t in p.items()}


def test_gradients_of_a_language_model_and_a_step():
    """bf16 products and stream: 2^-8 relative a rounding, a dozen of them on the way of each gradient, and 8-bit
    forms on top: held to 6 % in the norm."""
    from paper_2601_07876_b200 import ops
    from paper_2601_07876_b200.optim import Muon, Novak
    _, model, ids, target = model_and_reference()
    loss = F.cross_entropy(model(ids).float(), target)
    loss.backward()
    want, grads = reference_loss(model, ids, target)
    assert abs(float(loss.detach()) / want - 1) < 0.01
    for n, t in model.named_parameters():
        assert far(t.grad, grads[n]) < 0.06, n
    matrices = model.matrices()
    rest = [p for p in model.parameters() if all(p is not q for q in matrices)]
    before = [p.detach().clone() for p in model.parameters()]
    Muon(matrices).step()
    Novak(rest, lr=1e-3).step()
    for p, b in zip(model.parameters(), before):
        assert torch.isfinite(p).all() and not torch.equal(p.detach(), b)
    assert ops.wait_failures() == 0


def test_a_training_step_is_captured():
    """Forward, backward and Muon's step in one graph; replays go on like eager steps from the same start.  The eager
    gradients are gone before the capture."""
    from paper_2601_07876_b200.optim import Muon
    _, model, ids, target = model_and_reference()
    matrices = model.matrices()
    opt = Muon(matrices, lr=1e-2)

    def step():
        loss = F.cross_entropy(model(ids).float(), target)
        grads = torch.autograd.grad(loss, matrices)
        for p, g in zip(matrices, grads):
            p.grad = g
        opt.step()
        return loss.detach()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    start = [p.detach().clone() for p in matrices]
    momenta = [opt.state[p]["momentum"].clone() for p in matrices]
    for p in matrices:
        p.grad = None
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loss = step()

    def rewind():
        for p, s, m in zip(matrices, start, momenta):
            p.data.copy_(s)
            opt.state[p]["momentum"].copy_(m)
    rewind()
    for _ in range(3):
        graph.replay()
    got = [p.detach().clone() for p in matrices], float(loss)
    rewind()
    for _ in range(3):
        last = step()
    assert all(torch.equal(a, b.detach()) for a, b in zip(got[0], matrices)) and got[1] == float(last)


def test_the_example_runs():
    example, *_ = model_and_reference()
    losses = example.run(steps=3, vocab=512, width=128, hidden=256, tokens=512, depth=2)
    assert len(losses) == 3 and all(math.isfinite(x) for x in losses)
