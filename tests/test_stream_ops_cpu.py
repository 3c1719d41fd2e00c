"""Refusals of the C entry points of the norm with the residual's addition, the embedding and the orthogonalised
updates (made before any CUDA work), and the 64-bit definitions that the GPU tests compare with."""
import ctypes
import math

import pytest
import torch

import stream_reference as S
from paper_2601_07876_b200 import binding as B

P = 1 << 20            # an address that is never read: every call below is refused first
OK, EINVAL = B.NOVAK_OK, B.NOVAK_EINVAL


@pytest.fixture(scope="module")
def lib():
    return B.load_library()


def pointers(*p):
    return (ctypes.c_void_p * len(p))(*p)


def sizes(*n):
    return (ctypes.c_int64 * len(n))(*n)


def doubles(*x):
    return (ctypes.c_double * len(x))(*x)


MUON = (3.4445, -4.7750, 2.0315)


def call(lib, name, **change):
    base = {
        "novak_rms_norm": dict(x=P, xs=8, r=P, rs=8, h=P, hs=8, y=2 * P, ys=8, type=0, w=P, param=0, eps=1e-6, rstd=P, codes=P,
                               exps=P, rows=4, cols=8, stream=None),
        "novak_rms_norm_backward": dict(dy=P, dys=8, dh=P, dhs=8, h=None, hs=0, type=0, rstd=P, codes=P, exps=P, w=P, param=0, dx=P,
                                        dxs=8, dw=P, grad=0, work=P, bytes=1 << 30, rows=4, cols=8, stream=None),
        "novak_embedding": dict(ids=P, idt=0, table=P, ts=8, type=0, scale=1.0, out=P, os=8, otype=0, tokens=4, vocab=5, cols=8,
                                stream=None),
        "novak_embedding_grad": dict(dout=P, ds=8, type=0, ids=P, idt=1, scale=1.0, dt=P, dts=8, grad=0, add=0, work=P, bytes=1 << 40,
                                     tokens=4, vocab=5, cols=8, stream=None),
        "novak_orthogonalize": dict(g=pointers(P, P), gs=sizes(9, 9), type=0, out=pointers(P, P), os=sizes(9, 9), rows=sizes(4, 5),
                                    cols=sizes(9, 9), n=2, abc=doubles(*MUON), steps=1, eps=1e-7, work=P, bytes=1 << 40, stream=None),
        "novak_orthogonal_step": dict(theta=pointers(P), g=pointers(P), type=0, m=pointers(P), rows=sizes(4), cols=sizes(9), n=1,
                                      momentum=0.9, nesterov=1, step=doubles(0.1), decay=1.0, abc=doubles(*MUON), steps=1, eps=1e-7,
                                      work=P, bytes=1 << 40, stream=None),
    }[name]
    assert set(change) <= set(base)
    return getattr(lib, name)(*{**base, **change}.values())


BAD = [
    ("novak_rms_norm", dict(x=None)), ("novak_rms_norm", dict(y=None)), ("novak_rms_norm", dict(h=None)), ("novak_rms_norm", dict(r=None)),
    ("novak_rms_norm", dict(w=None)), ("novak_rms_norm", dict(xs=7)), ("novak_rms_norm", dict(rs=7)), ("novak_rms_norm", dict(hs=7)),
    ("novak_rms_norm", dict(type=2)), ("novak_rms_norm", dict(param=2)), ("novak_rms_norm", dict(eps=-1.0)),
    ("novak_rms_norm", dict(eps=math.nan)), ("novak_rms_norm", dict(codes=None)), ("novak_rms_norm", dict(codes=P + 8)),
    ("novak_rms_norm", dict(rstd=P + 2)), ("novak_rms_norm", dict(rows=-1)), ("novak_rms_norm", dict(cols=0)),
    ("novak_rms_norm", dict(h=2 * P)), ("novak_rms_norm", dict(r=P + 2)),
    ("novak_rms_norm_backward", dict(dy=None)), ("novak_rms_norm_backward", dict(dx=None)), ("novak_rms_norm_backward", dict(rstd=None)),
    ("novak_rms_norm_backward", dict(h=P, hs=8)), ("novak_rms_norm_backward", dict(codes=None, exps=None)),
    ("novak_rms_norm_backward", dict(codes=None, exps=None, h=P, hs=3)), ("novak_rms_norm_backward", dict(dhs=3)),
    ("novak_rms_norm_backward", dict(work=None)), ("novak_rms_norm_backward", dict(bytes=1)), ("novak_rms_norm_backward", dict(work=P + 4)),
    ("novak_rms_norm_backward", dict(grad=3)), ("novak_rms_norm_backward", dict(w=P + 1)),
    ("novak_embedding", dict(ids=None)), ("novak_embedding", dict(idt=2)), ("novak_embedding", dict(ids=P + 2)),
    ("novak_embedding", dict(ids=P + 4, idt=1)), ("novak_embedding", dict(table=None)), ("novak_embedding", dict(out=None)),
    ("novak_embedding", dict(type=2)), ("novak_embedding", dict(otype=2)), ("novak_embedding", dict(scale=math.nan)),
    ("novak_embedding", dict(scale=1e39)), ("novak_embedding", dict(tokens=1 << 31)), ("novak_embedding", dict(vocab=1 << 31)),
    ("novak_embedding", dict(vocab=-1)), ("novak_embedding", dict(ts=7)), ("novak_embedding", dict(os=7)), ("novak_embedding", dict(cols=0)),
    ("novak_embedding_grad", dict(ids=None)), ("novak_embedding_grad", dict(dout=None)), ("novak_embedding_grad", dict(dt=None)),
    ("novak_embedding_grad", dict(grad=2)), ("novak_embedding_grad", dict(ds=7)), ("novak_embedding_grad", dict(dts=7)),
    ("novak_embedding_grad", dict(scale=math.inf)), ("novak_embedding_grad", dict(vocab=1 << 31)), ("novak_embedding_grad", dict(idt=-1)),
    ("novak_orthogonalize", dict(g=pointers(P, None))), ("novak_orthogonalize", dict(out=pointers(None, P))),
    ("novak_orthogonalize", dict(gs=sizes(9, 8))), ("novak_orthogonalize", dict(os=sizes(8, 9))), ("novak_orthogonalize", dict(g=None)),
    ("novak_orthogonalize", dict(rows=None)), ("novak_orthogonalize", dict(type=2)), ("novak_orthogonalize", dict(n=-1)),
    ("novak_orthogonalize", dict(n=(1 << 14) + 1)), ("novak_orthogonalize", dict(rows=sizes(4, -5))),
    ("novak_orthogonalize", dict(rows=sizes(4, (1 << 16) + 1))), ("novak_orthogonalize", dict(steps=0)),
    ("novak_orthogonalize", dict(steps=33)), ("novak_orthogonalize", dict(abc=None)), ("novak_orthogonalize", dict(abc=doubles(5, 0, 0))),
    ("novak_orthogonalize", dict(abc=doubles(math.inf, 0, 0))), ("novak_orthogonalize", dict(abc=doubles(0, 16, 0))),
    ("novak_orthogonalize", dict(eps=-1.0)), ("novak_orthogonalize", dict(work=None)), ("novak_orthogonalize", dict(bytes=1000)),
    ("novak_orthogonalize", dict(work=P + 16)), ("novak_orthogonalize", dict(g=pointers(P, P + 2))),
    ("novak_orthogonalize", dict(out=pointers(P, P + 1))),
    ("novak_orthogonal_step", dict(theta=pointers(None))), ("novak_orthogonal_step", dict(m=pointers(None))),
    ("novak_orthogonal_step", dict(g=pointers(None))), ("novak_orthogonal_step", dict(momentum=1.0)),
    ("novak_orthogonal_step", dict(momentum=-0.1)), ("novak_orthogonal_step", dict(decay=math.nan)),
    ("novak_orthogonal_step", dict(step=doubles(math.nan))), ("novak_orthogonal_step", dict(step=None)),
    ("novak_orthogonal_step", dict(type=7)), ("novak_orthogonal_step", dict(theta=pointers(P + 2))),
    ("novak_orthogonal_step", dict(bytes=0)),
]


@pytest.mark.parametrize("name,change", BAD, ids=[f"{i}-{n}-{'-'.join(c)}" for i, (n, c) in enumerate(BAD)])
def test_refusals(lib, name, change):
    assert call(lib, name, **change) == EINVAL
    assert lib.novak_ops_error().decode() != ""


def test_nothing_to_do_needs_no_buffers(lib):
    assert call(lib, "novak_rms_norm", rows=0, x=None, y=None, h=None, r=None) == OK
    assert call(lib, "novak_embedding", tokens=0, ids=None, out=None) == OK
    assert call(lib, "novak_embedding_grad", vocab=0, dt=None) == OK
    assert call(lib, "novak_embedding_grad", tokens=0, ids=None, dout=None, add=1) == OK
    assert call(lib, "novak_orthogonalize", n=0, g=None, gs=None, out=None, os=None, rows=None, cols=None, work=None, bytes=0) == OK
    assert call(lib, "novak_orthogonalize", rows=sizes(0, 4), cols=sizes(9, 0), g=pointers(None, None), out=pointers(None, None), work=None,
                bytes=0) == OK


@pytest.mark.parametrize("theta,g,m,refused", [
    ((0, 1000), (2000, 3000), (4000, 5000), None), ((0, 1000), (2000, 2000), (4000, 5000), None),
    ((0, 144), (2000, 3000), (288, 5000), None), ((0, 1000), (856, 1144), (4000, 5000), None),
    ((0, 0), (2000, 3000), (4000, 5000), "theta and m"), ((0, 1000), (2000, 3000), (4000, 4000), "theta and m"),
    ((0, 1000), (2000, 3000), (4000, 1000), "theta and m"), ((0, 140), (2000, 3000), (4000, 5000), "theta and m"),
    ((0, 1000), (1000, 3000), (4000, 5000), "g overlaps"), ((0, 1000), (2000, 5000), (4000, 5000), "g overlaps"),
    ((0, 1000), (860, 3000), (4000, 5000), "g overlaps"), ((0, 1000), (2000, 5140), (4000, 5000), "g overlaps")])
def test_a_step_has_its_matrices_for_itself(lib, theta, g, m, refused):
    """Two of 4 x 9, 144 bytes each."""
    at = [pointers(*(P + x for x in p)) for p in (theta, g, m)]
    assert call(lib, "novak_orthogonal_step", theta=at[0], g=at[1], m=at[2], rows=sizes(4, 4), cols=sizes(9, 9), n=2,
                step=doubles(1.0, 1.0), bytes=0) == EINVAL
    assert (refused or "work") in lib.novak_ops_error().decode()


def test_no_workspace_is_asked_for_what_will_be_refused(lib):
    ask = lib.novak_orthogonalize_bytes
    assert ask(sizes(4), sizes(9), 1) > 0 and ask(sizes(4), sizes((1 << 16) + 1), 1) == 0 and ask(sizes(-4), sizes(9), 1) == 0
    assert ask(sizes(*[65536] * 20), sizes(*[65536] * 20), 20) == 0         # more than can be addressed in one call
    assert call(lib, "novak_orthogonalize", rows=sizes(*[65536] * 20), cols=sizes(*[65536] * 20), gs=sizes(*[65536] * 20),
                os=sizes(*[65536] * 20), g=pointers(*[P] * 20), out=pointers(*[P] * 20), n=20) == EINVAL
    assert "addressed" in lib.novak_ops_error().decode()
    assert lib.novak_embedding_grad_bytes(4, 1 << 31, 8) == 0 and lib.novak_rms_norm_backward_bytes(-1, 8) == 0


def test_operators_take_cuda_tensors_only():
    from paper_2601_07876_b200 import ops
    x, ids = torch.randn(4, 32), torch.zeros(3, dtype=torch.int64)
    for bad in (lambda: ops.rms_norm(x, x[0]), lambda: ops.embedding(ids, x), lambda: ops.orthogonalize(x),
                lambda: ops.embedding_grad(x[:3], ids, 4), lambda: ops.orthogonal_step([x], [x], [x], [1.0])):
        with pytest.raises(ValueError, match="CUDA"):
            bad()


@pytest.mark.parametrize("coefficients", [MUON * 5, (1.5, -0.5, 0.0) * 32, (1.875, -1.25, 0.375) * 10,
                                          (8.28721201814563, -23.595886519098837, 17.300387312530933)])
def test_polynomials_that_are_held(lib, coefficients):
    """Refused for the missing workspace alone."""
    assert call(lib, "novak_orthogonalize", abc=doubles(*coefficients), steps=len(coefficients) // 3, bytes=0) == EINVAL
    assert "work" in lib.novak_ops_error().decode()


# ---- the definitions themselves -----------------------------------------------
def test_norm_agrees_with_autograd():
    torch.manual_seed(0)
    x, r = (torch.randn(5, 70, dtype=torch.float64, requires_grad=True) for _ in range(2))
    w = torch.randn(70, dtype=torch.float64, requires_grad=True)
    h = x + r
    y = torch.nn.functional.rms_norm(h, (70,), w, 1e-6)
    dy, dh = torch.randn_like(y), torch.randn_like(y)
    (y * dy + h * dh).sum().backward()
    ry, rstd, xhat = S.rms_norm(h.detach(), w.detach(), 1e-6)
    assert torch.allclose(ry, y.detach(), rtol=1e-12, atol=1e-12)
    dx, dw = S.rms_norm_backward(dy, xhat, rstd, w.detach(), dh)
    assert torch.allclose(dx, x.grad, rtol=1e-11, atol=1e-12) and torch.allclose(dx, r.grad, rtol=1e-11, atol=1e-12)
    assert torch.allclose(dw, w.grad, rtol=1e-11, atol=1e-12)


def test_embedding_agrees_with_autograd():
    table = torch.randn(9, 5, requires_grad=True)
    ids = torch.tensor([[3, 0, 3], [8, -1, 9]])
    out = S.embedding(ids, table.detach(), 2.0, torch.float32)
    there = torch.tensor([[1, 1, 1], [1, 0, 0]])
    plain = torch.nn.functional.embedding(ids.clamp(0, 8), table) * 2.0 * there[..., None]
    assert torch.equal(out, plain.detach())
    dout = torch.randn(2, 3, 5)
    (plain * dout).sum().backward()
    got, _, count = S.embedding_grad(dout, ids, 9, 2.0)
    assert torch.allclose(got.float(), table.grad, rtol=1e-6, atol=1e-6) and count.tolist() == [1, 0, 0, 2, 0, 0, 0, 0, 1]


def test_newton_schulz_is_its_polynomial_of_the_singular_values():
    torch.manual_seed(0)
    for shape in ((20, 30), (30, 20), (1, 4)):
        g = torch.randn(*shape, dtype=torch.float64)
        u, s, v = torch.linalg.svd(g, full_matrices=False)
        s = s / s.norm()
        for a, b, c in S.STEPS:
            s = a * s + b * s ** 3 + c * s ** 5
        assert torch.allclose(S.orthogonalized(g), (u * s) @ v, rtol=1e-9, atol=1e-10)
