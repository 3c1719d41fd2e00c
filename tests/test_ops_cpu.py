"""Refusals of the training operators' C entry points (made before any CUDA work), the format's sizes, and
the 64-bit definitions that the GPU tests compare with, against torch's own autograd."""
import os
import re

import pytest
import torch

import ops_reference as R
from paper_2601_07876_b200 import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 1 << 20            # an address that is never read: every call below is refused first
OK, EINVAL = B.NOVAK_OK, B.NOVAK_EINVAL


@pytest.fixture(scope="module")
def lib():
    return B.load_library()


def test_every_operator_in_the_header_has_a_signature(lib):
    header = open(os.path.join(ROOT, "include", "novak.h")).read()
    header = re.sub(r"/\*.*?\*/", "", header, flags=re.S)
    names = set(re.findall(r"\b(novak_[a-z0-9_]+)\s*\(", header))
    src = open(os.path.join(ROOT, "paper_2601_07876_b200", "binding.py")).read()
    assert {"novak_act8_pack", "novak_layer_norm_backward", "novak_linear_weight_grad"} <= names
    for name in sorted(names):
        assert hasattr(lib, name) and f'"{name}"' in src, name


def test_pitch(lib):
    assert [lib.novak_act8_pitch(c) for c in (-1, 0, 1, 31, 32, 33, 1000)] == [0, 0, 32, 32, 32, 64, 1024]


def call(lib, name, **change):
    base = {
        "novak_act8_pack": dict(x=P, xs=8, type=0, codes=P, exps=P, rows=4, cols=8, stream=None),
        "novak_act8_unpack": dict(codes=P, exps=P, out=P, os=8, type=0, rows=4, cols=8, stream=None),
        "novak_layer_norm": dict(x=P, xs=8, y=P, ys=8, type=0, w=P, b=P, param=0, eps=1e-5, mean=P, rstd=P, codes=P,
                                 exps=P, rows=4, cols=8, stream=None),
        "novak_layer_norm_backward": dict(dy=P, dys=8, x=None, xs=0, type=0, mean=None, rstd=P, codes=P, exps=P, w=P,
                                          param=0, dx=P, dxs=8, dw=P, db=P, grad=0, work=P, bytes=1 << 30, rows=4,
                                          cols=8, stream=None),
        "novak_activation": dict(u=P, us=8, a=P, as_=8, type=0, kind=0, uc=P, ue=P, ac=P, ae=P, rows=4, cols=8,
                                 stream=None),
        "novak_activation_backward": dict(da=P, das=8, u=None, us=0, type=0, kind=0, codes=P, exps=P, du=P, dus=8,
                                          rows=4, cols=8, stream=None),
        "novak_linear_weight_grad": dict(dy=P, dys=8, type=0, codes=P, exps=P, w=P, b=P, param=0, dw=P, db=P, grad=0,
                                         work=P, bytes=1 << 30, rows=4, n_out=8, n_in=8, stream=None),
    }[name]
    assert set(change) <= set(base)
    return getattr(lib, name)(*{**base, **change}.values())


BAD = [
    ("novak_act8_pack", dict(x=None)), ("novak_act8_pack", dict(xs=7)), ("novak_act8_pack", dict(type=2)),
    ("novak_act8_pack", dict(codes=None)), ("novak_act8_pack", dict(exps=None)), ("novak_act8_pack", dict(codes=P + 8)),
    ("novak_act8_pack", dict(x=P + 2)), ("novak_act8_pack", dict(rows=-1)), ("novak_act8_pack", dict(cols=0)),
    ("novak_act8_pack", dict(rows=1 << 39, cols=1 << 39, xs=1 << 39)), ("novak_act8_pack", dict(xs=1 << 62)),
    ("novak_act8_unpack", dict(out=None)), ("novak_act8_unpack", dict(os=0)), ("novak_act8_unpack", dict(exps=None)),
    ("novak_layer_norm", dict(x=None)), ("novak_layer_norm", dict(y=None)), ("novak_layer_norm", dict(w=None)),
    ("novak_layer_norm", dict(w=P + 1)), ("novak_layer_norm", dict(param=5)), ("novak_layer_norm", dict(eps=-1e-9)),
    ("novak_layer_norm", dict(eps=float("nan"))), ("novak_layer_norm", dict(eps=float("inf"))),
    ("novak_layer_norm", dict(codes=None)), ("novak_layer_norm", dict(mean=P + 2)), ("novak_layer_norm", dict(ys=5)),
    ("novak_layer_norm_backward", dict(dy=None)), ("novak_layer_norm_backward", dict(dx=None)),
    ("novak_layer_norm_backward", dict(rstd=None)), ("novak_layer_norm_backward", dict(codes=None, exps=None)),
    ("novak_layer_norm_backward", dict(x=P, xs=8, mean=P)), ("novak_layer_norm_backward", dict(mean=P)),
    ("novak_layer_norm_backward", dict(x=P, xs=8, codes=None, exps=None)),
    ("novak_layer_norm_backward", dict(x=P, xs=4, mean=P, codes=None, exps=None)),
    ("novak_layer_norm_backward", dict(work=None)), ("novak_layer_norm_backward", dict(bytes=1)),
    ("novak_layer_norm_backward", dict(work=P + 4)), ("novak_layer_norm_backward", dict(grad=3)),
    ("novak_activation", dict(kind=3)), ("novak_activation", dict(kind=-1)), ("novak_activation", dict(u=None)),
    ("novak_activation", dict(ue=None)), ("novak_activation", dict(ac=None)), ("novak_activation", dict(as_=2)),
    ("novak_activation_backward", dict(codes=None, exps=None)), ("novak_activation_backward", dict(u=P, us=8)),
    ("novak_activation_backward", dict(du=None)), ("novak_activation_backward", dict(kind=9)),
    ("novak_linear_weight_grad", dict(dy=None)), ("novak_linear_weight_grad", dict(codes=None, exps=None)),
    ("novak_linear_weight_grad", dict(w=None)), ("novak_linear_weight_grad", dict(dw=None)),
    ("novak_linear_weight_grad", dict(grad=7)), ("novak_linear_weight_grad", dict(rows=1 << 31)),
    ("novak_linear_weight_grad", dict(n_out=0)), ("novak_linear_weight_grad", dict(n_in=(1 << 22) + 1)),
    ("novak_linear_weight_grad", dict(dys=3)), ("novak_linear_weight_grad", dict(b=P + 1)),
]


@pytest.mark.parametrize("name,change", BAD, ids=[f"{n}-{'-'.join(c)}" for n, c in BAD])
def test_refusals(lib, name, change):
    assert call(lib, name, **change) == EINVAL
    assert lib.novak_ops_error().decode() != ""


def test_no_rows_need_no_buffers(lib):
    assert call(lib, "novak_act8_pack", rows=0, x=None, codes=None, exps=None) == OK
    assert call(lib, "novak_act8_unpack", rows=0, out=None, codes=None, exps=None) == OK
    assert call(lib, "novak_layer_norm", rows=0, x=None, y=None) == OK
    assert call(lib, "novak_activation", rows=0, u=None) == OK
    assert call(lib, "novak_activation_backward", rows=0, da=None, du=None) == OK


def test_operators_take_cuda_tensors_only():
    from paper_2601_07876_b200 import ops
    x = torch.randn(4, 32)
    for bad in (lambda: ops.act8_pack(x), lambda: ops.layer_norm(x, x[0]), lambda: ops.activation(x)):
        with pytest.raises(ValueError, match="CUDA"):
            bad()
    with pytest.raises(ValueError, match="kind"):
        ops.activation(x, "relu")
    with pytest.raises(ValueError):
        ops.Act8(torch.zeros(4, 32, dtype=torch.int8), torch.zeros(4, 1, dtype=torch.uint8), 33)
    with pytest.raises(TypeError):
        ops.Act8(x, torch.zeros(4, 1, dtype=torch.uint8), 32)


# ---- the definitions themselves -----------------------------------------------
def test_definitions_agree_with_autograd():
    torch.manual_seed(0)
    x = torch.randn(5, 70, dtype=torch.float64, requires_grad=True)
    w = torch.randn(70, dtype=torch.float64, requires_grad=True)
    b = torch.randn(70, dtype=torch.float64, requires_grad=True)
    y = torch.nn.functional.layer_norm(x, (70,), w, b, 1e-5)
    dy = torch.randn_like(y)
    y.backward(dy)
    ry, mean, rstd, xhat = R.layer_norm(x.detach(), w.detach(), b.detach(), 1e-5)
    assert torch.allclose(ry, y.detach(), rtol=1e-12, atol=1e-12)
    for got, want in zip(R.layer_norm_backward(dy, xhat, rstd, w.detach()), (x.grad, w.grad, b.grad)):
        assert torch.allclose(got, want, rtol=1e-11, atol=1e-12)
    for kind, f in (("gelu", torch.nn.functional.gelu), ("silu", torch.nn.functional.silu),
                    ("gelu_tanh", lambda t: torch.nn.functional.gelu(t, approximate="tanh"))):
        u = torch.linspace(-9, 9, 301, dtype=torch.float64, requires_grad=True)
        a = f(u)
        a.sum().backward()
        assert torch.allclose(R.act(kind, u.detach()), a.detach(), rtol=1e-10, atol=1e-15)
        assert torch.allclose(R.act_slope(kind, u.detach()), u.grad, rtol=1e-10, atol=1e-14)


def test_the_format_by_hand():
    x = torch.zeros(1, 40)
    x[0, 0], x[0, 1], x[0, 2], x[0, 33] = 1.0, -0.5, 0.013, 3.0
    codes, exps = R.act8_forms(x)
    assert exps.tolist() == [[121, 122]]                     # 2^-6: 1.0 is 64 of them; 2^-5: 3.0 is 96
    assert codes[0, :3].tolist() == [64, -32, 1] and codes[0, 33] == 96 and codes.shape == (1, 64)
    assert R.act8_values(codes, exps, 40)[0, 2] == 2.0 ** -6
