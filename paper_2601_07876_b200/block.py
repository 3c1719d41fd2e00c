"""Layers that keep what their backward pass needs in 8 bits, over ``ops``.

Two pairs, each one autograd function, because one checkpoint serves two backward
passes:

* ``NormLinear8``: layer norm, then a linear layer.  The 8-bit form of xhat is all that
  is kept: the norm's backward pass and the linear layer's weight gradient (through the
  norm's weight and bias) both work from it.
* ``ActLinear8``: activation function, then a linear layer.  The 8-bit forms of the
  function's input and output are kept.

``MlpBlock8`` is the pre-norm residual block of both: 9.3 bytes per token and unit of
width instead of 20 in bf16 (with a hidden width of four times the width).  Parameters
are float32, as ``optim.Novak`` takes them; products run in the input's type (bfloat16
under ``x.to(torch.bfloat16)``), and the gradients arrive in float32.  The backward
passes have none of their own: asking for second derivatives raises.  What is kept are saved
tensors: the backward pass lets go of them, and saved-tensor hooks see them.  Forms that
no gradient needs (under ``no_grad``, of frozen parameters) are not made.
"""
from __future__ import annotations

import math

import torch
from torch.autograd.function import once_differentiable

from . import ops


def _dense(t):
    return t if t.is_contiguous() else t.contiguous()


def _linear(x, weight, bias):
    return torch.nn.functional.linear(x, weight.to(x.dtype), None if bias is None else bias.to(x.dtype))


def _recorded_linear(x, weight, bias, weight_trained):
    """The same where a backward pass is to come, which has to be able to take up its types."""
    if weight_trained:
        ops._type(weight.dtype, "weight")
    y = _linear(x, weight, bias)
    ops._type(y.dtype, "the output (under autocast)")
    return y


def _linear_backward(dy, kept, weight, needs, affine=None):
    """(dx, dW, db) of a linear layer whose input was kept in 8 bits."""
    dw = db = None
    if needs[1]:
        dw, db = ops.linear_weight_grad(dy, kept, affine=affine, bias=needs[2], dtype=weight.dtype)
    elif needs[2]:
        db = dy.reshape(-1, dy.shape[-1]).sum(0, dtype=torch.float32)
    return (torch.matmul(dy, weight.to(dy.dtype)) if needs[0] else None), dw, db


class _NormLinear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, gamma, beta, weight, bias, eps):
        x = _dense(x)
        keep = any(ctx.needs_input_grad[:4])            # (the bias's gradient needs nothing of it)
        h, _, rstd, kept = ops.layer_norm(x, gamma, beta, eps, checkpoint=keep)
        ctx.save_for_backward(kept.buffer if keep else None, rstd, gamma, beta, weight)
        ctx.width = x.shape[-1]
        return _recorded_linear(h, weight, bias, ctx.needs_input_grad[3])

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        buffer, rstd, gamma, beta, weight = ctx.saved_tensors
        kept = None if buffer is None else ops.Act8.from_buffer(buffer, ctx.width)
        dy = _dense(dy)
        norm = ctx.needs_input_grad[0] or ctx.needs_input_grad[1] or ctx.needs_input_grad[2]
        dh, dw, db = _linear_backward(dy, kept, weight, (norm, *ctx.needs_input_grad[3:5]), (gamma, beta))
        dx = dgamma = dbeta = None
        if norm:
            dx, dgamma, dbeta = ops.layer_norm_backward(dh, kept, rstd, gamma, grad_dtype=gamma.dtype)
        return dx, dgamma, None if beta is None else dbeta, dw, db, None


class _ActLinear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, u, weight, bias, kind):
        a, kept_u, kept_a = ops.activation(_dense(u), kind, *ctx.needs_input_grad[:2])
        ctx.save_for_backward(*(None if kept is None else kept.buffer for kept in (kept_u, kept_a)), weight)
        ctx.width, ctx.kind = u.shape[-1], kind
        return _recorded_linear(a, weight, bias, ctx.needs_input_grad[1])

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        of_u, of_a, weight = ctx.saved_tensors
        kept_u, kept_a = (None if t is None else ops.Act8.from_buffer(t, ctx.width) for t in (of_u, of_a))
        da, dw, db = _linear_backward(_dense(dy), kept_a, weight, ctx.needs_input_grad[:3])
        du = ops.activation_backward(da, kept_u, ctx.kind) if ctx.needs_input_grad[0] else None
        return du, dw, db, None


def _recorded(*inputs):
    return torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in inputs)


def norm_linear(x, gamma, beta, weight, bias=None, eps: float = 1e-5):
    """linear(layer_norm(x, gamma, beta), weight, bias), kept in 8 bits for the backward pass
    (where there is one to come).  beta and bias may be None."""
    if not _recorded(x, gamma, beta, weight, bias):
        return _linear(ops.layer_norm(_dense(x), gamma, beta, eps)[0], weight, bias)
    return _NormLinear.apply(x, gamma, beta, weight, bias, eps)


def act_linear(u, weight, bias=None, kind: str = "gelu"):
    """linear(f(u), weight, bias), kept in 8 bits for the backward pass (where there is one to come)."""
    if not _recorded(u, weight, bias):
        return _linear(ops.activation(_dense(u), kind, save_input=False)[0], weight, bias)
    return _ActLinear.apply(u, weight, bias, kind)


def _linear_parameters(n_in: int, n_out: int, device):
    weight = torch.empty(n_out, n_in, device=device)
    torch.nn.init.uniform_(weight, -1.0 / math.sqrt(n_in), 1.0 / math.sqrt(n_in))
    return torch.nn.Parameter(weight), torch.nn.Parameter(torch.zeros(n_out, device=device))


class NormLinear8(torch.nn.Module):
    def __init__(self, n_in: int, n_out: int, eps: float = 1e-5, device="cuda"):
        super().__init__()
        self.eps = eps
        self.gamma = torch.nn.Parameter(torch.ones(n_in, device=device))
        self.beta = torch.nn.Parameter(torch.zeros(n_in, device=device))
        self.weight, self.bias = _linear_parameters(n_in, n_out, device)

    def forward(self, x):
        return norm_linear(x, self.gamma, self.beta, self.weight, self.bias, self.eps)


class ActLinear8(torch.nn.Module):
    def __init__(self, n_in: int, n_out: int, kind: str = "gelu", device="cuda"):
        super().__init__()
        self.kind = kind
        self.weight, self.bias = _linear_parameters(n_in, n_out, device)

    def forward(self, u):
        return act_linear(u, self.weight, self.bias, self.kind)


class MlpBlock8(torch.nn.Module):
    """x + W2 f(W1 layer_norm(x) + b1) + b2."""

    def __init__(self, width: int, hidden: int, kind: str = "gelu", eps: float = 1e-5, device="cuda"):
        super().__init__()
        self.up = NormLinear8(width, hidden, eps, device)
        self.down = ActLinear8(hidden, width, kind, device)

    def forward(self, x):
        return x + self.down(self.up(x))
