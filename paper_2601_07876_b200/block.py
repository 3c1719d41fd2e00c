"""Layers that keep what their backward pass needs in 8 bits, over ``ops``.

Pairs, each one autograd function, because one checkpoint serves two backward passes:

* ``NormLinear8``: layer norm, then a linear layer.  The 8-bit form of xhat is all that
  is kept: the norm's backward pass and the linear layer's weight gradient (through the
  norm's weight and bias) both work from it.
* ``RmsLinear8``: the residual's addition, root-mean-square norm, then a linear layer.
  The 8-bit form of xhat is all that is kept here too; the stream, which the layer gives
  back beside its output, is not, and the gradient that comes down it is added where the
  norm's is formed.
* ``ActLinear8``: activation function, then a linear layer.  The 8-bit forms of the
  function's input and output are kept.

``MlpBlock8`` is the pre-norm residual block of both: 9.3 bytes per token and unit of
width instead of 20 in bf16 (with a hidden width of four times the width).
``RmsMlpBlock8`` is the same over ``RmsLinear8``, the residual stream handed from block to
block beside what is to be added to it, and ``Embedding`` starts the stream.  Parameters
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


class _RmsLinear(torch.autograd.Function):
    """(linear(rms_norm(x + residual)), x + residual)"""

    @staticmethod
    def forward(ctx, x, residual, gamma, weight, bias, eps):
        ctx.set_materialize_grads(False)
        keep = any(ctx.needs_input_grad[:4])            # (the bias's gradient needs nothing of it)
        y, h, rstd, kept = ops.rms_norm(_dense(x), gamma, residual=_dense(residual), eps=eps, checkpoint=keep)
        ctx.save_for_backward(kept.buffer if keep else None, rstd, gamma, weight)
        ctx.width = x.shape[-1]
        return _recorded_linear(y, weight, bias, ctx.needs_input_grad[3]), h

    @staticmethod
    @once_differentiable
    def backward(ctx, dy, dh):
        dx, dgamma, dw, db = _rms_linear_backward(ctx, dy, dh, (ctx.needs_input_grad[0] or ctx.needs_input_grad[1],
                                                                *ctx.needs_input_grad[2:5]))
        return dx, dx, dgamma, dw, db, None


class _RmsLinearOnly(torch.autograd.Function):
    """linear(rms_norm(x)): the first block's, whose stream is x."""

    @staticmethod
    def forward(ctx, x, gamma, weight, bias, eps):
        keep = any(ctx.needs_input_grad[:3])
        y, _, rstd, kept = ops.rms_norm(_dense(x), gamma, eps=eps, checkpoint=keep)
        ctx.save_for_backward(kept.buffer if keep else None, rstd, gamma, weight)
        ctx.width = x.shape[-1]
        return _recorded_linear(y, weight, bias, ctx.needs_input_grad[2])

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        return *_rms_linear_backward(ctx, dy, None, ctx.needs_input_grad[:4]), None


def _rms_linear_backward(ctx, dy, dh, needs):
    """(dx, dgamma, dW, db); the output's gradient dy or the stream's dh may be none."""
    buffer, rstd, gamma, weight = ctx.saved_tensors
    if dy is None:
        return (None if dh is None or not needs[0] else _dense(dh)), None, None, None
    kept = None if buffer is None else ops.Act8.from_buffer(buffer, ctx.width)
    norm = needs[0] or needs[1]
    dn, dw, db = _linear_backward(_dense(dy), kept, weight, (norm, *needs[2:4]), (gamma, None))
    dx = dgamma = None
    if norm:
        dx, dgamma = ops.rms_norm_backward(dn, kept, rstd, gamma, dh=None if dh is None else _dense(dh), grad_dtype=gamma.dtype)
    return dx, dgamma, dw, db


class _Embedding(torch.autograd.Function):
    @staticmethod
    def forward(ctx, ids, weight, scale, dtype):
        ctx.save_for_backward(ids)
        ctx.vocab, ctx.scale, ctx.dtype = weight.shape[0], scale, weight.dtype
        return ops.embedding(ids, weight, scale, dtype)

    @staticmethod
    @once_differentiable
    def backward(ctx, dout):
        ids, = ctx.saved_tensors
        return None, ops.embedding_grad(_dense(dout), ids, ctx.vocab, ctx.scale, ctx.dtype), None, None


def _recorded(*inputs):
    return torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in inputs)


def norm_linear(x, gamma, beta, weight, bias=None, eps: float = 1e-5):
    """linear(layer_norm(x, gamma, beta), weight, bias), kept in 8 bits for the backward pass
    (where there is one to come).  beta and bias may be None."""
    if not _recorded(x, gamma, beta, weight, bias):
        return _linear(ops.layer_norm(_dense(x), gamma, beta, eps)[0], weight, bias)
    return _NormLinear.apply(x, gamma, beta, weight, bias, eps)


def rms_linear(x, residual, gamma, weight, bias=None, eps: float = 1e-6):
    """(linear(rms_norm(h, gamma), weight, bias), h) with h = x + residual (residual None: h is x),
    kept in 8 bits for the backward pass (where there is one to come).  bias may be None."""
    if not _recorded(x, residual, gamma, weight, bias):
        y, h, _, _ = ops.rms_norm(_dense(x), gamma, residual=None if residual is None else _dense(residual), eps=eps)
        return _linear(y, weight, bias), h
    if residual is None:
        return _RmsLinearOnly.apply(x, gamma, weight, bias, eps), x
    return _RmsLinear.apply(x, residual, gamma, weight, bias, eps)


def embedding(ids, weight, scale: float = 1.0, dtype=None):
    """scale weight[ids] of ``dtype`` (None: the weight's); an id outside the table stands for no
    token, gives zeros and takes no part in the gradient."""
    return _Embedding.apply(ids, weight, scale, dtype)


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


class RmsLinear8(torch.nn.Module):
    def __init__(self, n_in: int, n_out: int, eps: float = 1e-6, bias: bool = False, device="cuda"):
        super().__init__()
        self.eps = eps
        self.gamma = torch.nn.Parameter(torch.ones(n_in, device=device))
        self.weight, b = _linear_parameters(n_in, n_out, device)
        self.bias = b if bias else None

    def forward(self, x, residual=None):
        return rms_linear(x, residual, self.gamma, self.weight, self.bias, self.eps)


class RmsMlpBlock8(torch.nn.Module):
    """(delta, stream) -> (W2 f(W1 rms_norm(h)), h), h = stream + delta (stream None: delta): what the
    block adds to the stream is added by the next one's norm."""

    def __init__(self, width: int, hidden: int, kind: str = "silu", eps: float = 1e-6, device="cuda"):
        super().__init__()
        self.up = RmsLinear8(width, hidden, eps, device=device)
        self.down = ActLinear8(hidden, width, kind, device)

    def forward(self, delta, stream=None):
        u, h = self.up(delta, stream)
        return self.down(u), h


class Embedding(torch.nn.Module):
    def __init__(self, vocab: int, width: int, scale: float = 1.0, dtype=torch.bfloat16, device="cuda"):
        super().__init__()
        self.scale, self.dtype = scale, dtype
        self.weight = torch.nn.Parameter(torch.empty(vocab, width, device=device).normal_(0.0, 0.02))

    def forward(self, ids):
        return embedding(ids, self.weight, self.scale, self.dtype)
