"""The operators around a language model's residual stream (root-mean-square norm with the residual's addition,
token embedding, orthogonalised updates) in 64 bits, from their definitions, and the error that their arithmetic
may add.  U, U16, chain, rounding: see ops_reference."""
import math

import torch

from ops_reference import U, chain, rounding


# ---- root-mean-square norm ------------------------------------------------------
def add(x, residual):
    """h as it is stored: the sum rounded to fp32, then to the type."""
    if residual is None:
        return x.cpu()
    return (x.cpu().float() + residual.cpu().float()).to(x.dtype)


def rms_norm(h, w, eps):
    h, w = h.cpu().double(), w.cpu().double()
    rstd = 1.0 / torch.sqrt(h.square().mean(1) + eps)
    xhat = h * rstd[:, None]
    return xhat * w, rstd, xhat


def rms_norm_bounds(h, w, eps, dtype):
    """Bounds of (y, rstd, xhat): the sum of squares is off by n U relative, its mean and eps by 3 U more, and
    the reciprocal root by half of both and 2 ulp (4 U); one product behind that, two for y."""
    y, rstd, xhat = rms_norm(h, w, eps)
    n = chain(h.shape[1])
    drstd = rstd * ((n + 3) / 2 + 4) * U
    dxhat = xhat.abs() * (drstd / rstd)[:, None] + U * xhat.abs()
    return dxhat * w.cpu().double().abs() + 2 * U * y.abs() + rounding(y, dtype), drstd, dxhat


def rms_norm_backward(dy, xhat, rstd, w, dh=None):
    dy, xhat, rstd, w = (t.cpu().double() for t in (dy, xhat, rstd, w))
    g = dy * w
    dx = rstd[:, None] * (g - xhat * (g * xhat).mean(1, keepdim=True))
    return (dx if dh is None else dx + dh.cpu().double()), (dy * xhat).sum(0)


def rms_norm_backward_bounds(dy, xhat, rstd, w, dtype, grad_dtype, dh=None, xhat_err=0.0):
    """xhat_err: relative error of the xhat that the kernel forms (U where it comes from h)."""
    dx, dw = rms_norm_backward(dy, xhat, rstd, w, dh)
    dy, xhat, rstd, w = (t.cpu().double() for t in (dy, xhat, rstd, w))
    g = (dy * w).abs()
    m = (g * xhat.abs()).mean(1, keepdim=True)
    n = chain(dy.shape[1]) + 6
    e = rstd[:, None] * (xhat.abs() * (n * U + 2 * xhat_err) * m + 6 * U * (g + xhat.abs() * m))
    if dh is not None:
        e = e + 2 * U * (dh.cpu().double().abs() + rstd[:, None] * (g + xhat.abs() * m))
    r = dy.shape[0] + 4
    return e + rounding(dx, dtype), (r * U + xhat_err) * (dy * xhat).abs().sum(0) + rounding(dw, grad_dtype)


# ---- embedding ------------------------------------------------------------------
def embedding(ids, table, scale, dtype):
    """To the bit: one product in fp32, rounded once."""
    ids, table = ids.cpu().long(), table.cpu().float()
    there = (ids >= 0) & (ids < table.shape[0])
    out = torch.zeros(*ids.shape, table.shape[1])
    out[there] = table[ids[there]] * torch.tensor(scale, dtype=torch.float32)
    return out.to(dtype)


def embedding_grad(dout, ids, vocab, scale, base=None):
    """(gradient, sum of magnitudes, tokens of each id)"""
    dout, ids = dout.cpu().double().reshape(-1, dout.shape[-1]), ids.cpu().long().reshape(-1)
    there = (ids >= 0) & (ids < vocab)
    scale = float(torch.tensor(scale, dtype=torch.float32))
    total = torch.zeros(vocab, dout.shape[1], dtype=torch.float64).index_add_(0, ids[there], dout[there])
    size = torch.zeros(vocab, dout.shape[1], dtype=torch.float64).index_add_(0, ids[there], dout[there].abs())
    count = torch.bincount(ids[there], minlength=vocab)
    return total * scale + (0 if base is None else base.cpu().double()), size * abs(scale), count


def embedding_grad_bound(want, size, count, grad_dtype, base=None):
    """A sum of n terms in fp32 in any order, the product with the scale, the addition to what was there."""
    bound = (count[:, None].double() + 2) * U * size + rounding(want, grad_dtype)
    return bound if base is None else bound + U * want.abs()


# ---- orthogonalised updates -----------------------------------------------------
STEPS = ((3.4445, -4.7750, 2.0315),) * 5


def orthogonalized(g, coefficients=STEPS, eps=1e-7):
    x = g.cpu().double()
    norm = float(x.norm())
    if norm == 0.0:
        return x
    x = x / max(norm, eps)
    tall = x.shape[0] > x.shape[1]
    x = x.t() if tall else x
    for a, b, c in coefficients:
        gram = x @ x.t()
        x = a * x + (b * gram + c * (gram @ gram)) @ x
    return x.t() if tall else x


def orthogonal_tolerance(rows, cols, steps=5):
    """How far X may be from the exact one, in the Frobenius norm, relative, with the coefficients above.
    u = 2^-12 is half a step of an operand in fp16.  At singular values around 1, where all end, a step adds, with
    t = s^2 <= 1.45, |B| = |b t + c t^2| <= 2.81 and |b + 2 c t| t <= 2.81: through the operand X of B X 2.81 u, through
    the operands of A, both X, 2 * 2.81 u / sqrt(2), through A' and B' 1.41 u and 2.81 u, and with |p'| <= 1.2 there it
    does not grow any more.  Roundings are independent, a uniform one u / sqrt(3) in the mean square: 5.6 u / sqrt(3)
    a step, sqrt(steps) times that in all, 1.8e-3; twice that is allowed where there are enough elements for means to
    hold, and the plain sum, 11 u a step, for matrices with a side below 16."""
    u = 2.0 ** -12
    if min(rows, cols) < 16:
        return 11 * u * steps
    return 2 * 5.6 * u / math.sqrt(3) * math.sqrt(steps)
