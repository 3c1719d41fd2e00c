"""The training operators in 64 bits, on the host, written from their definitions, and the error that
fp32 arithmetic may add to them.

U is the unit roundoff of fp32.  A sum of n terms in fp32, in any order, is off by at most (n - 1) U times
the sum of the terms' magnitudes (to first order); `chain(n)` is the n to use where at most n / 32 terms are
added one after another and the rest in a tree."""
import math

import torch

U = 2.0 ** -24
U16 = 2.0 ** -8           # unit roundoff of bf16 (8 significant bits)


def chain(n):
    return n / 32 + 16


def rounding(value, dtype):
    """What storing `value` in `dtype` may add (fp32: already in the arithmetic's bound)."""
    return value.abs() * (U16 if dtype == torch.bfloat16 else U) + 1e-38


def two_to(e):
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def act8_forms(x):
    """(codes, exps) of an exactly held matrix."""
    x = x.double()
    rows, cols = x.shape
    pitch = (cols + 31) // 32 * 32
    wide = torch.zeros(rows, pitch, dtype=torch.float64)
    wide[:, :cols] = x
    blocks = wide.view(rows, -1, 32)
    bad = ~torch.isfinite(blocks).all(2)
    top = blocks.abs().amax(2)
    top = torch.where(bad, torch.zeros_like(top), top)
    _, e = torch.frexp(top)                         # top = m 2^e, m in [1/2, 1)
    exps = torch.where(top > 0, e.long() - 1 - 6 + 127, torch.zeros_like(e).long()).clamp(min=0)
    codes = torch.round(blocks / two_to(exps - 127)[..., None]).clamp(-127, 127)
    codes = torch.where(bad[..., None], torch.zeros_like(codes), codes)
    exps = torch.where(bad, torch.full_like(exps, 255), exps)
    return codes.view(rows, pitch).to(torch.int8), exps.to(torch.uint8)


def act8_values(codes, exps, cols):
    codes, exps = codes.cpu().double(), exps.cpu().long()
    scale = torch.where(exps == 255, torch.full(exps.shape, math.nan, dtype=torch.float64), two_to(exps - 127))
    return (codes.view(exps.shape[0], -1, 32) * scale[..., None]).view(codes.shape)[:, :cols]


def layer_norm(x, w, b, eps):
    x, w = x.cpu().double(), w.cpu().double()
    b = torch.zeros_like(w) if b is None else b.cpu().double()
    mean = x.mean(1)
    var = (x - mean[:, None]).square().mean(1)
    rstd = 1.0 / torch.sqrt(var + eps)
    xhat = (x - mean[:, None]) * rstd[:, None]
    return xhat * w + b, mean, rstd, xhat


def layer_norm_bounds(x, w, b, eps, dtype):
    """Bounds of (y, mean, rstd, xhat): the mean is off by n U mean|x|; that moves the sum of squares only
    in second order, whose own rounding is n U relative; root and quotient add 3 U."""
    y, mean, rstd, xhat = layer_norm(x, w, b, eps)
    w = w.cpu().double()
    n = chain(x.shape[1])
    dmean = n * U * x.cpu().double().abs().mean(1) + U * mean.abs()
    # second order: (dmean / sigma)^2 / 2 relative
    drstd = rstd * ((n + 8) * U + 0.5 * (dmean * rstd) ** 2)
    dxhat = (dmean * rstd)[:, None] + xhat.abs() * ((drstd / rstd)[:, None] + 4 * U)
    dy = dxhat * w.abs() + 2 * U * (xhat * w).abs() + rounding(y, dtype)
    return dy, dmean, drstd, dxhat


def layer_norm_backward(dy, xhat, rstd, w):
    dy, xhat, rstd, w = (t.cpu().double() for t in (dy, xhat, rstd, w))
    g = dy * w
    dx = rstd[:, None] * (g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True))
    return dx, (dy * xhat).sum(0), dy.sum(0)


def layer_norm_backward_bounds(dy, xhat, rstd, w, dtype, grad_dtype, xhat_err=0.0):
    """xhat_err: relative error of the xhat that the kernel forms (3 U where it comes from x)."""
    dx, dw, db = layer_norm_backward(dy, xhat, rstd, w)
    dy, xhat, rstd, w = (t.cpu().double() for t in (dy, xhat, rstd, w))
    g = (dy * w).abs()
    gx = (g * xhat.abs())
    n = chain(dy.shape[1]) + 6
    m1, m2 = g.mean(1, keepdim=True), gx.mean(1, keepdim=True)
    e = rstd[:, None] * (n * U * m1 + xhat.abs() * (n * U + 2 * xhat_err) * m2 + 6 * U * (g + m1 + xhat.abs() * m2))
    r = dy.shape[0] + 4
    dwb = (r * U + xhat_err) * (dy * xhat).abs().sum(0) + rounding(dw, grad_dtype)
    dbb = r * U * dy.abs().sum(0) + rounding(db, grad_dtype)
    return e + rounding(dx, dtype), dwb, dbb


def act(kind, u):
    u = u.cpu().double()
    if kind == "gelu":
        return u * 0.5 * torch.special.erfc(-u / math.sqrt(2))
    z2 = math.sqrt(8 / math.pi) * (u + 0.044715 * u ** 3)
    return u * torch.sigmoid(z2 if kind == "gelu_tanh" else u)


def act_slope(kind, u):
    u = u.cpu().double()
    if kind == "gelu":
        return 0.5 * torch.special.erfc(-u / math.sqrt(2)) + u * torch.exp(-u * u / 2) / math.sqrt(2 * math.pi)
    if kind == "silu":
        p = torch.sigmoid(u)
        return p + u * p * torch.sigmoid(-u)
    c = math.sqrt(8 / math.pi)
    z2 = c * (u + 0.044715 * u ** 3)
    return torch.sigmoid(z2) + u * torch.sigmoid(z2) * torch.sigmoid(-z2) * c * (1 + 3 * 0.044715 * u * u)


def act_bound(value, u, dtype):
    """The functions are good to 2^-21 of max(1, |u|) in fp32."""
    return 2.0 ** -21 * u.cpu().double().abs().clamp(min=1) + rounding(value, dtype)


def weight_grad(dy, h):
    dy, h = dy.cpu().double(), h.cpu().double()
    return dy.t() @ h, dy.sum(0)


def weight_grad_bounds(dy, h, grad_dtype, affine=None):
    """Products are exact or rounded once; every addition may be off by an ulp (2 U: sums that round
    toward zero are allowed for).  With `affine` = (xhat, w, b) the two addends are summed apart."""
    dw, db = weight_grad(dy, h)
    dy, h = dy.cpu().double().abs(), h.cpu().double().abs()
    n = 2 * (dy.shape[0] + 8) * U
    total = dy.t() @ h
    if affine is not None:
        xhat, w, b = (t.cpu().double().abs() for t in affine)
        total = (dy.t() @ xhat) * w + dy.sum(0)[:, None] * b
    return n * total + rounding(dw, grad_dtype), n * dy.sum(0) + rounding(db, grad_dtype)


def assert_within(got, want, bound, what):
    got = got.detach().cpu().double()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    bad_want, bad_got = ~torch.isfinite(want), ~torch.isfinite(got)
    assert torch.equal(bad_want, bad_got), f"{what}: non-finite values in other places"
    off = torch.where(bad_want, torch.zeros_like(want), (got - want).abs() - bound)
    if off.numel():
        worst = int(off.reshape(-1).argmax())
        assert float(off.reshape(-1)[worst]) <= 0, (
            f"{what}: {got.reshape(-1)[worst].item()!r} for {want.reshape(-1)[worst].item()!r}, "
            f"{float(off.reshape(-1)[worst])!r} over the bound at {worst}")
