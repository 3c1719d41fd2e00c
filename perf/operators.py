"""The training operators in their plain form, and the calls that a user makes of them.

The cases are the pieces of a pre-norm MLP block's training step that keeps what its
backward pass needs in 8 bits: the 8-bit checkpoint itself, layer norm, an activation
function, and the weight gradient of a linear layer from the checkpoint of its input.

The checkpoint's format: 32 consecutive features of a row share an exponent byte E
(scale 2^(E-127)), the codes are int8 in [-127, 127], rows are padded to a multiple of
32 codes.  E is the exponent of the block's largest magnitude less 6, so that it falls
into [64, 128) scales; codes are rounded to nearest, ties to even, and clamped to 127.
"""
import math

import torch

own = False

BLOCK = 32
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZES = {"f32": 4, "bf16": 2}


# ---------------------------------------------------------------------------
# The cases
# ---------------------------------------------------------------------------
def listed():
    return [
        # hidden states of a wide layer put away in 8 bits and brought back
        dict(name="pack 8192x4096 bf16", op="pack", rows=8192, cols=4096, type="bf16"),
        # the 1000 logits of one 197-token image: small, and no multiple of the block
        dict(name="pack 197x1000 f32", op="pack", rows=197, cols=1000, type="f32"),
        # ViT-B/16's layer norm over a batch of 64 images, checkpointed for its backward pass
        dict(name="norm 12608x768 bf16", op="norm", rows=12608, cols=768, type="bf16", param="f32", save=True),
        # the same layer norm on a single token, as in evaluation: nothing is kept
        dict(name="norm 1x768 bf16", op="norm", rows=1, cols=768, type="bf16", param="bf16", save=False),
        # its backward pass from the checkpoint
        dict(name="norm_back 12608x768 bf16", op="norm_back", rows=12608, cols=768, type="bf16", param="f32",
             saved="8 bits"),
        # fp32 training at a wide layer and an odd number of tokens, from the input itself
        dict(name="norm_back 4099x4096 f32", op="norm_back", rows=4099, cols=4096, type="f32", param="f32",
             saved="input"),
        # ViT-B/16's MLP activation over 64 images: forward pass with both checkpoints, backward pass
        dict(name="act 12608x3072 gelu bf16", op="act", kind="gelu", rows=12608, cols=3072, type="bf16"),
        # one 197-token image, an odd width, fp32
        dict(name="act 197x1003 silu f32", op="act", kind="silu", rows=197, cols=1003, type="f32"),
        # the weight and bias gradient of ViT-B/16's qkv projection, whose input is a layer norm's output
        dict(name="weight 12608 768->2304 bf16", op="weight", rows=12608, n_in=768, n_out=2304, type="bf16",
             grad="bf16", norm=True, bias=True),
        # a square layer of VGG-16's width over a long batch, fp32 gradients for fp32 master weights
        dict(name="weight 16384 4096->4096 bf16", op="weight", rows=16384, n_in=4096, n_out=4096, type="bf16",
             grad="f32", norm=False, bias=False),
        # ResNet-50's classifier over a batch of 250, everything in fp32
        dict(name="weight 250 2048->1000 f32", op="weight", rows=250, n_in=2048, n_out=1000, type="f32",
             grad="f32", norm=False, bias=True),
        # a single token's outer product at odd sizes
        dict(name="weight 1 771->1001 bf16", op="weight", rows=1, n_in=771, n_out=1001, type="bf16", grad="f32",
             norm=True, bias=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A layer's width: any number, or a multiple of 64 as most layers have."""
    n = _log(rng, lo, hi)
    return n if rng.random() < 0.5 else max(64, n // 64 * 64)


def draw(rng):
    op = rng.choice(["pack", "norm", "norm_back", "act", "weight"])
    type_ = rng.choice(["f32", "bf16", "bf16"])
    rows = _log(rng, 1, 16384)
    if op == "weight":
        return dict(op=op, rows=rows, n_in=_width(rng, 16, 4096), n_out=_width(rng, 16, 4096), type=type_,
                    grad=rng.choice(["f32", "bf16"]), norm=rng.random() < 0.4, bias=rng.random() < 0.6)
    cols = _width(rng, 16, 8192)
    rows = max(1, min(rows, 33_554_432 // cols))       # at most the elements of the largest listed ones
    if op == "pack":
        return dict(op=op, rows=rows, cols=cols, type=type_)
    if op == "act":
        return dict(op=op, kind=rng.choice(["gelu", "gelu_tanh", "silu"]), rows=rows, cols=cols, type=type_)
    param = rng.choice(["f32", "bf16"])
    if op == "norm":
        return dict(op=op, rows=rows, cols=cols, type=type_, param=param, save=rng.random() < 0.7)
    return dict(op=op, rows=rows, cols=cols, type=type_, param=param, saved=rng.choice(["8 bits", "input"]))


def work(case):
    """Bytes that have to be moved and operations that have to be done: inputs read once, outputs written
    once; a checkpoint that the path both leaves and takes up counts for both."""
    op, rows, b = case["op"], case["rows"], SIZES[case["type"]]
    if op == "weight":
        n_in, n_out = case["n_in"], case["n_out"]
        moved = rows * n_out * b + _code_bytes(rows, n_in) + n_in * n_out * SIZES[case["grad"]]
        moved += (8 * n_in if case["norm"] else 0) + (n_out * SIZES[case["grad"]] if case["bias"] else 0)
        return {"bytes": moved, "flops": 2 * rows * n_in * n_out}
    cols = case["cols"]
    n, codes = rows * cols, _code_bytes(rows, cols)
    if op == "pack":
        return {"bytes": 2 * n * b + 2 * codes, "flops": 4 * n}
    if op == "norm":
        moved = 2 * n * b + 8 * rows + 2 * cols * SIZES[case["param"]]
        return {"bytes": moved + (2 * codes + 2 * n if case["save"] else 0), "flops": 8 * n}
    if op == "norm_back":
        moved = 2 * n * b + cols * (SIZES[case["param"]] + 8) + 4 * rows
        return {"bytes": moved + (codes if case["saved"] == "8 bits" else n * b + 4 * rows), "flops": 14 * n}
    # forward: u read, a and two checkpoints written; one of them unpacked; backward: da and the other read, du written
    return {"bytes": 4 * n * b + 4 * codes + 2 * n, "flops": 40 * n}


def _code_bytes(rows, cols):
    blocks = -(-cols // BLOCK)
    return rows * blocks * (BLOCK + 1)


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------
def _hidden(rows, cols, gen):
    """Hidden states: features of unlike scales and offsets, a few of them large."""
    scale = torch.empty(cols, device="cuda").normal_(0.0, 0.5, generator=gen).exp_()
    shift = torch.empty(cols, device="cuda").normal_(0.0, 0.3, generator=gen)
    return torch.empty(rows, cols, device="cuda").normal_(generator=gen) * scale + shift


def _checkpoint(x):
    """(codes, exponents) of fp32 values, as the format says."""
    codes, exps = _pack(x)
    return codes.contiguous(), exps.contiguous()


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(1_000_003 * int(seed) + 7)
    op, rows, dtype = case["op"], case["rows"], DTYPES[case["type"]]
    s = dict(case)
    if op == "weight":
        n_in, n_out = case["n_in"], case["n_out"]
        s["dy"] = torch.empty(rows, n_out, device="cuda").normal_(0.0, 1e-3, generator=gen).to(dtype)
        x = _hidden(rows, n_in, gen)
        if case["norm"]:
            x = x - x.mean(1, keepdim=True)
            x = x / (x.square().mean(1, keepdim=True) + 1e-5).sqrt()
            s["weight"] = torch.empty(n_in, device="cuda").normal_(1.0, 0.1, generator=gen)
            s["bias_in"] = torch.empty(n_in, device="cuda").normal_(0.0, 0.1, generator=gen)
        s["codes"], s["exps"] = _checkpoint(x)
        return s
    cols = case["cols"]
    x = _hidden(rows, cols, gen)
    s["x"] = x.to(dtype)
    if op in ("norm", "norm_back"):
        param = DTYPES[case["param"]]
        s["weight"] = torch.empty(cols, device="cuda").normal_(1.0, 0.1, generator=gen).to(param)
        s["bias_in"] = torch.empty(cols, device="cuda").normal_(0.0, 0.1, generator=gen).to(param)
    if op == "norm_back":
        s["dy"] = torch.empty(rows, cols, device="cuda").normal_(0.0, 1e-3, generator=gen).to(dtype)
        x = s["x"].float()
        s["mean"] = x.mean(1)
        x = x - s["mean"][:, None]
        s["rstd"] = 1.0 / (x.square().mean(1) + 1e-5).sqrt()
        if case["saved"] == "8 bits":
            s["codes"], s["exps"] = _checkpoint(x * s["rstd"][:, None])
            del s["x"]
    if op == "act":
        s["da"] = torch.empty(rows, cols, device="cuda").normal_(0.0, 1e-3, generator=gen).to(dtype)
    return s


# ---------------------------------------------------------------------------
# The operators: a user's calls, and the plain form
# ---------------------------------------------------------------------------
_ops = None


def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(s):
    global _ops
    if _ops is None:
        from paper_2601_07876_b200 import ops
        _ops = ops
    ops, op = _ops, s["op"]
    if op == "pack":
        return ops.act8_unpack(ops.act8_pack(s["x"]), dtype=s["x"].dtype)
    if op == "norm":
        y, mean, rstd, kept = ops.layer_norm(s["x"], s["weight"], s["bias_in"], eps=1e-5, checkpoint=s["save"])
        out = dict(y=y, mean=mean, rstd=rstd)
        if s["save"]:
            out["xhat"] = ops.act8_unpack(kept)
        return out
    if op == "norm_back":
        if s["saved"] == "8 bits":
            kept = ops.Act8(s["codes"], s["exps"], s["cols"])
            dx, dw, db = ops.layer_norm_backward(s["dy"], kept, s["rstd"], s["weight"])
        else:
            dx, dw, db = ops.layer_norm_backward(s["dy"], s["x"], s["rstd"], s["weight"], mean=s["mean"])
        return dict(dx=dx, dw=dw, db=db)
    if op == "act":
        a, kept_u, kept_a = ops.activation(s["x"], s["kind"], save_input=True, save_output=True)
        du = ops.activation_backward(s["da"], kept_u, s["kind"])
        return dict(a=a, du=du, kept=ops.act8_unpack(kept_a))
    kept = ops.Act8(s["codes"], s["exps"], s["n_in"])
    affine = (s["weight"], s["bias_in"]) if s["norm"] else None
    dw, db = ops.linear_weight_grad(s["dy"], kept, affine=affine, bias=s["bias"], dtype=DTYPES[s["grad"]])
    return dict(dw=dw, db=db) if s["bias"] else dict(dw=dw)


def _pack(x):
    rows, cols = x.shape
    blocks = -(-cols // BLOCK)
    if blocks * BLOCK != cols:
        wide = torch.zeros(rows, blocks * BLOCK, device=x.device)
        wide[:, :cols] = x
        x = wide
    x = x.reshape(rows, blocks, BLOCK)
    largest = x.abs().amax(2)
    exps = ((largest.view(torch.int32) >> 23) - 6).clamp(min=0)
    inverse = ((254 - exps) << 23).view(torch.float32)
    codes = torch.round(x * inverse[:, :, None]).clamp(-127, 127).to(torch.int8)
    return codes.view(rows, blocks * BLOCK), exps.to(torch.uint8)


def _values(codes, exps, cols):
    rows, blocks = exps.shape
    scale = (exps.to(torch.int32) << 23).view(torch.float32)
    return (codes.view(rows, blocks, BLOCK).float() * scale[:, :, None]).view(rows, blocks * BLOCK)[:, :cols]


def _f(kind, u):
    if kind == "gelu":
        return 0.5 * u * (1.0 + torch.erf(u * math.sqrt(0.5)))
    if kind == "gelu_tanh":
        return 0.5 * u * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (u + 0.044715 * u * u * u)))
    return u / (1.0 + torch.exp(-u))


def _df(kind, u):
    if kind == "gelu":
        cdf = 0.5 * (1.0 + torch.erf(u * math.sqrt(0.5)))
        return cdf + u * torch.exp(-0.5 * u * u) * (1.0 / math.sqrt(2.0 * math.pi))
    if kind == "gelu_tanh":
        c = math.sqrt(2.0 / math.pi)
        t = torch.tanh(c * (u + 0.044715 * u * u * u))
        return 0.5 * (1.0 + t) + 0.5 * u * (1.0 - t * t) * c * (1.0 + 3 * 0.044715 * u * u)
    p = 1.0 / (1.0 + torch.exp(-u))
    return p * (1.0 + u * (1.0 - p))


def _run_plain(s):
    op = s["op"]
    if op == "pack":
        codes, exps = _pack(s["x"].float())
        return _values(codes, exps, s["cols"]).to(s["x"].dtype).contiguous()
    if op == "norm":
        x = s["x"].float()
        mean = x.mean(1)
        x = x - mean[:, None]
        rstd = 1.0 / (x.square().mean(1) + 1e-5).sqrt()
        x = x * rstd[:, None]
        y = x * s["weight"].float() + s["bias_in"].float()
        out = dict(y=y.to(s["x"].dtype), mean=mean, rstd=rstd)
        if s["save"]:
            codes, exps = _pack(x)
            out["xhat"] = _values(codes, exps, s["cols"]).to(torch.bfloat16).contiguous()
        return out
    if op == "norm_back":
        dy, rstd = s["dy"].float(), s["rstd"][:, None]
        if s["saved"] == "8 bits":
            x = _values(s["codes"], s["exps"], s["cols"])
        else:
            x = (s["x"].float() - s["mean"][:, None]) * rstd
        g = dy * s["weight"].float()
        dx = rstd * (g - g.mean(1, keepdim=True) - x * (g * x).mean(1, keepdim=True))
        return dict(dx=dx.to(s["dy"].dtype), dw=(dy * x).sum(0), db=dy.sum(0))
    if op == "act":
        u = s["x"].float()
        a = _f(s["kind"], u).to(s["x"].dtype)
        codes, exps = _pack(u)
        du = s["da"].float() * _df(s["kind"], _values(codes, exps, s["cols"]))
        # what is kept of the output is what the next layer reads of it: the rounded one
        codes, exps = _pack(a.float())
        return dict(a=a, du=du.to(s["da"].dtype), kept=_values(codes, exps, s["cols"]).to(torch.bfloat16).contiguous())
    x = _values(s["codes"], s["exps"], s["n_in"])
    if s["norm"]:
        x = x * s["weight"] + s["bias_in"]
    dy = s["dy"].float()
    out = dict(dw=torch.matmul(dy.t(), x).to(DTYPES[s["grad"]]))
    if s["bias"]:
        out["db"] = dy.sum(0).to(DTYPES[s["grad"]])
    return out


# ---------------------------------------------------------------------------
# The definitions in 64 bits
# ---------------------------------------------------------------------------
def _two_to(e):
    """2^e in 64 bits from its bits: pow() may be an ulp off, which decides ties."""
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def _stands_for64(x):
    """What the checkpoint of 64-bit values stands for: each block on the grid of 2^(e - 6), e the exponent
    of its largest magnitude."""
    rows, cols = x.shape
    pad = -cols % BLOCK
    x = torch.cat([x, x.new_zeros(rows, pad)], 1).view(rows, -1, BLOCK)
    _, e = torch.frexp(x.abs().amax(2, keepdim=True))       # largest = m 2^e, m in [1/2, 1)
    step = _two_to(e - 7)
    return ((x / step).round().clamp(-127, 127) * step).view(rows, -1)[:, :cols]


def _decoded64(codes, exps, cols):
    step = _two_to(exps.to(torch.int64) - 127).repeat_interleave(BLOCK, 1)
    return (codes.double() * step)[:, :cols]


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "pack":
        return _stands_for64(s["x"].double())
    if op == "weight":
        x = _decoded64(s["codes"], s["exps"], case["n_in"])
        if case["norm"]:
            x = x * s["weight"].double() + s["bias_in"].double()
        out = dict(dw=s["dy"].double().t() @ x)
        if case["bias"]:
            out["db"] = s["dy"].double().sum(0)
        return out
    if op == "act":
        u, da = s["x"].double(), s["da"].double()
        f, back = _exact_f[case["kind"]]
        a = f(u)
        # (the kept output goes by the rounded one)
        return dict(a=a, du=da * back(_stands_for64(u)), kept=_stands_for64(a.to(s["x"].dtype).double()))
    w, b = s["weight"].double(), s["bias_in"].double()
    if op == "norm":
        x = s["x"].double()
        mean, var = x.mean(1), x.var(1, unbiased=False)
        rstd = (var + 1e-5).rsqrt()
        xhat = (x - mean[:, None]) * rstd[:, None]
        out = dict(y=xhat * w + b, mean=mean, rstd=rstd)
        if case["save"]:
            out["xhat"] = _stands_for64(xhat)
        return out
    dy, rstd = s["dy"].double(), s["rstd"].double()
    if case["saved"] == "8 bits":
        xhat = _decoded64(s["codes"], s["exps"], case["cols"])
    else:
        xhat = (s["x"].double() - s["mean"].double()[:, None]) * rstd[:, None]
    g = dy * w
    proj = (g * xhat).sum(1) / case["cols"]
    dx = (g - g.mean(1)[:, None] - xhat * proj[:, None]) * rstd[:, None]
    return dict(dx=dx, dw=(dy * xhat).sum(0), db=dy.sum(0))


def _phi(z):
    return torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)


def _cdf(z):
    return torch.special.ndtr(z)


def _sig(z):
    return torch.sigmoid(z)


_C = math.sqrt(8 / math.pi)         # tanh-GELU is u times the logistic function of _C (u + 0.044715 u^3)


def _inner(u):
    return _C * (u + 0.044715 * u ** 3)


_exact_f = {
    "gelu": (lambda u: u * _cdf(u), lambda u: _cdf(u) + u * _phi(u)),
    "gelu_tanh": (lambda u: u * _sig(_inner(u)),
                  lambda u: _sig(_inner(u)) * (1 + u * _sig(-_inner(u)) * _C * (1 + 3 * 0.044715 * u ** 2))),
    "silu": (lambda u: u * _sig(u), lambda u: _sig(u) * (1 + u * _sig(-u))),
}
