"""Operators around a language model's residual stream in their plain form, and the calls that a user makes
of them: the token embedding that starts the stream and its gradient, the root-mean-square norm with the
residual's addition at each block's door and its backward pass, and the orthogonalised update (Newton-Schulz
products) of the weight matrices whose gradients come out at the end.

The 8-bit form of a normalised row is the framework's: 32 consecutive features share an exponent byte E
(scale 2^(E-127)), the codes are int8 in [-127, 127], rows are padded to a multiple of 32 codes.  E is the
exponent of the block's largest magnitude less 6; codes are rounded to nearest, ties to even, and clamped.
"""
import math

import torch

own = False

BLOCK = 32
EPS = 1e-6                       # of the norm
TINY = 1e-7                      # the least Frobenius norm that a matrix is divided by
NEWTON_SCHULZ = ((3.4445, -4.7750, 2.0315),) * 5
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "i64": torch.int64, "i32": torch.int32}
SIZES = {"f32": 4, "bf16": 2, "i64": 8, "i32": 4}


# ---------------------------------------------------------------------------
# The cases
# ---------------------------------------------------------------------------
def listed():
    return [
        # the update of a square layer of VGG-16's width, from fp32 momentum
        dict(name="orth 4096x4096 f32", op="orth", shapes="4096x4096", type="f32"),
        # the attention matrices of ViT-B/16's twelve blocks, one call for all of them
        dict(name="orth 12x(2304x768, 768x768) bf16", op="orth", shapes="2304x768*12 768x768*12", type="bf16"),
        # ResNet-50's classifier, wide and of odd height
        dict(name="orth 1001x2048 f32", op="orth", shapes="1001x2048", type="f32"),
        # a small adapter's matrix: latency
        dict(name="orth 33x770 bf16", op="orth", shapes="33x770", type="bf16"),
        # the norm before a block of width 768 over 64 sequences of 197 tokens, kept in 8 bits for its backward pass
        dict(name="norm 12608x768 bf16", op="norm", rows=12608, cols=768, type="bf16", param="f32", residual=True,
             save=True),
        # one token of a wide model, as in answering: nothing is kept
        dict(name="norm 1x4096 bf16", op="norm", rows=1, cols=4096, type="bf16", param="bf16", residual=True, save=False),
        # its backward pass from the 8-bit form, with the gradient that comes down the stream
        dict(name="norm_back 12608x768 bf16", op="norm_back", rows=12608, cols=768, type="bf16", param="f32",
             saved="8 bits", stream=True),
        # fp32 training at a wide layer and an odd number of tokens, from the stream itself
        dict(name="norm_back 4099x4096 f32", op="norm_back", rows=4099, cols=4096, type="f32", param="f32",
             saved="input", stream=True),
        # a batch of 16 sequences of 1024 tokens through an fp32 master table, scaled, into a bf16 stream
        dict(name="embed 16384 of 50000x768 f32", op="embed", tokens=16384, vocab=50000, dim=768, ids="i64", table="f32",
             out="bf16", scaled=True, padded=False),
        # the next token of 8 sequences being answered
        dict(name="embed 8 of 32000x4096 bf16", op="embed", tokens=8, vocab=32000, dim=4096, ids="i32", table="bf16",
             out="bf16", scaled=False, padded=False),
        # the gradient of that batch for the fp32 master table; the ids are as unevenly spread as words are
        dict(name="embed_grad 16384 of 50000x768 bf16", op="embed_grad", tokens=16384, vocab=50000, dim=768, ids="i64",
             type="bf16", grad="f32", scaled=True, padded=True),
        # one sequence of 197 tokens over 1003 classes of patches, odd width, everything in fp32
        dict(name="embed_grad 197 of 1003x771 f32", op="embed_grad", tokens=197, vocab=1003, dim=771, ids="i32", type="f32",
             grad="f32", scaled=False, padded=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A layer's width: any number, or a multiple of 64 as most layers have."""
    n = _log(rng, lo, hi)
    return n if rng.random() < 0.5 else max(64, n // 64 * 64)


def draw(rng):
    op = rng.choice(["orth", "norm", "norm_back", "embed", "embed_grad"])
    type_ = rng.choice(["f32", "bf16"])
    if op == "orth":
        left, parts = work(listed()[0])["flops"], []
        for _ in range(rng.choice([1, 1, 2, 3])):
            rows, cols = _width(rng, 8, 4096), _width(rng, 8, 4096)
            one = _orth_flops(rows, cols)
            count = max(0, min(_log(rng, 1, 24), left // one))
            if count:
                parts.append("%dx%d*%d" % (rows, cols, count))
                left -= one * count
        return dict(op=op, shapes=" ".join(parts), type=type_)
    if op in ("norm", "norm_back"):
        cols = _width(rng, 16, 8192)
        rows = max(1, min(_log(rng, 1, 16384), 16_777_216 // cols))
        case = dict(op=op, rows=rows, cols=cols, type=type_, param=rng.choice(["f32", "bf16"]))
        if op == "norm":
            return dict(case, residual=rng.random() < 0.7, save=rng.random() < 0.6)
        return dict(case, saved=rng.choice(["8 bits", "input"]), stream=rng.random() < 0.7)
    vocab, dim = _log(rng, 100, 128000), _width(rng, 16, 4096)
    vocab = min(vocab, 50000 * 768 // dim)                     # at most the listed table
    tokens = max(1, min(_log(rng, 1, 65536), 16384 * 768 // dim))
    case = dict(op=op, tokens=tokens, vocab=vocab, dim=dim, ids=rng.choice(["i64", "i32"]), scaled=rng.random() < 0.5,
                padded=rng.random() < 0.5)
    if op == "embed":
        return dict(case, table=type_, out=rng.choice(["f32", "bf16"]))
    return dict(case, type=type_, grad=rng.choice(["f32", "bf16"]))


def _matrices(shapes):
    found = []
    for part in shapes.split():
        size, _, count = part.partition("*")
        rows, _, cols = size.partition("x")
        found += [(int(rows), int(cols))] * int(count or 1)
    return found


def _orth_flops(rows, cols):
    """A step of Newton-Schulz on the shorter side s: X X^T and its square are symmetric, half of each
    is enough (s^2 l + s^3 operations), and the product with X takes 2 s^2 l."""
    s, l = min(rows, cols), max(rows, cols)
    return len(NEWTON_SCHULZ) * (3 * s * s * l + s * s * s)


def work(case):
    """Bytes that have to be moved and operations that have to be done: inputs read once, outputs written
    once; a form that the path both leaves and takes up counts for both."""
    op = case["op"]
    if op == "orth":
        sizes = _matrices(case["shapes"])
        return {"bytes": sum(r * c for r, c in sizes) * (SIZES[case["type"]] + 2),
                "flops": sum(_orth_flops(r, c) for r, c in sizes)}
    if op in ("norm", "norm_back"):
        rows, cols, b = case["rows"], case["cols"], SIZES[case["type"]]
        n, codes = rows * cols, rows * -(-cols // BLOCK) * (BLOCK + 1)
        if op == "norm":
            moved = n * b * (4 if case["residual"] else 2) + 4 * rows + cols * SIZES[case["param"]]
            return {"bytes": moved + (2 * codes + 2 * n if case["save"] else 0), "flops": 6 * n}
        moved = n * b * (3 if case["stream"] else 2) + cols * (SIZES[case["param"]] + 4) + 4 * rows
        return {"bytes": moved + (codes if case["saved"] == "8 bits" else n * b), "flops": 10 * n}
    tokens, vocab, dim = case["tokens"], case["vocab"], case["dim"]
    if op == "embed":
        # rows of the table that are asked for twice are read once; words repeat, half of the tokens at most counts
        return {"bytes": tokens * (SIZES[case["ids"]] + dim * SIZES[case["out"]]) + min(tokens, vocab) * dim * SIZES[case["table"]] // 2,
                "flops": tokens * dim}
    return {"bytes": tokens * (SIZES[case["ids"]] + dim * SIZES[case["type"]]) + vocab * dim * SIZES[case["grad"]],
            "flops": tokens * dim}


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------
def _normal(gen, *shape, std=1.0):
    return torch.empty(*shape, device="cuda").normal_(0.0, std, generator=gen)


def _hidden(rows, cols, gen):
    """Hidden states: features of unlike scales and offsets, a few of them large."""
    return _normal(gen, rows, cols) * _normal(gen, cols, std=0.5).exp() + _normal(gen, cols, std=0.3)


def _gradient(rows, cols, gen):
    """A weight gradient: a few directions that matter, of falling strength, over noise."""
    rank = max(1, min(rows, cols) // 16)
    strength = torch.exp(-4.0 * torch.arange(rank, device="cuda") / rank)
    return 1e-3 * ((_normal(gen, rows, rank) * strength) @ _normal(gen, rank, cols) / math.sqrt(rank) + _normal(gen, rows, cols, std=0.2))


def _words(tokens, vocab, gen, padded):
    """Token ids whose frequency falls as one over their rank; -1 where a padded batch has none."""
    rank = torch.exp(torch.rand(tokens, device="cuda", generator=gen) * math.log(vocab + 1)).long() - 1
    ids = torch.randperm(vocab, device="cuda", generator=gen)[rank.clamp(0, vocab - 1)]
    if padded:
        ids[torch.rand(tokens, device="cuda", generator=gen) < 0.05] = -1
    return ids


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(1_000_003 * int(seed) + 11)
    op, s = case["op"], dict(case)
    if op == "orth":
        s["grads"] = [_gradient(r, c, gen).to(DTYPES[case["type"]]) for r, c in _matrices(case["shapes"])]
        return s
    if op in ("norm", "norm_back"):
        rows, cols, dtype = case["rows"], case["cols"], DTYPES[case["type"]]
        s["x"] = _hidden(rows, cols, gen).to(dtype)
        s["weight"] = (1.0 + _normal(gen, cols, std=0.1)).to(DTYPES[case["param"]])
        if op == "norm":
            s["stream_in"] = _hidden(rows, cols, gen).to(dtype) if case["residual"] else None
            return s
        s["dy"] = _normal(gen, rows, cols, std=1e-3).to(dtype)
        s["dh"] = _normal(gen, rows, cols, std=1e-3).to(dtype) if case["stream"] else None
        x = s["x"].float()
        s["rstd"] = 1.0 / (x.square().mean(1) + EPS).sqrt()
        if case["saved"] == "8 bits":
            codes, exps = _pack(x * s["rstd"][:, None])
            s["codes"], s["exps"] = codes.contiguous(), exps.contiguous()
            del s["x"]
        return s
    tokens, vocab, dim = case["tokens"], case["vocab"], case["dim"]
    s["tokens_in"] = _words(tokens, vocab, gen, case["padded"]).to(DTYPES[case["ids"]])
    s["scale"] = math.sqrt(dim) if case["scaled"] else 1.0
    if op == "embed":
        s["weight"] = _normal(gen, vocab, dim, std=0.02).to(DTYPES[case["table"]])
    else:
        s["dy"] = _normal(gen, tokens, dim, std=1e-3).to(DTYPES[case["type"]])
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
    if op == "orth":
        return ops.orthogonalize(s["grads"], coefficients=NEWTON_SCHULZ, eps=TINY)
    if op == "norm":
        y, h, rstd, kept = ops.rms_norm(s["x"], s["weight"], residual=s["stream_in"], eps=EPS, checkpoint=s["save"])
        out = dict(y=y, rstd=rstd)
        if s["residual"]:
            out["h"] = h
        if s["save"]:
            out["xhat"] = ops.act8_unpack(kept)
        return out
    if op == "norm_back":
        saved = ops.Act8(s["codes"], s["exps"], s["cols"]) if s["saved"] == "8 bits" else s["x"]
        dx, dw = ops.rms_norm_backward(s["dy"], saved, s["rstd"], s["weight"], dh=s["dh"])
        return dict(dx=dx, dw=dw)
    if op == "embed":
        return ops.embedding(s["tokens_in"], s["weight"], scale=s["scale"], dtype=DTYPES[s["out"]])
    return ops.embedding_grad(s["dy"], s["tokens_in"], s["vocab"], scale=s["scale"], dtype=DTYPES[s["grad"]])


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


def _orthogonal(g):
    x = g.float()
    tall = x.shape[0] > x.shape[1]
    x = x.t() if tall else x
    x = x / x.square().sum().sqrt().clamp(min=TINY)
    for a, b, c in NEWTON_SCHULZ:
        gram = x @ x.t()
        x = a * x + (b * gram + c * (gram @ gram)) @ x
    return (x.t() if tall else x).to(torch.bfloat16).contiguous()


def _run_plain(s):
    op = s["op"]
    if op == "orth":
        return [_orthogonal(g) for g in s["grads"]]
    if op == "norm":
        h = s["x"]
        if s["residual"]:
            h = (h.float() + s["stream_in"].float()).to(h.dtype)
        x = h.float()
        rstd = 1.0 / (x.square().mean(1) + EPS).sqrt()
        x = x * rstd[:, None]
        out = dict(y=(x * s["weight"].float()).to(h.dtype), rstd=rstd)
        if s["residual"]:
            out["h"] = h
        if s["save"]:
            codes, exps = _pack(x)
            out["xhat"] = _values(codes, exps, s["cols"]).to(torch.bfloat16).contiguous()
        return out
    if op == "norm_back":
        dy, rstd = s["dy"].float(), s["rstd"][:, None]
        x = _values(s["codes"], s["exps"], s["cols"]) if s["saved"] == "8 bits" else s["x"].float() * rstd
        g = dy * s["weight"].float()
        dx = rstd * (g - x * (g * x).mean(1, keepdim=True))
        if s["stream"]:
            dx = dx + s["dh"].float()
        return dict(dx=dx.to(s["dy"].dtype), dw=(dy * x).sum(0))
    ids = s["tokens_in"].long()
    there = (ids >= 0) & (ids < s["vocab"])
    if op == "embed":
        rows = s["weight"][torch.where(there, ids, torch.zeros_like(ids))].float() * s["scale"]
        return torch.where(there[:, None], rows, torch.zeros_like(rows)).to(DTYPES[s["out"]])
    total = torch.zeros(s["vocab"] + 1, s["dim"], device=ids.device)
    total.index_add_(0, torch.where(there, ids, torch.full_like(ids, s["vocab"])), s["dy"].float())
    return (total[:s["vocab"]] * s["scale"]).to(DTYPES[s["grad"]])


# ---------------------------------------------------------------------------
# The definitions in 64 bits
# ---------------------------------------------------------------------------
def _two_to(e):
    """2^e in 64 bits from its bits: pow() may be an ulp off, which decides ties."""
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def _stands_for64(x):
    """What the 8-bit form of 64-bit values stands for: each block on the grid of 2^(e - 6), e the exponent
    of its largest magnitude."""
    rows, cols = x.shape
    pad = -cols % BLOCK
    x = torch.cat([x, x.new_zeros(rows, pad)], 1).view(rows, -1, BLOCK)
    _, e = torch.frexp(x.abs().amax(2, keepdim=True))       # largest = m 2^e, m in [1/2, 1)
    step = _two_to(e - 7)
    return ((x / step).round().clamp(-127, 127) * step).view(rows, -1)[:, :cols]


def _orthogonal64(g):
    """x p(x^T x) or p(x x^T) x, whichever is the smaller product, p(t) = a + b t + c t^2 at each step."""
    x = g.double()
    x = x / max(float(torch.linalg.vector_norm(x)), TINY)
    one = torch.eye(min(x.shape), dtype=torch.float64, device=x.device)
    for a, b, c in NEWTON_SCHULZ:
        if x.shape[0] <= x.shape[1]:
            t = torch.mm(x, x.t())
            x = torch.mm(torch.addmm(b * t, t, t, alpha=c) + a * one, x)
        else:
            t = torch.mm(x.t(), x)
            x = torch.mm(x, torch.addmm(b * t, t, t, alpha=c) + a * one)
    return x


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "orth":
        return [_orthogonal64(g) for g in s["grads"]]
    if op == "norm":
        h = s["x"].double()
        if case["residual"]:
            # (what is normalised is the stream as it is stored)
            h = (h + s["stream_in"].double()).to(s["x"].dtype).double()
        rstd = (h.pow(2).sum(1) / case["cols"] + EPS).rsqrt()
        xhat = torch.einsum("rc,r->rc", h, rstd)
        out = dict(y=xhat * s["weight"].double(), rstd=rstd)
        if case["residual"]:
            out["h"] = s["x"].double() + s["stream_in"].double()
        if case["save"]:
            out["xhat"] = _stands_for64(xhat)
        return out
    if op == "norm_back":
        dy, rstd = s["dy"].double(), s["rstd"].double()
        if case["saved"] == "8 bits":
            step = _two_to(s["exps"].to(torch.int64) - 127).repeat_interleave(BLOCK, 1)
            xhat = (s["codes"].double() * step)[:, :case["cols"]]
        else:
            xhat = torch.einsum("rc,r->rc", s["x"].double(), rstd)
        g = dy * s["weight"].double()
        proj = torch.einsum("rc,rc->r", g, xhat) / case["cols"]
        dx = torch.einsum("rc,r->rc", g - xhat * proj[:, None], rstd)
        if case["stream"]:
            dx = dx + s["dh"].double()
        return dict(dx=dx, dw=torch.einsum("rc,rc->c", dy, xhat))
    ids = s["tokens_in"].long()
    there = (ids >= 0) & (ids < case["vocab"])
    if op == "embed":
        out = torch.zeros(case["tokens"], case["dim"], dtype=torch.float64, device="cuda")
        out[there] = s["weight"][ids[there]].double() * s["scale"]
        return out
    # tokens in the order of their ids: a token's id begins a new sum or continues the one before
    order = torch.sort(torch.where(there, ids, case["vocab"]), stable=True).indices
    kept = order[:int(there.sum())]
    found, counts = torch.unique_consecutive(ids[kept], return_counts=True)
    out = torch.zeros(case["vocab"], case["dim"], dtype=torch.float64, device="cuda")
    if len(kept):
        ends = counts.cumsum(0)
        out[found] = torch.segment_reduce(s["dy"][kept].double(), "sum", offsets=torch.cat([ends.new_zeros(1), ends]), axis=0)
    return out * s["scale"]
