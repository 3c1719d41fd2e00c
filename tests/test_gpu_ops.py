"""The training operators on the GPU against their definitions in 64 bits (ops_reference)."""
import ctypes
import math

import pytest
import torch

import ops_reference as R

gpu = pytest.mark.gpu
pytestmark = gpu
F32, BF16 = torch.float32, torch.bfloat16
TYPES = [F32, BF16]


@pytest.fixture(scope="module")
def ops():
    from paper_2601_07876_b200 import ops
    return ops


def gen(seed):
    return torch.Generator().manual_seed(seed)


def matrix(rows, cols, dtype, seed, offset=0, extra=0, scale=1.0):
    """A rows x cols CUDA matrix of unlike features whose rows are `extra` elements apart and whose first
    element sits `offset` elements off a 16-byte boundary."""
    stride = cols + extra
    g = gen(seed)
    x = torch.randn(rows, cols, generator=g) * torch.randn(cols, generator=g).exp() + 0.3 * torch.randn(cols, generator=g)
    buf = torch.full((offset + max(rows, 1) * stride + 8,), 1e30, dtype=dtype, device="cuda")
    view = buf[offset:offset + rows * stride].view(rows, stride)[:, :cols] if rows else buf[:0].view(0, cols)
    view.copy_((x * scale).to(dtype))
    return view


def vector(n, dtype, seed, mean=0.0, std=1.0):
    return (mean + std * torch.randn(n, generator=gen(seed))).to(dtype).cuda()


# rows, cols, offset, extra: one element, a warp's edges, blocks cut short, odd strides and bases, each size of row
# that a kernel of its own takes, rows too long for all of them
SHAPES = [(1, 1, 0, 0), (3, 7, 0, 0), (2, 31, 1, 0), (5, 32, 0, 0), (5, 33, 0, 0), (7, 100, 0, 28), (197, 64, 0, 0),
          (64, 256, 0, 8), (33, 257, 3, 0), (197, 768, 0, 0), (9, 768, 0, 1), (21, 1000, 0, 0), (5, 1024, 0, 0),
          (11, 1031, 0, 0), (3, 2048, 0, 0), (6, 4096, 0, 64), (4, 5000, 0, 0), (2, 8192, 0, 0), (2, 20001, 0, 0),
          (2, 33000, 0, 0), (700, 48, 0, 0), (1500, 768, 0, 0)]


def forms_equal(kept, x, what):
    codes, exps = R.act8_forms(x.cpu())
    assert torch.equal(kept.exps.cpu(), exps), what
    assert torch.equal(kept.codes.cpu(), codes), what


# ---- 8-bit form --------------------------------------------------------------
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols,offset,extra", SHAPES)
def test_pack_is_the_format_to_the_bit(ops, rows, cols, offset, extra, dtype):
    x = matrix(rows, cols, dtype, rows + cols, offset, extra)
    kept = ops.act8_pack(x)
    forms_equal(kept, x, "pack")
    want = R.act8_values(kept.codes, kept.exps, cols)
    for out in TYPES:                      # 7 significant bits: exact in either type
        got = ops.act8_unpack(kept, dtype=out)
        assert got.dtype == out and torch.equal(got.cpu().double(), want)


@pytest.mark.parametrize("dtype", TYPES)
def test_pack_of_every_exponent(ops, dtype):
    """Blocks at every magnitude of fp32, subnormals and the largest numbers among them."""
    g = gen(5)
    x = torch.randn(278, 32, generator=g, dtype=torch.float64)
    x = (x / x.abs().amax(1, keepdim=True) * 1.9990234375).float()
    x = torch.ldexp(x.double(), torch.arange(-149, 129).double()[:, None] - 1).clamp(-3.4028234e38, 3.4028234e38)
    x = x.to(dtype).cuda()
    x[3] = 0
    x[4] = -0.0
    kept = ops.act8_pack(x)
    forms_equal(kept, x, "every exponent")
    want = R.act8_values(kept.codes, kept.exps, 32)
    fits = torch.isfinite(x).all(1).cpu()            # (fp32's largest number is an infinity in bf16)
    assert fits.sum() >= 277 and torch.isfinite(want[fits]).all() and torch.isnan(want[~fits]).all()
    assert torch.equal(ops.act8_unpack(kept, dtype=F32).cpu().double()[fits], want[fits])
    got = ops.act8_unpack(kept, dtype=BF16).cpu()[fits]
    assert torch.equal(got, want[fits].float().to(BF16)) and torch.isfinite(got.float()).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_pack_rounds_ties_to_even_and_clamps(ops, dtype):
    x = torch.zeros(4, 32)
    x[0, :5] = torch.tensor([127.0, 0.5, 1.5, -2.5, 126.5])
    x[1, :3] = torch.tensor([-127.5, 64.5, -3.5])
    x[2, :2] = torch.tensor([127.99, -127.99])       # (128 in bf16: the next exponent)
    x[3, :2] = torch.tensor([1.0, 2.0 ** -8])
    x = x.to(dtype).cuda()
    kept = ops.act8_pack(x)
    forms_equal(kept, x, "ties")
    assert kept.codes[0, :5].tolist() == [127, 0, 2, -2, 126]
    assert kept.codes[1, :3].tolist() == [-127, 64, -4]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_pack_of_what_8_bits_cannot_hold(ops, dtype, bad):
    x = matrix(4, 100, dtype, 1)
    x[1, 40] = bad
    x[2, 99] = bad
    kept = ops.act8_pack(x)
    forms_equal(kept, x, "non-finite")
    got = ops.act8_unpack(kept, dtype=dtype).cpu().float()
    nan = torch.zeros(4, 100, dtype=torch.bool)
    nan[1, 32:64] = nan[2, 96:] = True
    assert torch.equal(torch.isnan(got), nan)


def test_pack_error_is_half_a_scale(ops):
    x = matrix(50, 640, F32, 9)
    kept = ops.act8_pack(x)
    scale = R.two_to(kept.exps.cpu().long() - 127).repeat_interleave(32, 1)[:, :640]
    v, off = x.cpu().double(), (ops.act8_unpack(kept, dtype=F32).cpu().double() - x.cpu().double()).abs()
    clamped = v.abs() > 127.5 * scale
    assert (off <= torch.where(clamped, scale, 0.5 * scale)).all()
    top = v.abs().view(50, 20, 32).amax(2).repeat_interleave(32, 1)
    assert ((top >= 64 * scale) & (top < 128 * scale)).all()


# ---- layer norm --------------------------------------------------------------
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols,offset,extra", SHAPES)
def test_layer_norm(ops, rows, cols, offset, extra, dtype):
    x = matrix(rows, cols, dtype, 3 * rows + cols, offset, extra)
    for param, with_bias, checkpoint in ((F32, True, True), (BF16, True, False), (F32, False, True)):
        w, b = vector(cols, param, 1, 1.0, 0.2), vector(cols, param, 2) if with_bias else None
        y, mean, rstd, kept = ops.layer_norm(x, w, b, eps=1e-5, checkpoint=checkpoint)
        check_layer_norm(ops, x, w, b, 1e-5, y, mean, rstd, kept)
        assert (kept is not None) == checkpoint


def check_layer_norm(ops, x, w, b, eps, y, mean, rstd, kept):
    want = R.layer_norm(x, w, b, eps)
    bounds = R.layer_norm_bounds(x, w, b, eps, x.dtype)
    for got, ref, bound, what in zip((y, mean, rstd), want, bounds, ("y", "mean", "rstd")):
        R.assert_within(got, ref, bound, what)
    if kept is not None:
        check_kept(ops, kept, want[3], bounds[3], "xhat")


def check_kept(ops, kept, values, err, what):
    """The 8-bit form of computed values: within half a scale (one where 127 clamps) and their error; the
    scale that of the block's largest magnitude, or its neighbour where the error reaches across."""
    cols = values.shape[1]
    exps = kept.exps.cpu().long()
    scale = R.two_to(exps - 127)
    full = scale.repeat_interleave(32, 1)[:, :cols]
    got = R.act8_values(kept.codes, kept.exps, cols)
    limit = torch.where(values.abs() + err > 127.5 * full, full, 0.5 * full) + err
    assert ((got - values).abs() <= limit).all(), what
    pad = kept.codes.shape[1] - cols
    top = torch.nn.functional.pad(values.abs(), (0, pad)).view(exps.shape + (32,)).amax(2)
    slack = torch.nn.functional.pad(err, (0, pad)).view(exps.shape + (32,)).amax(2)
    small = exps == 0
    assert ((top + slack >= 64 * scale) | small).all() and (top - slack < 128 * scale).all(), what
    assert not kept.codes[:, cols:].any()


def test_layer_norm_of_rows_without_variance(ops):
    x = torch.full((3, 768), 5.0, device="cuda")
    x[1] = 0
    w, b = vector(768, F32, 1), vector(768, F32, 2)
    y, mean, rstd, kept = ops.layer_norm(x, w, b, eps=1e-5, checkpoint=True)
    assert torch.equal(y, b.expand(3, 768)) and mean.tolist() == [5.0, 0.0, 5.0]
    assert torch.allclose(rstd, torch.full((3,), 1e-5, device="cuda").rsqrt(), rtol=1e-6)
    assert not kept.codes.any()


def test_layer_norm_far_from_zero(ops):
    """A mean of 1000 standard deviations: E[x^2] - mean^2 would have no digits left."""
    x = (1000.0 + torch.randn(20, 1024, generator=gen(4))).cuda()
    w, b = torch.ones(1024, device="cuda"), None
    out = ops.layer_norm(x, w, b, checkpoint=True)
    check_layer_norm(ops, x, w, b, 1e-5, *out)


def test_layer_norm_keeps_a_bad_row_to_itself(ops):
    for cols in (768, 5000, 33000):
        x = matrix(4, cols, F32, 3)
        clean = ops.layer_norm(x, torch.ones(cols, device="cuda"), checkpoint=True)
        x[2, 7] = math.nan
        y, mean, rstd, kept = ops.layer_norm(x, torch.ones(cols, device="cuda"), checkpoint=True)
        keep = [0, 1, 3]
        assert torch.equal(y[keep], clean[0][keep]) and torch.isnan(y[2]).all() and torch.isnan(rstd[2])
        assert torch.equal(kept.codes[keep], clean[3].codes[keep]) and (kept.exps[2] == 255).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols,offset,extra", SHAPES)
def test_layer_norm_backward(ops, rows, cols, offset, extra, dtype):
    x = matrix(rows, cols, dtype, 3 * rows + cols, offset, extra)
    dy = matrix(rows, cols, dtype, rows + 5 * cols, (offset * 3) % 8, extra, scale=1e-3)
    _, mean, rstd, xhat = R.layer_norm(x, torch.ones(cols), None, 1e-5)
    mean, rstd = mean.float().cuda(), rstd.float().cuda()
    from_x = (x.cpu().double() - mean.cpu().double()[:, None]) * rstd.cpu().double()[:, None]
    kept = ops.act8_pack(xhat.float().cuda())
    from_8 = R.act8_values(kept.codes, kept.exps, cols)
    for param, grad in ((F32, F32), (BF16, BF16)):
        w = vector(cols, param, 1, 1.0, 0.2)
        for saved, m, ref, err in ((kept, None, from_8, 0.0), (x, mean, from_x, 3 * R.U)):
            got = ops.layer_norm_backward(dy, saved, rstd, w, mean=m, grad_dtype=grad)
            want = R.layer_norm_backward(dy, ref, rstd, w)
            bounds = R.layer_norm_backward_bounds(dy, ref, rstd, w, dtype, grad, err)
            for a, b, c, what in zip(got, want, bounds, ("dx", "dw", "db")):
                R.assert_within(a, b, c, what)
            assert got[0].dtype == dtype and got[1].dtype == grad


def test_layer_norm_backward_against_differences(ops):
    """The slope of <y, dy> along a direction, by central differences of the forward kernel in fp32.
    h = 2^-5: the curvature's part is h^2 / 6 times the third derivative (of the order of the slope itself
    for directions as long as the rows' deviation); rounding adds 2^-22 |y| |dy| / h summed at random."""
    rows, cols, h = 8, 768, 2.0 ** -5
    g = gen(3)
    x = torch.randn(rows, cols, generator=g).cuda()
    v = torch.randn(rows, cols, generator=g).cuda()
    dy = torch.randn(rows, cols, generator=g).cuda()
    w, b = vector(cols, F32, 1, 1.0, 0.2), vector(cols, F32, 2)
    y, mean, rstd, _ = ops.layer_norm(x, w, b)
    dx, dw, db = ops.layer_norm_backward(dy, x, rstd, w, mean=mean)

    def dot(p, q):
        return float((p.double() * q.double()).sum())

    def slope(step):
        return (dot(step(h), dy) - dot(step(-h), dy)) / (2 * h)
    scale = float(dy.double().norm() * v.double().norm())
    assert abs(slope(lambda s: ops.layer_norm(x + s * v, w, b)[0]) - dot(dx, v)) <= 2e-3 * scale
    vw = torch.randn(cols, generator=g).cuda()
    lin = float(dy.double().abs().sum()) * 2.0 ** -20 / h      # linear in w and b: rounding alone
    assert abs(slope(lambda s: ops.layer_norm(x, w + s * vw, b)[0]) - dot(dw, vw)) <= 4 * lin
    assert abs(slope(lambda s: ops.layer_norm(x, w, b + s * vw)[0]) - dot(db, vw)) <= 4 * lin


# ---- activation functions ------------------------------------------------------
KINDS = ["gelu", "gelu_tanh", "silu"]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols,offset,extra", [s for s in SHAPES if s[0] * s[1] < 40000])
def test_activation(ops, rows, cols, offset, extra, dtype, kind):
    u = matrix(rows, cols, dtype, rows + 7 * cols, offset, extra)
    a, kept_u, kept_a = ops.activation(u, kind, save_input=True, save_output=True)
    want = R.act(kind, u)
    R.assert_within(a, want, R.act_bound(want, u, dtype), "a")
    forms_equal(kept_u, u, "kept input")
    forms_equal(kept_a, a, "kept output is the rounded one")
    only, none_u, none_a = ops.activation(u, kind, save_input=False)
    assert torch.equal(only, a) and none_u is None and none_a is None
    da = matrix(rows, cols, dtype, rows + 11 * cols, (offset * 5) % 8, extra, scale=1e-2)
    for saved, base in ((kept_u, R.act8_values(kept_u.codes, kept_u.exps, cols)), (u, u.cpu().double())):
        du = ops.activation_backward(da, saved, kind)
        slope = R.act_slope(kind, base)
        want = da.cpu().double() * slope
        bound = da.cpu().double().abs() * (2.0 ** -20 * base.abs().clamp(min=1)) + R.rounding(want, dtype)
        R.assert_within(du, want, bound, "du")


@pytest.mark.parametrize("kind", KINDS)
def test_activation_over_the_whole_line(ops, kind):
    """Every scale of u from the smallest to the largest fp32 number, both signs: finite, and right."""
    e = torch.arange(-140, 128, dtype=torch.float64)
    u = torch.cat([torch.ldexp(torch.tensor(m, dtype=torch.float64), e) for m in (1.0, 1.37, 1.81)])
    u = torch.cat([u, -u, torch.linspace(-20, 20, 4001, dtype=torch.float64), torch.zeros(1, dtype=torch.float64)])
    u = u.float()[None].cuda()
    a, _, _ = ops.activation(u, kind, save_input=False)
    ref = R.act(kind, u)
    if kind == "gelu_tanh":          # (z^3 overflows in 64 bits too: its limits)
        ref = torch.where(u.cpu() > 100, u.cpu().double(), torch.where(u.cpu() < -100, torch.zeros_like(ref), ref))
    R.assert_within(a, ref, R.act_bound(ref, u, F32), "a")
    du = ops.activation_backward(torch.ones_like(u), u, kind)
    clipped = u.clamp(-100, 100)     # the slope is 0 or 1 beyond
    ref = R.act_slope(kind, clipped)
    R.assert_within(du, ref, 2.0 ** -20 * clipped.cpu().double().abs().clamp(min=1) + 1e-38, "du")


@pytest.mark.parametrize("kind", KINDS)
def test_activation_backward_against_differences(ops, kind):
    """h = 2^-6: h^2 / 6 |f'''| (at most 2) is 8e-5, rounding 2^-21 8 / h 2.5e-4 at |u| <= 8."""
    h = 2.0 ** -6
    u = torch.linspace(-8, 8, 2049)[None].cuda()
    up, _, _ = ops.activation(u + h, kind, save_input=False)
    down, _, _ = ops.activation(u - h, kind, save_input=False)
    du = ops.activation_backward(torch.ones_like(u), u, kind)
    assert float((du.double() - (up.double() - down.double()) / (2 * h)).abs().max()) <= 4e-4


# ---- weight gradient -------------------------------------------------------------
# rows, n_in, n_out, dy's offset and extra stride
GRADS = [(1, 1, 1, 0, 0), (1, 771, 1001, 0, 0), (2, 33, 65, 1, 0), (3, 64, 64, 0, 0), (17, 128, 136, 0, 0),
         (63, 100, 40, 0, 0), (64, 256, 128, 0, 0), (65, 257, 129, 0, 3), (127, 96, 200, 0, 8), (250, 2048, 1000, 0, 0),
         (300, 16, 16, 0, 0), (513, 320, 264, 0, 0), (1000, 768, 512, 0, 0), (2049, 300, 130, 0, 2), (4100, 512, 256, 0, 0)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,n_in,n_out,offset,extra", GRADS)
def test_weight_grad(ops, rows, n_in, n_out, offset, extra, dtype):
    dy = matrix(rows, n_out, dtype, rows + n_out, offset, extra, scale=1e-3)
    kept = ops.act8_pack(matrix(rows, n_in, F32, rows + n_in))
    x = R.act8_values(kept.codes, kept.exps, n_in)
    for grad, param, bias in ((F32, None, True), (BF16, F32, True), (F32, BF16, False)):
        affine = None
        h, parts = x, None
        if param is not None:
            affine = (vector(n_in, param, 1, 1.0, 0.2), vector(n_in, param, 2, 0.0, 0.2))
            h = x * affine[0].cpu().double() + affine[1].cpu().double()
            parts = (x,) + affine
        dw, db = ops.linear_weight_grad(dy, kept, affine=affine, bias=bias, dtype=grad)
        want = R.weight_grad(dy, h)
        bounds = R.weight_grad_bounds(dy, h, grad, parts)
        R.assert_within(dw, want[0], bounds[0], "dw")
        assert (db is not None) == bias
        if bias:
            R.assert_within(db, want[1], bounds[1], "db")


@pytest.mark.parametrize("dtype", TYPES)
def test_weight_grad_of_small_whole_numbers_is_exact(ops, dtype):
    """Every product and partial sum below 2^24: any order gives the same bits, an index off by one another."""
    rows, n_in, n_out = 777, 416, 392
    g = gen(8)
    x = torch.randint(-127, 128, (rows, n_in), generator=g).float()
    x[:, ::32] = 100.0                     # every block's largest: a scale of 1
    dy = torch.randint(-8, 9, (rows, n_out), generator=g).float()
    kept = ops.act8_pack(x.cuda())
    dw, db = ops.linear_weight_grad(dy.to(dtype).cuda(), kept)
    assert torch.equal(dw.cpu().double(), dy.double().t() @ x.double())
    assert torch.equal(db.cpu().double(), dy.double().sum(0))


def test_weight_grad_of_fp32_holds_all_24_bits(ops):
    """dy with 24 significant bits against a single row: the product is one rounding away."""
    g = gen(6)
    dy = torch.randn(1, 264, generator=g).cuda()
    x = torch.zeros(1, 160)
    x[0, ::32] = 64.0
    dw, db = ops.linear_weight_grad(dy, ops.act8_pack(x.cuda()))
    want = dy.cpu().double().t() @ x.double()
    R.assert_within(dw, want, 3 * R.U * want.abs(), "dw")
    R.assert_within(db, dy.cpu().double()[0], 3 * R.U * dy.cpu().double()[0].abs(), "db")


@pytest.mark.parametrize("dtype", TYPES)
def test_weight_grad_keeps_bad_values_to_their_columns(ops, dtype):
    rows, n_in, n_out = 200, 160, 136
    dy, x = matrix(rows, n_out, dtype, 1), matrix(rows, n_in, F32, 2)
    clean, _ = ops.linear_weight_grad(dy, ops.act8_pack(x))
    x[70, 40] = math.inf
    dw, db = ops.linear_weight_grad(dy, ops.act8_pack(x))
    assert torch.isnan(dw[:, 32:64]).all() and torch.equal(dw[:, :32], clean[:, :32])
    assert torch.equal(dw[:, 64:], clean[:, 64:]) and torch.isfinite(db).all()
    dy[5, 9] = math.nan
    dw, db = ops.linear_weight_grad(dy, ops.act8_pack(matrix(rows, n_in, F32, 2)))
    assert torch.isnan(dw[9]).all() and torch.isnan(db[9])
    keep = [i for i in range(n_out) if i != 9]
    assert torch.equal(dw[keep], clean[keep]) and torch.isfinite(db[keep]).all()


def test_weight_grad_of_large_fp32_gradients(ops):
    """fp32 values whose leading bf16 part would round up to infinity, and tiny ones whose rest is subnormal."""
    dy = torch.zeros(64, 128, device="cuda")
    dy[0, 0], dy[1, 1], dy[2, 2], dy[3, 3] = 3.4028234e38, -3.4028234e38, 1.17549435e-38, 3e-39
    x = torch.zeros(64, 64)
    x[:, 0] = x[:, 32] = 0.0
    for i in range(4):
        x[i, i] = 1.0
    dw, _ = ops.linear_weight_grad(dy, ops.act8_pack(x.cuda()))
    want = dy.cpu().double().t() @ x.double()
    # (what lies below the smallest subnormal of bf16, 2^-133, may be lost)
    R.assert_within(dw, want, 4 * R.U * want.abs() + 2.0 ** -132, "dw")


# ---- what holds for all of them ------------------------------------------------
def everything(ops, x, dy, w, b):
    """One call of each operator; every output."""
    y, mean, rstd, kept = ops.layer_norm(x, w, b, checkpoint=True)
    a, ku, ka = ops.activation(y, "gelu", save_output=True)
    dw, db = ops.linear_weight_grad(dy, ka)
    du = ops.activation_backward(dy, ku, "gelu")
    dw2, db2 = ops.linear_weight_grad(du, kept, affine=(w, b))
    dx, dg, dbeta = ops.layer_norm_backward(du, kept, rstd, w)
    dx2, _, _ = ops.layer_norm_backward(du, x, rstd, w, mean=mean)
    p = ops.act8_pack(dx)
    return [y, mean, rstd, kept.codes, kept.exps, a, ku.codes, ka.exps, dw, db, du, dw2, db2, dx, dg, dbeta, dx2,
            p.codes, ops.act8_unpack(p)]


def inputs(rows, cols, dtype):
    return (matrix(rows, cols, dtype, 1), matrix(rows, cols, dtype, 2, scale=1e-3), vector(cols, F32, 3, 1.0, 0.1),
            vector(cols, F32, 4))


def same(a, b):
    return all(torch.equal(p, q) for p, q in zip(a, b))


@pytest.mark.parametrize("dtype", TYPES)
def test_same_bits_from_run_to_run_and_stream_to_stream(ops, dtype):
    args = inputs(1234, 320, dtype)
    first = everything(ops, *args)
    for _ in range(3):
        assert same(everything(ops, *args), first)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = everything(ops, *args)
    torch.cuda.current_stream().wait_stream(side)
    assert same(other, first)


def test_capture_and_replay(ops):
    args = inputs(300, 320, BF16)
    want = [t.clone() for t in everything(ops, *args)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = everything(ops, *args)
    for _ in range(2):
        for t in out:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert same(out, want)
    args[0].mul_(0.5).add_(0.25)
    graph.replay()
    assert same(out, everything(ops, *args))


@pytest.mark.parametrize("dtype", TYPES)
def test_no_rows(ops, dtype):
    x = torch.empty(0, 96, dtype=dtype, device="cuda")
    w, b = torch.ones(96, device="cuda"), torch.zeros(96, device="cuda")
    y, mean, rstd, kept = ops.layer_norm(x, w, b, checkpoint=True)
    a, ku, ka = ops.activation(x, "silu", save_output=True)
    assert y.shape == a.shape == x.shape and mean.shape == (0,) and kept.rows == 0
    for saved in (kept, x):
        dx, dw, db = ops.layer_norm_backward(x, saved, rstd, w, mean=mean)
        assert dx.shape == x.shape and not dw.any() and not db.any()
    dw, db = ops.linear_weight_grad(x, ops.act8_pack(torch.empty(0, 40, dtype=dtype, device="cuda")), dtype=BF16)
    assert dw.shape == (96, 40) and not dw.any() and db.shape == (96,) and not db.any()
    assert ops.act8_unpack(ku).shape == (0, 96) and ops.activation_backward(x, ku, "silu").shape == x.shape


def test_leading_dimensions_fold(ops):
    x = torch.randn(6, 50, 96, device="cuda").to(BF16)
    w, b = torch.ones(96, device="cuda"), torch.zeros(96, device="cuda")
    y, mean, rstd, kept = ops.layer_norm(x, w, b, checkpoint=True)
    flat = ops.layer_norm(x.view(300, 96), w, b)
    assert y.shape == x.shape and mean.shape == (6, 50) and torch.equal(y.view(300, 96), flat[0])
    assert kept.shape == x.shape and ops.act8_unpack(kept).shape == x.shape
    dx, _, _ = ops.layer_norm_backward(y, kept, rstd, w)
    assert dx.shape == x.shape
    part = x[:, :, 32:64]                    # rows 96 apart, folding
    assert torch.equal(ops.activation(part, "gelu")[0], ops.activation(part.contiguous(), "gelu")[0])
    with pytest.raises(ValueError, match="fold"):
        ops.activation(x[:, :20], "gelu")
    with pytest.raises(ValueError, match="contiguous"):
        ops.activation(x.transpose(1, 2), "gelu")


@pytest.mark.parametrize("cols", [96, 4096, 40000])
def test_in_place(ops, cols):
    """y over x, dx over dy, a over u, through the C entry points."""
    from paper_2601_07876_b200 import binding as B
    lib = B.load_library()
    x, dy = matrix(40, cols, F32, 1), matrix(40, cols, F32, 2)
    w, b = vector(cols, F32, 3), vector(cols, F32, 4)
    y, mean, rstd, kept = ops.layer_norm(x, w, b, checkpoint=True)
    s = torch.cuda.current_stream().cuda_stream
    buf = x.clone()
    p = buf.data_ptr()
    assert lib.novak_layer_norm(p, cols, p, cols, 0, w.data_ptr(), b.data_ptr(), 0, 1e-5, None, None, None, None, 40,
                                cols, s) == 0
    assert torch.equal(buf, y)
    want = ops.layer_norm_backward(dy, kept, rstd, w)
    buf = dy.clone()
    p = buf.data_ptr()
    need = lib.novak_layer_norm_backward_bytes(40, cols)
    work = torch.empty(need, dtype=torch.uint8, device="cuda")
    dw, db = torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
    assert lib.novak_layer_norm_backward(p, cols, None, 0, 0, None, rstd.data_ptr(), kept.codes.data_ptr(),
                                         kept.exps.data_ptr(), w.data_ptr(), 0, p, cols, dw.data_ptr(), db.data_ptr(),
                                         0, work.data_ptr(), need, 40, cols, s) == 0
    assert torch.equal(buf, want[0]) and torch.equal(dw, want[1]) and torch.equal(db, want[2])
    a = ops.activation(x, "gelu")[0]
    buf = x.clone()
    p = buf.data_ptr()
    assert lib.novak_activation(p, cols, p, cols, 0, 0, None, None, None, None, 40, cols, s) == 0
    assert torch.equal(buf, a)


def test_nothing_outside_a_strided_output_is_written(ops):
    from paper_2601_07876_b200 import binding as B
    lib = B.load_library()
    for cols, extra, offset in ((100, 20, 0), (96, 32, 0), (33, 2, 1)):
        stride = cols + extra
        kept = ops.act8_pack(matrix(9, cols, F32, 1))
        buf = torch.full((offset + 9 * stride + 16,), 7.0, device="cuda")
        view = buf[offset:offset + 9 * stride].view(9, stride)
        assert lib.novak_act8_unpack(kept.codes.data_ptr(), kept.exps.data_ptr(), view.data_ptr(), stride, 0, 9, cols,
                                     torch.cuda.current_stream().cuda_stream) == 0
        assert torch.equal(view[:, :cols], ops.act8_unpack(kept, dtype=F32))
        assert (view[:, cols:] == 7).all() and (buf[:offset] == 7).all() and (buf[offset + 9 * stride:] == 7).all()


def test_more_than_2_to_the_31_elements(ops):
    """Offsets past 32 bits, elementwise and over rows (about 17 GB in all)."""
    rows, cols = 530_000, 4160
    assert rows * cols > 2 ** 31
    x = torch.empty(rows, cols, dtype=BF16, device="cuda")
    x.normal_()
    w, b = torch.ones(cols, device="cuda"), torch.zeros(cols, device="cuda")
    y, mean, rstd, kept = ops.layer_norm(x, w, b, checkpoint=True)
    tail = slice(rows - 3, rows)
    part = ops.layer_norm(x[tail], w, b, checkpoint=True)
    assert torch.equal(y[tail], part[0]) and torch.equal(kept.codes[tail], part[3].codes)
    del y
    packed = ops.act8_pack(x)
    assert torch.equal(packed.codes[tail], ops.act8_pack(x[tail]).codes)
    assert torch.equal(ops.act8_unpack(packed)[tail], ops.act8_unpack(ops.act8_pack(x[tail])))
    del packed
    dx, dw, db = ops.layer_norm_backward(x, kept, rstd, w)
    assert torch.equal(dx[tail], ops.layer_norm_backward(x[tail], part[3], part[2], w)[0])
    # dy = x is close to xhat here: dw near the rows' number, db the columns' sums (8 bits and bf16 apart)
    assert float((dw / rows - 1).abs().max()) < 0.02
    del dx
    dy = x[:, :16].contiguous()
    got, _ = ops.linear_weight_grad(dy, kept)
    want = torch.zeros(16, cols, dtype=torch.float64, device="cuda")
    for lo in range(0, rows, 53_000):
        hi = min(lo + 53_000, rows)
        k = ops.Act8(kept.codes[lo:hi], kept.exps[lo:hi], cols)
        want += dy[lo:hi].double().t() @ ops.act8_unpack(k, dtype=F32).double()
    # terms of about 1: 2^-24 of their number's root, with room for sums that round toward zero
    assert float((got.double() - want).abs().max()) < 1e-5 * rows
