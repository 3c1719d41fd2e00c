"""Orthogonalised updates by Newton-Schulz products, against the definition in 64 bits."""
import math

import pytest
import torch

import ops_reference as R
import stream_reference as S
from test_gpu_ops import TYPES, gen

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
# single elements and lines, sides at the edges of a panel (64), a block (128) and a tile (256), tall and wide
SIZES = [(1, 1), (1, 7), (5, 1), (3, 2), (16, 16), (33, 70), (70, 33), (64, 64), (63, 65), (127, 129), (128, 128), (129, 64), (130, 500),
         (500, 130), (256, 256), (255, 257), (257, 300), (300, 1000), (777, 513), (385, 2049), (1024, 320)]


@pytest.fixture(scope="module")
def ops():
    from paper_2601_07876_b200 import ops
    return ops


def spectrum(rows, cols, kind, seed, dtype=F32):
    """Matrices whose singular values are spread in unlike ways."""
    g = gen(seed)
    x = torch.randn(rows, cols, generator=g, dtype=torch.float64)
    if kind == "low rank":
        r = max(1, min(rows, cols) // 16)
        x = 0.05 * x + (torch.randn(rows, r, generator=g, dtype=torch.float64) * torch.exp(-torch.arange(r) / 4.0)) @ torch.randn(r, cols, generator=g, dtype=torch.float64)
    elif kind == "rank one":
        x = torch.randn(rows, 1, generator=g, dtype=torch.float64) @ torch.randn(1, cols, generator=g, dtype=torch.float64)
    elif kind == "unlike features":
        x = x * torch.randn(rows, 1, generator=g, dtype=torch.float64).exp() * (1.5 * torch.randn(1, cols, generator=g, dtype=torch.float64)).exp()
    elif kind == "decay":
        u, _, v = torch.linalg.svd(x, full_matrices=False)
        x = (u * torch.logspace(0, -5, u.shape[1], dtype=torch.float64)) @ v
    elif kind == "orthogonal":
        u, _, v = torch.linalg.svd(x, full_matrices=False)
        x = u @ v
    return (1e-3 * x).to(dtype).cuda()


def far(got, want):
    got, want = got.detach().cpu().double(), want.cpu()
    assert torch.isfinite(got).all()
    return float((got - want).norm() / want.norm())


def check(got, g, coefficients=S.STEPS, eps=1e-7):
    want = S.orthogonalized(g, coefficients, eps)
    assert got.dtype == BF16 and got.shape == g.shape and got.is_contiguous()
    limit = S.orthogonal_tolerance(*g.shape, len(coefficients)) + R.U16
    assert far(got, want) <= limit


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", SIZES)
def test_sizes(ops, rows, cols, dtype):
    g = spectrum(rows, cols, "gauss", rows + cols, dtype)
    before = g.clone()
    check(ops.orthogonalize(g), g)
    assert torch.equal(g, before)


def unrounded(ops, g, **kw):
    """X before it is rounded to bf16: the step of a parameter of zeros."""
    theta, m = torch.zeros(g.shape, device="cuda"), torch.zeros(g.shape, device="cuda")
    ops.orthogonal_step([theta], [g], [m], [-1.0], momentum=0.0, nesterov=False, **kw)
    assert torch.equal(m, g.float())
    return theta


@pytest.mark.parametrize("kind", ["gauss", "low rank", "rank one", "unlike features", "decay", "orthogonal"])
@pytest.mark.parametrize("rows,cols", [(33, 70), (64, 64), (300, 200), (256, 1024), (1024, 256), (768, 768)])
def test_any_spectrum(ops, rows, cols, kind):
    g = spectrum(rows, cols, kind, rows, F32)
    x = unrounded(ops, g)
    assert far(x, S.orthogonalized(g)) <= S.orthogonal_tolerance(rows, cols)
    assert torch.equal(ops.orthogonalize(g), x.to(BF16))


def test_singular_values_come_close_to_one(ops):
    x = ops.orthogonalize(spectrum(200, 300, "gauss", 1)).double()
    s = torch.linalg.svdvals(x)
    assert 0.6 < float(s.min()) and float(s.max()) < 1.25


@pytest.mark.parametrize("coefficients", [((1.5, -0.5, 0.0),) * 12, ((1.875, -1.25, 0.375),) * 7, ((1.0, 0.0, 0.0),),
                                          ((3.4445, -4.7750, 2.0315), (2.0, -1.5, 0.5), (1.875, -1.25, 0.375))])
def test_other_polynomials(ops, coefficients):
    """|B| is below 2.81 for all of these too, and slopes are below 1.2 where singular values end."""
    for rows, cols in ((96, 130), (260, 140)):
        g = spectrum(rows, cols, "gauss", 3)
        check(ops.orthogonalize(g, coefficients=coefficients), g, coefficients)


def test_numbers_below_the_normal_ones(ops):
    g = spectrum(70, 90, "low rank", 5) * 1e3 * 2.0 ** -126     # (most of them lose bits on the way there)
    check(ops.orthogonalize(g, eps=0.0), g, eps=0.0)


@pytest.mark.parametrize("scale", [1e-30, 1e-12, 1e20, 1e35])
def test_any_magnitude(ops, scale):
    """Powers of two, with no element below the normal numbers: the same bits but for eps."""
    g = spectrum(70, 90, "low rank", 5) * 1e3
    power = 2.0 ** round(math.log2(scale))
    assert torch.equal(ops.orthogonalize(g * power, eps=0.0), ops.orthogonalize(g, eps=0.0))


def test_eps(ops):
    """Below eps the norm is not brought to 1: the result shrinks with G, 3.4445^5 times what it was at most."""
    g = spectrum(40, 50, "gauss", 5)
    g = g / g.norm() * 1e-9
    x = ops.orthogonalize(g, eps=1e-3)
    check(x, g, eps=1e-3)
    assert float(x.float().norm()) < 1e-6 * 3.4445 ** 5 * 1.01


def test_zeros_infinities_and_nans_stay_in_their_matrix(ops):
    ms = [spectrum(80, 100, "gauss", i) for i in range(5)]
    want = [ops.orthogonalize(m) for m in ms]
    ms[1].zero_()
    ms[2][3, 4], ms[4][79, 99] = math.inf, math.nan
    got = ops.orthogonalize(ms)
    assert not got[1].any() and torch.isnan(got[2]).all() and torch.isnan(got[4]).all()
    assert torch.equal(got[0], want[0]) and torch.equal(got[3], want[3])


@pytest.mark.parametrize("dtype", TYPES)
def test_many_at_once_are_each_as_if_alone(ops, dtype):
    sizes = [(64, 64), (300, 500), (1, 9), (500, 300), (64, 64), (129, 1), (777, 200), (256, 256)] * 3
    ms = [spectrum(r, c, "low rank", i, dtype) for i, (r, c) in enumerate(sizes)]
    got = ops.orthogonalize(ms)
    for m, x in zip(ms, got):
        check(x, m)
        assert torch.equal(ops.orthogonalize(m), x)


def test_more_matrices_than_go_with_one_launch(ops):
    ms = [spectrum(20 + i % 3, 30, "gauss", i) for i in range(600)]
    got = ops.orthogonalize(ms)
    for i in (0, 1, 255, 256, 257, 511, 512, 599):
        assert torch.equal(ops.orthogonalize(ms[i]), got[i])


# one CTA and eight, the longest that stay in shared memory and the first that do not, shares that are empty or a part
SMALL = [(64, 128), (128, 64), (64, 129), (17, 1000), (1000, 17), (64, 6000), (6000, 48), (1, 28000), (30000, 2), (65, 66), (97, 512), (512, 128),
         (128, 128), (128, 513), (600, 65), (8, 130), (50, 200)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", SMALL)
def test_small_ones(ops, rows, cols, dtype):
    g = spectrum(rows, cols, "low rank", rows + cols, dtype)
    check(ops.orthogonalize(g), g)


@pytest.mark.parametrize("rows,cols", [(60, 500), (500, 60), (100, 100), (33, 12), (300, 400)])
def test_small_steps_are_the_large_ones_step(ops, rows, cols):
    """theta by the step, m, and X, of one gradient in rows that are apart."""
    torch.manual_seed(3)
    g, theta, m = (torch.randn(rows, cols, device="cuda") for _ in range(3))
    want_m = 0.9 * m.double() + g.double()
    u = (g.double() + 0.9 * want_m).cpu()
    before = theta.double().cpu()
    ops.orthogonal_step([theta], [g], [m], [0.5], momentum=0.9, decay=0.75)
    R.assert_within(m, want_m.cpu(), 2 * R.U * (want_m.abs().cpu() + 1), "m")
    x = S.orthogonalized(u)
    off = float((theta.cpu().double() - (0.75 * before - 0.5 * x)).norm())
    assert off <= 0.5 * S.orthogonal_tolerance(rows, cols) * float(x.norm()) + 4 * R.U * float(before.norm())


def test_more_large_matrices_than_go_with_one_launch(ops):
    ms = [spectrum(130 + i % 3, 140, "gauss", i) for i in range(230)]
    got = ops.orthogonalize(ms)
    for i in (0, 7, 8, 199, 200, 229):
        assert torch.equal(ops.orthogonalize(ms[i]), got[i])


def test_batches_strides_and_nothing(ops):
    base = spectrum(6 * 40, 70, "gauss", 1).view(6, 40, 70)
    batch = base[1::2, 3:37, 5:60]                      # three matrices, rows and matrices apart, bases unaligned
    got = ops.orthogonalize(batch)
    assert got.shape == batch.shape and got.is_contiguous()
    for a, b in zip(batch, got):
        check(b, a)
        assert torch.equal(ops.orthogonalize(a.contiguous()), b)
    one = ops.orthogonalize(base.view(2, 3, 40, 70)).view(6, 40, 70)
    assert torch.equal(one[4], ops.orthogonalize(base[4]))
    none = torch.empty(3, 0, 5, device="cuda")
    assert ops.orthogonalize(none).shape == (3, 0, 5) and ops.orthogonalize([]) == []
    got = ops.orthogonalize([none, base[0], none[0]])
    assert torch.equal(got[1], one[0]) and got[2].shape == (0, 5)


def test_the_same_bits_from_run_to_run_and_on_other_streams(ops):
    ms = [spectrum(r, c, "gauss", r) for r, c in ((600, 700), (256, 2000), (900, 128))]
    first = ops.orthogonalize(ms)
    side = [torch.cuda.Stream() for _ in range(2)]
    for s in side:
        s.wait_stream(torch.cuda.current_stream())
    results = []
    for _ in range(3):
        for s in side:                                  # two at once
            with torch.cuda.stream(s):
                results.append(ops.orthogonalize(ms))
    for s in side:
        torch.cuda.current_stream().wait_stream(s)
    for r in results:
        assert all(torch.equal(a, b) for a, b in zip(first, r))
    assert ops.wait_failures() == 0


def test_captured_and_replayed_with_other_matrices(ops):
    ms = [spectrum(200, 300, "gauss", 1), spectrum(300, 100, "gauss", 2)]
    ops.orthogonalize(ms)
    graphs = []
    for _ in range(2):                                  # two graphs of one pool
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, pool=graphs[0][0].pool() if graphs else None):
            graphs.append((graph, ops.orthogonalize(ms)))
    for seed in (5, 6):
        for m in ms:
            m.copy_(spectrum(*m.shape, "low rank", seed))
        want = ops.orthogonalize(ms)
        for graph, out in graphs:
            graph.replay()
            assert all(torch.equal(a, b) for a, b in zip(out, want))


# ---- the step -------------------------------------------------------------------
@pytest.mark.parametrize("nesterov", [False, True])
@pytest.mark.parametrize("grad", TYPES)
def test_steps_of_momentum(ops, grad, nesterov):
    """Three steps.  m is fp32: a rounding a step.  theta takes step X, X within its tolerance."""
    sizes, mu, decay, lr = [(40, 90), (200, 130), (7, 3)], 0.9, 0.995, 0.02
    theta = [spectrum(r, c, "gauss", i) * 1e3 for i, (r, c) in enumerate(sizes)]
    m = [torch.zeros_like(t) for t in theta]
    ref = [(t.cpu().double(), t.cpu().double() * 0) for t in theta]
    for k in range(3):
        g = [spectrum(r, c, "low rank", 10 * k + i, grad) for i, (r, c) in enumerate(sizes)]
        ops.orthogonal_step(theta, g, m, [lr, 2 * lr, 0.5 * lr], momentum=mu, nesterov=nesterov, decay=decay)
        for i, (scale, (t, mo)) in enumerate(zip((1, 2, 0.5), ref)):
            mo = mu * mo + g[i].cpu().double()
            u = g[i].cpu().double() + mu * mo if nesterov else mo
            ref[i] = (decay * t - lr * scale * S.orthogonalized(u), mo)
    for i, (t, mo) in enumerate(ref):
        size = mo.abs() + 1e-3
        R.assert_within(m[i], mo, 8 * R.U * size, "m")
        scale = (1, 2, 0.5)[i] * lr
        off = (theta[i].cpu().double() - t).norm()
        want = 3 * scale * S.orthogonal_tolerance(*sizes[i]) * math.sqrt(min(sizes[i])) * 1.2 + 8 * R.U * float(t.norm())
        assert float(off) <= want


def test_refusals(ops):
    from paper_2601_07876_b200 import binding as B
    g = torch.randn(8, 9, device="cuda")
    for bad, error in ((lambda: ops.orthogonalize(g[0]), ValueError), (lambda: ops.orthogonalize(g.half()), TypeError),
                       (lambda: ops.orthogonalize(g.t()), ValueError), (lambda: ops.orthogonalize([g, g.bfloat16()]), ValueError),
                       (lambda: ops.orthogonalize(g.cpu()), ValueError), (lambda: ops.orthogonalize(g[:1].expand(4, 9)), ValueError),
                       (lambda: ops.orthogonalize([g, 3]), TypeError), (lambda: ops.orthogonalize(g, coefficients=((1.0, 2.0),)), ValueError),
                       (lambda: ops.orthogonal_step([g], [g], [], [1.0]), ValueError),
                       (lambda: ops.orthogonal_step([g], [g[:4]], [g], [1.0]), ValueError),
                       (lambda: ops.orthogonal_step([g.bfloat16()], [g], [g], [1.0]), TypeError)):
        with pytest.raises(error):
            bad()
    for bad in (lambda: ops.orthogonalize(g, coefficients=()), lambda: ops.orthogonalize(g, coefficients=((9.0, 0.0, 0.0),)),
                lambda: ops.orthogonalize(g, coefficients=((3.4445, -4.7750, 5.0),) * 5), lambda: ops.orthogonalize(g, eps=-1.0),
                lambda: ops.orthogonalize(g, coefficients=((math.nan, 0.0, 0.0),)),
                lambda: ops.orthogonalize(g, coefficients=((1.0, 0.0, 0.0),) * 33),
                lambda: ops.orthogonal_step([g], [g], [g.clone()], [1.0], momentum=1.0),
                lambda: ops.orthogonal_step([g], [g], [g.clone()], [math.inf])):
        with pytest.raises(B.NovakError):
            bad()
