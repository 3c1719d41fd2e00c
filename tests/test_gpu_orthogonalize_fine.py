"""Orthogonalised updates whose products have operands of two parts (`fine`), of matrices that go to the tensor cores."""
import ctypes
import math

import pytest
import torch

import stream_reference as S
from test_gpu_ops import TYPES
from test_gpu_orthogonalize import far, spectrum
from test_gpu_orthogonalize_bounds import kinds

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def ops():
    from paper_2601_07876_b200 import ops
    return ops


def tolerance(rows, cols, one_direction):
    """As for small matrices (test_gpu_orthogonalize_bounds), and what sums over up to max(rows, cols) terms add: an
    addition of fp32 for each 16 of them, 2^-24, in the mean square."""
    u = 2.0 ** -23 * (1 + math.sqrt(max(rows, cols) / 16) / 2)
    return (485 + 5.6 * 198) * u if one_direction else 3 * 5 * 11 * u


def unrounded(ops, g):
    theta, m = ([torch.zeros(x.shape, device="cuda") for x in g] for _ in range(2))
    ops.orthogonal_step(theta, g, m, [-1.0] * len(g), momentum=0.0, nesterov=False, fine=True)
    return theta


@pytest.mark.parametrize("rows,cols,count", [(65, 600, 8), (129, 129, 20), (200, 300, 10), (300, 200, 10), (255, 257, 5), (257, 255, 5), (700, 257, 3),
                                             (768, 768, 2), (385, 2049, 2), (2049, 385, 2), (1001, 1500, 1)])
def test_as_good_as_fp32(ops, rows, cols, count):
    for kind, g in kinds(rows, cols, count):
        for a, x in zip(g, unrounded(ops, g)):
            assert far(x, S.orthogonalized(a)) <= tolerance(rows, cols, kind in ("rank one", "low rank")), kind


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", [(1, 1), (33, 70), (64, 64), (128, 500), (130, 500), (500, 130), (257, 300), (777, 513)])
def test_rounded_to_bf16(ops, rows, cols, dtype):
    """Half a step, 2^-8 of an element at most, on top of that."""
    g = spectrum(rows, cols, "gauss", rows + cols, dtype)
    before = g.clone()
    x = ops.orthogonalize(g, fine=True)
    assert x.dtype == BF16 and torch.equal(g, before)
    assert far(x, S.orthogonalized(g)) <= tolerance(rows, cols, False) + 2.0 ** -8
    if min(rows, cols) <= 64 or max(rows, cols) <= 512 and min(rows, cols) <= 128:
        assert torch.equal(x, ops.orthogonalize(g))     # (small ones are so anyway)


def test_other_polynomials(ops):
    """Slopes of up to 1.875 a step on the way up: below 3.4445."""
    for c in (((1.5, -0.5, 0.0),) * 12, ((1.0, 0.0, 0.0),), ((3.4445, -4.7750, 2.0315), (1.875, -1.25, 0.375))):
        for shape in ((260, 140), (140, 260)):
            g = spectrum(*shape, "gauss", 3)
            assert far(ops.orthogonalize(g, coefficients=c, fine=True), S.orthogonalized(g, c)) <= 4 * tolerance(*shape, False) + 2.0 ** -8


def test_many_at_once_are_each_as_if_alone_and_from_run_to_run(ops):
    sizes = [(64, 64), (300, 500), (500, 300), (129, 129), (777, 200), (256, 256), (2000, 1100)] * 3
    ms = [spectrum(r, c, "low rank", i) for i, (r, c) in enumerate(sizes)]
    got = ops.orthogonalize(ms, fine=True)
    for m, x in zip(ms, got):
        assert torch.equal(ops.orthogonalize(m, fine=True), x)
    side = [torch.cuda.Stream() for _ in range(2)]
    for s in side:
        s.wait_stream(torch.cuda.current_stream())
    results = []
    for fine, s in ((True, side[0]), (False, side[1]), (True, side[1])):        # two at once, of both kinds
        with torch.cuda.stream(s):
            results.append((fine, ops.orthogonalize(ms, fine=fine)))
    for s in side:
        torch.cuda.current_stream().wait_stream(s)
    plain = ops.orthogonalize(ms)
    for fine, r in results:
        assert all(torch.equal(a, b) for a, b in zip(got if fine else plain, r))
    assert ops.wait_failures() == 0


def test_magnitudes_zeros_infinities_and_nans(ops):
    g = spectrum(300, 140, "low rank", 5) * 1e3
    want = ops.orthogonalize(g, eps=0.0, fine=True)
    for power in (-100, -40, 66, 116):
        assert torch.equal(ops.orthogonalize(g * 2.0 ** power, eps=0.0, fine=True), want)
    ms = [spectrum(180, 200, "gauss", i) for i in range(5)]
    want = [ops.orthogonalize(m, fine=True) for m in ms]
    ms[1].zero_()
    ms[2][3, 4], ms[4][179, 199] = math.inf, math.nan
    got = ops.orthogonalize(ms, fine=True)
    assert not got[1].any() and torch.isnan(got[2]).all() and torch.isnan(got[4]).all()
    assert torch.equal(got[0], want[0]) and torch.equal(got[3], want[3])


def test_strides_and_batches(ops):
    base = spectrum(6 * 140, 270, "gauss", 1).view(6, 140, 270)
    batch = base[1::2, 3:137, 5:260]
    got = ops.orthogonalize(batch, fine=True)
    for a, b in zip(batch, got):
        assert torch.equal(ops.orthogonalize(a.contiguous(), fine=True), b)


def test_groups(ops):
    """More than 1 GiB of workspace at once."""
    torch.manual_seed(0)
    g = [torch.randn(2900, 2900, device="cuda", dtype=BF16) for _ in range(10)]
    alone = [ops.orthogonalize(x, fine=True) for x in g]
    assert all(torch.equal(a, b) for a, b in zip(alone, ops.orthogonalize(g, fine=True)))


def test_captured_and_replayed_with_other_matrices(ops):
    ms = [spectrum(200, 300, "gauss", 1), spectrum(300, 140, "gauss", 2)]
    ops.orthogonalize(ms, fine=True)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = ops.orthogonalize(ms, fine=True)
    for seed in (5, 6):
        for m in ms:
            m.copy_(spectrum(*m.shape, "low rank", seed))
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(out, ops.orthogonalize(ms, fine=True)))


@pytest.mark.parametrize("byte", [0, 0xff, 0x7f])
def test_workspaces_full_of_anything(ops, byte):
    from paper_2601_07876_b200 import binding as B
    lib, shapes = B.load_library(), [(70, 33), (130, 300), (1, 5), (513, 257)]
    torch.manual_seed(1)
    g = [torch.randn(*s, device="cuda") for s in shapes]
    want, n = ops.orthogonalize(g, fine=True), len(shapes)
    rows, cols = ((ctypes.c_int64 * n)(*(s[i] for s in shapes)) for i in range(2))
    need = lib.novak_orthogonalize_fine_bytes(rows, cols, n)
    assert need > lib.novak_orthogonalize_bytes(rows, cols, n)
    base = torch.full((need + 512,), byte, dtype=torch.uint8, device="cuda")
    out = [torch.empty_like(w) for w in want]
    args = [(ctypes.c_void_p * n)(*(t.data_ptr() for t in g)), cols, 0, (ctypes.c_void_p * n)(*(t.data_ptr() for t in out)), cols, rows, cols, n,
            (ctypes.c_double * 15)(*(x for c in ops.NEWTON_SCHULZ for x in c)), 5, 1e-7, base.data_ptr() + 256]
    stream = torch.cuda.current_stream().cuda_stream
    assert lib.novak_orthogonalize_fine(*args, need - 1, stream) == B.NOVAK_EINVAL
    assert lib.novak_orthogonalize_fine(*args, need, stream) == B.NOVAK_OK
    assert all(torch.equal(a, b) for a, b in zip(out, want)) and (base[:256] == byte).all() and (base[-256:] == byte).all()


def test_muon(ops):
    from paper_2601_07876_b200.optim import Muon
    torch.manual_seed(2)
    p = torch.nn.Parameter(torch.randn(300, 200, device="cuda"))
    p.grad = torch.randn(300, 200, device="cuda")
    before = p.detach().cpu().double()
    opt = Muon([p], lr=0.5, fine=True)
    opt.step()
    x = S.orthogonalized(p.grad)
    off = float((p.detach().cpu().double() - (before - 0.5 * math.sqrt(1.5) * x)).norm())
    assert off <= 0.7 * tolerance(300, 200, False) * float(x.norm()) + 4 * 2.0 ** -24 * float(before.norm())
    saved = opt.state_dict()
    again = Muon([p], lr=0.5)
    again.load_state_dict(saved)
    assert again.param_groups[0]["fine"] is True
