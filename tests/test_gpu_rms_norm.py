"""Root-mean-square norm with the residual's addition and its backward pass, against the definition in 64 bits."""
import math

import pytest
import torch

import ops_reference as R
import stream_reference as S
from test_gpu_ops import SHAPES, TYPES, check_kept, matrix, vector

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def ops():
    from paper_2601_07876_b200 import ops
    return ops


def check(x, residual, w, eps, y, h, rstd, kept):
    want_h = S.add(x, residual)
    assert torch.equal(h.cpu(), want_h) and (h is x or residual is not None)
    want, bounds = S.rms_norm(want_h, w, eps), S.rms_norm_bounds(want_h, w, eps, x.dtype)
    R.assert_within(y, want[0], bounds[0], "y")
    R.assert_within(rstd, want[1], bounds[1], "rstd")
    if kept is not None:
        check_kept(None, kept, want[2], bounds[2], "xhat")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols,offset,extra", SHAPES)
def test_forward(ops, rows, cols, offset, extra, dtype):
    x = matrix(rows, cols, dtype, 3 * rows + cols, offset, extra)
    for param, with_residual, checkpoint in ((F32, True, True), (BF16, True, False), (F32, False, True), (BF16, False, False)):
        w = vector(cols, param, 1, 1.0, 0.2)
        residual = matrix(rows, cols, dtype, 5 * rows + cols, 2 * offset, extra) if with_residual else None
        before = [None if t is None else t.clone() for t in (x, residual)]
        y, h, rstd, kept = ops.rms_norm(x, w, residual=residual, eps=1e-6, checkpoint=checkpoint)
        assert (kept is not None) == checkpoint
        check(x, residual, w, 1e-6, y, h, rstd, kept)
        assert torch.equal(x, before[0]) and (residual is None or torch.equal(residual, before[1]))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols,offset,extra", SHAPES)
def test_backward(ops, rows, cols, offset, extra, dtype):
    dy = matrix(rows, cols, dtype, 11 * rows + cols, offset, extra)
    x = matrix(rows, cols, dtype, 13 * rows + cols, offset, 2 * extra)
    for param, saved, stream, grad in ((F32, "8 bits", True, F32), (BF16, "input", True, F32), (F32, "input", False, BF16),
                                       (F32, "8 bits", False, F32)):
        w = vector(cols, param, 3, 1.0, 0.2)
        dh = matrix(rows, cols, dtype, 17 * rows + cols, 3 * offset, extra) if stream else None
        _, _, rstd, kept = ops.rms_norm(x, w, checkpoint=True)
        if saved == "8 bits":
            xhat, err = R.act8_values(kept.codes, kept.exps, cols), 0.0
            dx, dw = ops.rms_norm_backward(dy, kept, rstd, w, dh=dh, grad_dtype=grad)
        else:
            xhat, err = x.cpu().double() * rstd.cpu().double()[:, None], R.U
            dx, dw = ops.rms_norm_backward(dy, x, rstd, w, dh=dh, grad_dtype=grad)
        want = S.rms_norm_backward(dy, xhat, rstd, w, dh)
        bounds = S.rms_norm_backward_bounds(dy, xhat, rstd, w, dtype, grad, dh, err)
        assert dx.dtype == dtype and dw.dtype == grad
        R.assert_within(dx, want[0], bounds[0], "dx")
        R.assert_within(dw, want[1], bounds[1], "dw")


def test_gradient_against_differences(ops):
    """Central differences of the definition, with steps of 1e-6, are good to 1e-8 here; the kernel's fp32 to
    1e-5 of each gradient's scale (bounds as above are far below that)."""
    x, r, w = matrix(3, 40, F32, 1), matrix(3, 40, F32, 2), vector(40, F32, 3, 1.0, 0.2)
    dy, dh = matrix(3, 40, F32, 4), matrix(3, 40, F32, 5)
    _, h, rstd, _ = ops.rms_norm(x, w, residual=r)
    dx, dw = ops.rms_norm_backward(dy, h, rstd, w, dh=dh)

    def value(hd, wd):
        y = S.rms_norm(hd, wd, 1e-6)[0]
        return float((y * dy.cpu().double()).sum() + (hd * dh.cpu().double()).sum())
    for got, which in ((dx, 0), (dw, 1)):
        at = [h.cpu().double(), w.cpu().double()]
        found = torch.zeros(got.numel(), dtype=torch.float64)
        for i in range(got.numel()):
            both = []
            for d in (1e-6, -1e-6):
                moved = [t.clone() for t in at]
                moved[which].view(-1)[i] += d
                both.append(value(*moved))
            found[i] = (both[0] - both[1]) / 2e-6
        got = got.cpu().double().view(-1)
        assert float((got - found).norm() / found.norm()) < 1e-5


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", [40, 768, 9000])
def test_rows_of_zeros_infinities_and_nans(ops, cols, dtype):
    """A row of zeros: xhat and y are zeros, rstd is 1 / sqrt(eps).  An infinity or a NaN stays in its row."""
    x, r, w = matrix(6, cols, dtype, 1), matrix(6, cols, dtype, 2), vector(cols, F32, 3, 1.0, 0.2)
    x[0] = 0
    r[0] = 0
    x[2, 5], x[4, cols - 1] = math.inf, math.nan
    y, h, rstd, kept = ops.rms_norm(x, w, residual=r, eps=1e-6, checkpoint=True)
    assert torch.equal(y[0], torch.zeros_like(y[0])) and abs(float(rstd[0]) * 1e-3 - 1) < 1e-6
    assert torch.equal(torch.isfinite(h).all(1).cpu(), torch.tensor([True, True, False, True, False, True]))
    fine = [0, 1, 3, 5]
    check(x[fine], r[fine], w, 1e-6, y[fine], h[fine], rstd[fine], None)
    assert float(rstd[2]) == 0.0 and math.isnan(float(rstd[4]))
    assert torch.isnan(y[2, 5]) and torch.isnan(y[4]).all()
    back = ops.act8_unpack(kept).float()
    assert torch.isfinite(back[fine]).all() and torch.isnan(back[4]).all() and torch.isnan(back[2, :32]).all()
    dx, _ = ops.rms_norm_backward(matrix(6, cols, dtype, 4), kept, rstd, w)
    assert torch.isfinite(dx[fine]).all()


def test_no_rows(ops):
    w = vector(64, F32, 1)
    x = torch.empty(0, 64, device="cuda")
    y, h, rstd, kept = ops.rms_norm(x, w, residual=x, checkpoint=True)
    assert y.shape == h.shape == (0, 64) and rstd.shape == (0,) and kept.rows == 0
    dx, dw = ops.rms_norm_backward(x, kept, rstd, w, dh=x)
    assert dx.shape == (0, 64) and torch.equal(dw, torch.zeros(64, device="cuda"))


def test_more_dimensions_and_broadcast_rows(ops):
    x = matrix(24, 96, BF16, 1).view(2, 3, 4, 96)
    w = vector(96, F32, 2, 1.0, 0.1)
    y, h, rstd, kept = ops.rms_norm(x, w, residual=x, checkpoint=True)
    assert y.shape == x.shape and rstd.shape == (2, 3, 4) and kept.shape == x.shape
    flat = ops.rms_norm(x.view(24, 96), w, residual=x.view(24, 96))[0]
    assert torch.equal(y.view(24, 96), flat)
    with pytest.raises(ValueError, match="overlap"):
        ops.rms_norm(x[0, 0, :1].expand(4, 96), w)


def test_in_place_through_the_c_entry_point(ops):
    """h over the residual and y over x; dx over dh."""
    from paper_2601_07876_b200 import binding as B
    lib, stream = B.load_library(), torch.cuda.current_stream().cuda_stream
    for dtype, cols in ((F32, 771), (BF16, 768), (BF16, 9001)):
        x, r, w = matrix(50, cols, dtype, 1), matrix(50, cols, dtype, 2), vector(cols, F32, 3, 1.0, 0.2)
        y, h, rstd, _ = ops.rms_norm(x, w, residual=r)
        kind = ops._TYPE[dtype]
        again = torch.empty_like(rstd)
        assert lib.novak_rms_norm(x.data_ptr(), cols, r.data_ptr(), cols, r.data_ptr(), cols, x.data_ptr(), cols, kind,
                                  w.data_ptr(), 0, 1e-6, again.data_ptr(), None, None, 50, cols, stream) == B.NOVAK_OK
        assert torch.equal(x, y) and torch.equal(r, h) and torch.equal(again, rstd)
        dy, dh = matrix(50, cols, dtype, 4), matrix(50, cols, dtype, 5)
        dx, dw = ops.rms_norm_backward(dy, h, rstd, w, dh=dh)
        need = lib.novak_rms_norm_backward_bytes(50, cols)
        work, dw2 = torch.empty(need, dtype=torch.uint8, device="cuda"), torch.empty(cols, device="cuda")
        assert lib.novak_rms_norm_backward(dy.data_ptr(), cols, dh.data_ptr(), cols, h.data_ptr(), cols, kind, rstd.data_ptr(),
                                           None, None, w.data_ptr(), 0, dh.data_ptr(), cols, dw2.data_ptr(), 0, work.data_ptr(),
                                           need, 50, cols, stream) == B.NOVAK_OK
        assert torch.equal(dh, dx) and torch.equal(dw, dw2)


def test_captured_and_replayed_with_other_inputs(ops):
    x, r, dy = (matrix(300, 512, BF16, i) for i in range(3))
    w = vector(512, F32, 3, 1.0, 0.2)

    def step():
        y, h, rstd, kept = ops.rms_norm(x, w, residual=r, checkpoint=True)
        return (y, h, rstd, *ops.rms_norm_backward(dy, kept, rstd, w, dh=y))
    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for seed in (7, 8):
        for t in (x, r, dy):
            t.copy_(matrix(300, 512, BF16, seed))
        graph.replay()
        for a, b in zip(out, step()):
            assert torch.equal(a, b)


def test_other_streams(ops):
    x, r, w = matrix(4000, 512, BF16, 1), matrix(4000, 512, BF16, 2), vector(512, F32, 3, 1.0, 0.2)
    want = ops.rms_norm(x, w, residual=r)[0]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = ops.rms_norm(x, w, residual=r)[0]
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want)


def test_refusals(ops):
    x, w = matrix(4, 64, F32, 1), vector(64, F32, 2)
    for bad, error in ((lambda: ops.rms_norm(x, w, residual=x[:3]), ValueError), (lambda: ops.rms_norm(x, w, residual=x.bfloat16()), TypeError),
                       (lambda: ops.rms_norm(x, w[:63]), ValueError), (lambda: ops.rms_norm(x.half(), w), TypeError),
                       (lambda: ops.rms_norm_backward(x, x, torch.ones(3, device="cuda"), w), ValueError),
                       (lambda: ops.rms_norm_backward(x, x[:2], torch.ones(4, device="cuda"), w), ValueError),
                       (lambda: ops.rms_norm_backward(x, x, torch.ones(4, device="cuda"), w, dh=x.bfloat16()), TypeError),
                       (lambda: ops.rms_norm_backward(x, x, torch.ones(4, device="cuda"), w, grad_dtype=torch.half), TypeError),
                       (lambda: ops.rms_norm(x[:, ::2], w[::2].contiguous()), ValueError)):
        with pytest.raises(error):
            bad()
    from paper_2601_07876_b200 import binding as B
    with pytest.raises(B.NovakError, match="eps"):
        ops.rms_norm(x, w, eps=-1.0)
