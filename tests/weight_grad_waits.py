"""Lets waits inside the weight gradient's kernel run out and checks what is left behind.  A program of its own (run by
test_gpu_weight_grad_waits.py): the count of such waits is the process's, and other tests ask for 0."""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2601_07876_b200 import binding as B  # noqa: E402
from paper_2601_07876_b200 import ops  # noqa: E402

# 160 tiles: two whole ones and a part of another for each of 74 pairs of SMs; 81: one and a part; one that is cut
# among pairs; 32 tiles on a pair each
SHAPES = [(200, 2560, 4096), (2100, 2304, 2304), (1024, 256, 256), (250, 2048, 1000)]


def check(lib, rows, n_in, n_out, affine, dtype):
    """The first sum of one pair of SMs is never announced.  Whole numbers: every element of dW is exact, or a NaN in a
    tile that the pair had to do with, its first one and all that follow it; db is exact; the count goes up; the next
    call is as ever."""
    g = torch.Generator(device="cuda").manual_seed(0)
    x = torch.randint(-127, 128, (rows, n_in), generator=g, device="cuda").float()
    x[:, ::32] = 100.0                          # every block's largest: a scale of 1
    dy = torch.randint(-4, 5, (rows, n_out), generator=g, device="cuda").float()
    kept, want, sums = ops.act8_pack(x), dy.double().t() @ x.double(), dy.double().sum(0)
    w = b = None
    if affine:
        w = torch.full((n_in,), 2.0, device="cuda")
        b = torch.arange(n_in, device="cuda").remainder(3).float() - 1
        want = want * w.double() + sums[:, None] * b.double()
    dy = dy.to(dtype)
    kind, stream = ops._TYPE[dtype], torch.cuda.current_stream().cuda_stream
    need = lib.novak_linear_weight_grad_bytes(dy.data_ptr(), n_out, kind, rows, n_out, n_in)
    work = torch.full((need // 4,), 3.0, device="cuda")
    dw, db = torch.full((n_out, n_in), 7.0, device="cuda"), torch.full((n_out,), 7.0, device="cuda")
    before = ops.wait_failures()

    def call(pair):
        return lib.novak_selftest_weight_grad_wait(
            dy.data_ptr(), n_out, kind, kept.codes_ptr, kept.exps_ptr, w.data_ptr() if affine else None,
            b.data_ptr() if affine else None, 0, dw.data_ptr(), db.data_ptr(), 0, work.data_ptr(), need, rows, n_out,
            n_in, pair, 20_000_000, stream)
    assert call(0) == B.NOVAK_OK
    assert ops.wait_failures() == before + 16            # the warps that store, of both SMs
    nan = torch.isnan(dw)
    assert torch.equal(torch.where(nan, want, dw.double()), want) and torch.equal(db.double(), sums)
    tiles = [nan[i:i + 256, k:k + 256] for i in range(0, n_out, 256) for k in range(0, n_in, 256)]
    assert all(t.all() or not t.any() for t in tiles)
    lost, whole = sum(bool(t.all()) for t in tiles), len(tiles) // 74
    # the whole ones and one or two of those left over; where all tiles are, its own
    assert max(whole + (whole > 0), 1) <= lost <= whole + 2
    assert call(-1) == B.NOVAK_EINVAL and call(74) == B.NOVAK_EINVAL
    again, db = ops.linear_weight_grad(dy, kept, affine=(w, b) if affine else None)
    assert torch.equal(again.double(), want) and torch.equal(db.double(), sums)
    assert ops.wait_failures() == before + 16


def check_refused(lib):
    """A few rows: the ordinary cores do the work and wait for nothing."""
    x = torch.zeros(8, 64, device="cuda")
    kept = ops.act8_pack(x)
    assert lib.novak_selftest_weight_grad_wait(x.data_ptr(), 64, 0, kept.codes_ptr, kept.exps_ptr, None, None, 0,
                                               x.data_ptr(), None, 0, None, 0, 8, 64, 64, 0, 0, None) == B.NOVAK_EINVAL
    assert "pair" in lib.novak_ops_error().decode()


if __name__ == "__main__":
    lib = B.load_library()
    check_refused(lib)
    for shape in SHAPES:
        for affine in (False, True):
            for dtype in (torch.float32, torch.bfloat16):
                check(lib, *shape, affine, dtype)
                print("ok", shape, affine, dtype)
