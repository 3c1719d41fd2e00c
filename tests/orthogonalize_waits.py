"""Lets waits inside the orthogonalising kernel run out and checks what is left behind.  A program of its own (run by
test_gpu_orthogonalize_waits.py): the count of such waits is the process's, and other tests ask for 0."""
import ctypes
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2601_07876_b200 import binding as B  # noqa: E402
from paper_2601_07876_b200 import ops  # noqa: E402

# one tile a product; tall and wide together; more tiles than pairs of SMs
SHAPES = [[(40, 70)], [(600, 200), (200, 600)], [(2304, 768), (768, 768), (1000, 2000), (2500, 2500)]]
COEFFICIENTS = ops.NEWTON_SCHULZ


def check(lib, shapes, dtype, withheld):
    """The end of one tile is never announced: every output is NaN to the last element and nothing beside it is
    written, the count goes up, and the next call, with the same workspace, is as ever."""
    torch.manual_seed(0)
    g = [torch.randn(r, c, device="cuda").to(dtype) for r, c in shapes]
    want = ops.orthogonalize(g)
    n = len(shapes)
    rows, cols = ((ctypes.c_int64 * n)(*(s[i] for s in shapes)) for i in range(2))
    need = lib.novak_orthogonalize_bytes(rows, cols, n)
    work = torch.full((need // 4,), float("nan"), device="cuda")
    out = [torch.full((r + 1, c + 3), 7.0, device="cuda", dtype=torch.bfloat16) for r, c in shapes]
    before, stream = ops.wait_failures(), torch.cuda.current_stream().cuda_stream

    def call(tile):
        return lib.novak_selftest_orthogonalize_wait(
            (ctypes.c_void_p * n)(*(t.data_ptr() for t in g)), cols, ops._TYPE[dtype],
            (ctypes.c_void_p * n)(*(t.data_ptr() for t in out)), (ctypes.c_int64 * n)(*(c + 3 for _, c in shapes)), rows, cols, n,
            (ctypes.c_double * (3 * len(COEFFICIENTS)))(*(x for c in COEFFICIENTS for x in c)), len(COEFFICIENTS), 1e-7,
            work.data_ptr(), need, tile, 20_000_000, stream)

    def around():
        return all((o[r:] == 7).all() and (o[:, c:] == 7).all() for o, (r, c) in zip(out, shapes))
    assert call(withheld) == B.NOVAK_OK
    assert ops.wait_failures() > before
    assert all(torch.isnan(o[:r, :c]).all() for o, (r, c) in zip(out, shapes)) and around()
    before = ops.wait_failures()
    assert call(-1) == B.NOVAK_OK
    assert all(torch.equal(o[:r, :c], w) for o, w, (r, c) in zip(out, want, shapes)) and around()
    assert ops.wait_failures() == before


if __name__ == "__main__":
    lib = B.load_library()
    for shapes in SHAPES:
        for dtype in (torch.float32, torch.bfloat16):
            for withheld in (0, 2):
                check(lib, shapes, dtype, withheld)
                print("ok", shapes, dtype, withheld)
