"""A wait that runs out in one group of a call's matrices.  A program of its own, as orthogonalize_waits.py is."""
import ctypes
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2601_07876_b200 import binding as B  # noqa: E402
from paper_2601_07876_b200 import ops  # noqa: E402

if __name__ == "__main__":
    lib, n, side = B.load_library(), 20, 2900
    rows = (ctypes.c_int64 * n)(*[side] * n)
    one, need = lib.novak_orthogonalize_bytes(rows, rows, 1), lib.novak_orthogonalize_bytes(rows, rows, n)
    group = need // (one - 4096)                        # (records and counts aside)
    assert 5 < group < n - 5
    torch.manual_seed(0)
    g = [torch.randn(side, side, device="cuda") for _ in range(n)]
    want = ops.orthogonalize(g)
    out = [torch.zeros_like(w) for w in want]
    work = torch.full((need // 4,), float("nan"), device="cuda")
    # of 12 rows of 256 x 256 tiles: 78 of A and of B, 144 of X, five times
    tiles = 5 * (78 + 78 + 144)
    # (a group's last 144 times as many tiles are the last step's X, for which nobody waits)
    for withheld, bad in ((group * tiles + 100, range(group, n)), (100, range(group)), (group * tiles - 100, ())):
        before = ops.wait_failures()
        assert lib.novak_selftest_orthogonalize_wait(
            (ctypes.c_void_p * n)(*(t.data_ptr() for t in g)), rows, 0, (ctypes.c_void_p * n)(*(t.data_ptr() for t in out)), rows, rows, rows,
            n, (ctypes.c_double * 15)(*(x for c in ops.NEWTON_SCHULZ for x in c)), 5, 1e-7, work.data_ptr(), need, withheld, 20_000_000,
            torch.cuda.current_stream().cuda_stream) == B.NOVAK_OK
        assert (ops.wait_failures() > before) == (len(bad) > 0)
        for i in range(n):
            assert torch.isnan(out[i]).all() if i in bad else torch.equal(out[i], want[i]), (withheld, i)
        print("ok", withheld)
