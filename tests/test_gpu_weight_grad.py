"""The weight gradient's ways of cutting its work up, on numbers whose every product and partial sum is a whole
number below 2^24: any order of adding gives the same bits, and a row, column or step that is lost, doubled or
read before its time gives others."""
import pytest
import torch

F32, BF16 = torch.float32, torch.bfloat16
pytestmark = pytest.mark.gpu

# (rows, n_in, n_out): 74 pairs of SMs, tiles of 256 x 256, steps of 64 rows
SHAPES = [
    (1, 40, 8), (16, 72, 65), (17, 72, 65), (33, 257, 130), (192, 256, 256),    # little: ordinary cores
    (193, 256, 256), (193, 8, 8), (64, 2048, 1024), (250, 2048, 1000),          # whole tiles, fewer than pairs
    (1024, 256, 256), (4099, 768, 264), (1500, 513, 255), (700, 96, 1000),      # all of them cut
    (200, 2304, 2304), (129, 4096, 4096),                                       # whole tiles, and tiles left over whole
    (2100, 2304, 2304), (1200, 1600, 2560),                                     # whole tiles, and tiles left over cut
]


@pytest.fixture(scope="module")
def ops():
    from paper_2601_07876_b200 import ops
    return ops


def whole(rows, n_in, n_out, seed=0):
    """dy and x of whole numbers, each block's largest |x| the same (a scale of 1)."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randint(-127, 128, (rows, n_in), generator=g, device="cuda").float()
    x[:, ::32] = 100.0
    dy = torch.randint(-4, 5, (rows, n_out), generator=g, device="cuda").float()
    return dy, x


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,n_in,n_out", SHAPES)
def test_every_cut_is_exact(ops, rows, n_in, n_out, dtype):
    dy, x = whole(rows, n_in, n_out)
    assert rows * 127 * 4 * 3 < 2 ** 24
    kept = ops.act8_pack(x)
    want, sums = dy.double().t() @ x.double(), dy.double().sum(0)
    dw, db = ops.linear_weight_grad(dy.to(dtype), kept)
    assert torch.equal(dw.double(), want) and torch.equal(db.double(), sums)
    dw, db = ops.linear_weight_grad(dy.to(dtype), kept, bias=False)
    assert torch.equal(dw.double(), want) and db is None
    w = torch.arange(n_in, device="cuda").remainder(2).float() + 1          # 1 or 2
    b = torch.arange(n_in, device="cuda").remainder(3).float() - 1          # -1, 0 or 1
    for bias in (True, False):
        dw, db = ops.linear_weight_grad(dy.to(dtype), kept, affine=(w, b), bias=bias)
        assert torch.equal(dw.double(), want * w.double() + sums[:, None] * b.double())
        assert db is None if not bias else torch.equal(db.double(), sums)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("offset,extra", [(1, 0), (0, 3), (8, 8)])
def test_every_cut_is_exact_from_unaligned_rows(ops, offset, extra, dtype):
    rows, n_in, n_out = 1024, 300, 517
    dy, x = whole(rows, n_in, n_out, 1)
    room = torch.full((offset + rows * (n_out + extra),), float("nan"), dtype=dtype, device="cuda")
    view = room[offset:].view(rows, n_out + extra)[:, :n_out]
    view.copy_(dy)
    dw, db = ops.linear_weight_grad(view, ops.act8_pack(x))
    assert torch.equal(dw.double(), dy.double().t() @ x.double()) and torch.equal(db.double(), dy.double().sum(0))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_long_sums_are_exact_time_after_time(ops, dtype):
    """Hundreds of steps per pair of SMs, rings of buffers gone round many times."""
    rows, n_in, n_out = 18944, 2048, 2304
    dy, x = whole(rows, n_in, n_out, 2)
    kept, want = ops.act8_pack(x), dy.double().t() @ x.double()
    dy = dy.to(dtype)
    for _ in range(4):
        dw, _ = ops.linear_weight_grad(dy, kept)
        assert torch.equal(dw.double(), want)
    assert ops.wait_failures() == 0


def test_large_and_tiny_fp32_gradients_in_the_tensor_cores(ops):
    """Values whose leading bf16 part would round up to infinity, and ones whose rest is subnormal there."""
    rows = 256
    dy = torch.zeros(rows, 256, device="cuda")
    dy[0, 0], dy[1, 1], dy[2, 2], dy[3, 3] = 3.4028234e38, -3.4028234e38, 1.17549435e-38, 3e-39
    x = torch.zeros(rows, 256, device="cuda")
    for i in range(4):
        x[i, i] = 1.0
    dw, _ = ops.linear_weight_grad(dy, ops.act8_pack(x))
    want = dy.double().t() @ x.double()
    # one rounding of the sum of three parts, each exact down to the smallest subnormal of bf16, 2^-133
    assert ((dw.double() - want).abs() <= 2.0 ** -22 * want.abs() + 2.0 ** -132).all()


def test_bad_values_keep_to_their_columns_in_the_tensor_cores(ops):
    rows, n_in, n_out = 640, 320, 264
    dy, x = whole(rows, n_in, n_out, 3)
    clean, sums = ops.linear_weight_grad(dy, ops.act8_pack(x))
    x[70, 40] = float("inf")
    dw, db = ops.linear_weight_grad(dy, ops.act8_pack(x))
    assert torch.isnan(dw[:, 32:64]).all() and torch.equal(db, sums)
    keep = [i for i in range(n_in) if not 32 <= i < 64]
    assert torch.equal(dw[:, keep], clean[:, keep])


@pytest.mark.parametrize("rows,n_in,n_out", [(3, 8, 1 << 22), (200, 8, 1 << 22), (3, 1 << 22, 8), (200, 1 << 22, 8)])
def test_the_widest_matrices(ops, rows, n_in, n_out):
    dy, x = whole(rows, n_in, n_out, 4)
    dw, db = ops.linear_weight_grad(dy.to(BF16), ops.act8_pack(x))
    assert torch.equal(dw, dy.t() @ x) and torch.equal(db, dy.sum(0))        # (whole numbers: exact in fp32 too)
