"""Token embedding and its gradient, against the definition."""
import math

import pytest
import torch

import ops_reference as R
import stream_reference as S
from test_gpu_ops import TYPES, gen, matrix

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
# tokens, vocab, dim, offset, extra: single ones, odd widths, strides and bases, more rows of the table than tokens and
# fewer, wide rows
SHAPES = [(1, 1, 1, 0, 0), (1, 50, 8, 0, 0), (7, 3, 5, 0, 0), (33, 1000, 31, 1, 0), (100, 17, 64, 0, 8), (197, 1003, 771, 3, 0),
          (500, 70000, 16, 0, 0), (1025, 333, 768, 0, 0), (3, 40, 20001, 0, 0), (2, 9, 8192, 0, 0), (4100, 257, 129, 0, 3),
          (20000, 5, 32, 0, 0)]


@pytest.fixture(scope="module")
def ops():
    from paper_2601_07876_b200 import ops
    return ops


def words(tokens, vocab, seed, dtype=torch.int64, none=0.1):
    """Ids of falling frequency, some of which are none."""
    g = gen(seed)
    ids = (torch.exp(torch.rand(tokens, generator=g) * math.log(vocab + 1)).long() - 1).clamp(0, vocab - 1)
    ids = torch.randperm(vocab, generator=g)[ids]
    strange = torch.tensor([-1, vocab, -2 ** 31, 2 ** 31 - 1])
    lost = torch.rand(tokens, generator=g) < none
    ids = torch.where(lost, strange[torch.randint(4, (tokens,), generator=g)], ids)
    return ids.to(dtype).cuda()


@pytest.mark.parametrize("table_type", TYPES)
@pytest.mark.parametrize("tokens,vocab,dim,offset,extra", SHAPES)
def test_lookup_to_the_bit(ops, tokens, vocab, dim, offset, extra, table_type):
    table = matrix(vocab, dim, table_type, tokens + dim, offset, extra)
    for id_type, scale, dtype in ((torch.int64, 1.0, None), (torch.int32, math.sqrt(dim), BF16), (torch.int64, 0.1, F32)):
        ids = words(tokens, vocab, dim, id_type)
        out = ops.embedding(ids, table, scale=scale, dtype=dtype)
        assert out.dtype == (dtype or table_type)
        assert torch.equal(out.cpu(), S.embedding(ids, table, scale, out.dtype))


def check(ops, dout, ids, vocab, scale, dtype, base=None):
    out = base
    if base is not None:
        base = base.clone()
    got = ops.embedding_grad(dout, ids, vocab, scale=scale, dtype=dtype, out=out)
    assert got.dtype == dtype and (out is None or got.data_ptr() == out.data_ptr())
    want, size, count = S.embedding_grad(dout, ids, vocab, scale, base)
    R.assert_within(got, want, S.embedding_grad_bound(want, size, count, dtype, base), "dtable")
    named = count.cuda() > 0
    left = torch.zeros_like(got) if base is None else base
    assert torch.equal(got[~named], left[~named])           # to the bit
    return got


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens,vocab,dim,offset,extra", SHAPES)
def test_gradient(ops, tokens, vocab, dim, offset, extra, dtype):
    dout = matrix(tokens, dim, dtype, 3 * tokens + dim, offset, extra)
    for id_type, scale, grad, add in ((torch.int64, 1.0, F32, False), (torch.int32, math.sqrt(dim), BF16, False),
                                      (torch.int64, 0.5, F32, True), (torch.int32, 1.0, BF16, True)):
        ids = words(tokens, vocab, tokens + dim, id_type)
        base = matrix(vocab, dim, grad, 5, offset, extra) if add else None
        check(ops, dout, ids, vocab, scale, grad, base)


@pytest.mark.parametrize("kind", ["one id", "all others", "first and last", "none", "runs", "descending"])
@pytest.mark.parametrize("tokens", [1, 31, 64, 1000, 9000, 70001])
def test_gradient_of_any_order(ops, tokens, kind):
    """Whole numbers, whose sums are exact in fp32 in any order: to the bit."""
    vocab, dim = 5000, 24
    i = torch.arange(tokens)
    ids = {"one id": i * 0 + 4321, "all others": i * 2 % vocab, "first and last": (i % 2) * (vocab - 1), "none": i * 0 - 1,
           "runs": i // 37 % vocab, "descending": vocab - 1 - i % vocab}[kind].cuda()
    dout = torch.randint(-8, 9, (tokens, dim), generator=gen(1)).float().cuda()
    got = ops.embedding_grad(dout, ids, vocab)
    want, _, _ = S.embedding_grad(dout, ids, vocab, 1.0)
    assert torch.equal(got.cpu().double(), want)


@pytest.mark.parametrize("vocab", [2, 255, 256, 257, 65536, 65537, 300000, 20_000_000])
def test_gradient_of_any_vocabulary(ops, vocab):
    """Ids at every digit's edges."""
    near = [0, 1, 254, 255, 256, 257, 511, 512, 65535, 65536, 65537, 131071, vocab - 2, vocab - 1, vocab, vocab + 1]
    ids = torch.tensor(near)[torch.randint(len(near), (3000,), generator=gen(2))].cuda()
    dout = torch.randint(-8, 9, (3000, 4), generator=gen(3)).float().cuda()
    got = ops.embedding_grad(dout, ids, vocab)
    want, _, _ = S.embedding_grad(dout, ids, vocab, 1.0)
    assert torch.equal(got.cpu().double(), want)


def test_the_same_bits_from_run_to_run(ops):
    dout, ids = matrix(30000, 200, BF16, 1), words(30000, 900, 2)
    first = ops.embedding_grad(dout, ids, 900)
    for _ in range(3):
        assert torch.equal(ops.embedding_grad(dout, ids, 900), first)


def test_an_infinity_or_a_nan_stays_with_its_word(ops):
    ids = torch.tensor([3, 1, 3, 2, -1], device="cuda")
    dout = torch.ones(5, 40, device="cuda")
    dout[1, 7], dout[3, 9], dout[4] = math.inf, math.nan, math.nan
    got = ops.embedding_grad(dout, ids, 5, scale=2.0)
    assert torch.equal(got[3], torch.full((40,), 4.0, device="cuda")) and not got[0].any() and not got[4].any()
    assert float(got[1, 7]) == math.inf and math.isnan(float(got[2, 9])) and torch.isfinite(got).sum() == 5 * 40 - 2
    table = torch.ones(5, 40, device="cuda")
    table[0] = math.nan
    out = ops.embedding(ids, table)
    assert torch.isfinite(out).all() and not out[4].any()


def test_nothing(ops):
    none = torch.empty(0, dtype=torch.int64, device="cuda")
    table = torch.ones(5, 8, device="cuda")
    assert ops.embedding(none, table).shape == (0, 8)
    dout = torch.empty(0, 8, device="cuda")
    assert torch.equal(ops.embedding_grad(dout, none, 5), torch.zeros(5, 8, device="cuda"))
    assert torch.equal(ops.embedding_grad(dout, none, 5, out=table), torch.ones(5, 8, device="cuda"))
    assert ops.embedding_grad(torch.ones(3, 8, device="cuda"), none.new_zeros(3), 0).shape == (0, 8)
    assert not ops.embedding(none.new_zeros(3), table[:0]).any()


def test_shapes_strides_and_streams(ops):
    wide = matrix(64, 100, F32, 1)
    table = wide[::2, 10:90]                             # a matrix with rows of its own
    ids = words(24, 32, 3).view(2, 3, 4)
    assert torch.equal(ops.embedding(ids, table).cpu(), S.embedding(ids, table, 1.0, F32))
    turned = words(24, 32, 4).view(4, 6).t()             # ids that are not dense
    assert torch.equal(ops.embedding(turned, table).cpu(), S.embedding(turned, table, 1.0, F32))
    dout, out = matrix(24, 80, F32, 5).view(2, 3, 4, 80), wide[::2, 10:90]
    before = wide.clone()
    check(ops, dout, ids, 32, 1.0, F32, out)
    assert torch.equal(wide[1::2], before[1::2]) and torch.equal(wide[:, :10], before[:, :10]) and torch.equal(wide[:, 90:], before[:, 90:])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = ops.embedding_grad(dout, ids, 32)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, ops.embedding_grad(dout, ids, 32))


def test_captured_and_replayed_with_other_words(ops):
    ids, dout = words(2000, 700, 1), matrix(2000, 96, BF16, 2)
    ops.embedding_grad(dout, ids, 700)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = ops.embedding_grad(dout, ids, 700, scale=3.0)
    for seed in (5, 6, 7):
        ids.copy_(words(2000, 700, seed, none=0.0 if seed == 5 else 0.6))
        graph.replay()
        assert torch.equal(out, ops.embedding_grad(dout, ids, 700, scale=3.0))


def test_a_table_beyond_32_bits_of_elements(ops):
    """2^32 elements and more: rows behind the border, read and written."""
    vocab, dim = 70000, 65536
    table = torch.zeros(vocab, dim, dtype=BF16, device="cuda")
    table[vocab - 1] = 3.0
    table[32768] = 2.0                                   # the first one behind 2^31 elements
    ids = torch.tensor([vocab - 1, 0, 32768, vocab - 1], device="cuda")
    out = ops.embedding(ids, table, scale=0.5)
    assert [float(r.float().min()) for r in out] == [1.5, 0.0, 1.0, 1.5] and [float(r.float().max()) for r in out] == [1.5, 0.0, 1.0, 1.5]
    ops.embedding_grad(out, ids, vocab, dtype=BF16, out=table)
    assert float(table[vocab - 1].float().min()) == float(table[vocab - 1].float().max()) == 6.0
    assert float(table[32768].float().min()) == 3.0 and not table[vocab - 2].any() and not table[32769].any()


def test_refusals(ops):
    table, ids = torch.ones(5, 8, device="cuda"), torch.tensor([1, 2], device="cuda")
    dout = torch.ones(2, 8, device="cuda")
    for bad, error in ((lambda: ops.embedding(ids.float(), table), TypeError), (lambda: ops.embedding(ids, table.half()), TypeError),
                       (lambda: ops.embedding(ids, table[0]), ValueError), (lambda: ops.embedding(ids, table.t()), ValueError),
                       (lambda: ops.embedding(ids.cpu(), table), ValueError), (lambda: ops.embedding(ids, table.cpu()), ValueError),
                       (lambda: ops.embedding(ids, table, dtype=torch.half), TypeError),
                       (lambda: ops.embedding_grad(dout, ids[:1], 5), ValueError), (lambda: ops.embedding_grad(dout, ids, -1), ValueError),
                       (lambda: ops.embedding_grad(dout, ids, 5, out=table[:4]), ValueError),
                       (lambda: ops.embedding_grad(dout, ids, 5, out=table.cpu()), ValueError)):
        with pytest.raises(error):
            bad()
    from paper_2601_07876_b200 import binding as B
    with pytest.raises(B.NovakError, match="scale"):
        ops.embedding(ids, table, scale=math.inf)
