"""The embedding's gradient of more tokens than one CTA keeps in shared memory, and of more than its map has bits for."""
import pytest
import torch

import stream_reference as S
from test_gpu_embedding import words
from test_gpu_ops import gen

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ops():
    from paper_2601_07876_b200 import ops
    return ops


def ids_of(kind, tokens, vocab):
    i = torch.arange(tokens)
    return {"uniform": torch.randint(vocab, (tokens,), generator=gen(tokens)), "one id": i * 0 + vocab // 3,
            "two by turns": torch.where(i % 2 == 0, vocab - 1, 0), "runs": i // 61 % vocab, "descending": vocab - 1 - i % vocab,
            "few at the end": torch.where(i < tokens - 40, -1, i % min(vocab, 7)), "words": words(tokens, vocab, tokens).cpu()}[kind]


@pytest.mark.parametrize("kind", ["uniform", "one id", "two by turns", "runs", "descending", "few at the end", "words"])
@pytest.mark.parametrize("tokens,vocab", [(4097, 3), (65536, 300), (65537, 300), (70000, 1), (131073, 50000), (300001, 5000), (1 << 20, 50000),
                                          (200000, 3_000_000)])
def test_to_the_bit(ops, tokens, vocab, kind):
    """Whole numbers whose sums stay below 2^24, exact in fp32 in any order."""
    dim = 4
    ids = ids_of(kind, tokens, vocab).cuda()
    dout = torch.randint(-8, 9, (tokens, dim), generator=gen(1)).float().cuda()
    got = ops.embedding_grad(dout, ids, vocab)
    want, _, _ = S.embedding_grad(dout, ids, vocab, 1.0)
    assert torch.equal(got.cpu().double(), want)


@pytest.mark.parametrize("tokens", [65537, 300001])
def test_the_same_bits_from_run_to_run(ops, tokens):
    """Sums in fp32: their order goes by the tokens' places alone."""
    for vocab in (7, 900, 20000):
        ids = words(tokens, vocab, 2)
        dout = torch.randn(tokens, 40, device="cuda")
        first = ops.embedding_grad(dout, ids, vocab)
        want, size, count = S.embedding_grad(dout, ids, vocab, 1.0)
        bound = (count[:, None].double() + 2) * 2.0 ** -24 * size + 2.0 ** -24 * want.abs()
        assert ((first.cpu().double() - want).abs() <= bound).all()
        for _ in range(3):
            assert torch.equal(ops.embedding_grad(dout, ids, vocab), first)


def test_time_grows_with_the_tokens_and_not_with_their_square(ops):
    """Eight times as many tokens of one word, and of words that all come often: sixteen times the time is allowed."""
    def least(tokens, vocab):
        ids = torch.randint(vocab, (tokens,), device="cuda")
        dout, times = torch.randn(tokens, 8, device="cuda"), []
        for _ in range(4):
            start, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
            start.record()
            ops.embedding_grad(dout, ids, vocab)
            end.record()
            torch.cuda.synchronize()
            times.append(start.elapsed_time(end))
        return min(times)
    for vocab in (1, 50000):
        assert least(1 << 23, vocab) < 16 * least(1 << 20, vocab)
