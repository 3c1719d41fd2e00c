"""Workspaces whose contents are anything, and two of everything at a time: the C entries as a program with its own
buffers calls them."""
import ctypes

import pytest
import torch

from paper_2601_07876_b200 import binding as B

pytestmark = pytest.mark.gpu
F32 = torch.float32
FILLS = [0, 0xff, 0x7f, 0x01]          # zeros, NaNs, large numbers, small ones


@pytest.fixture(scope="module")
def ops():
    from paper_2601_07876_b200 import ops
    return ops


@pytest.fixture(scope="module")
def lib():
    return B.load_library()


def filled(size, byte):
    """A workspace and guards on both sides of it."""
    t = torch.full((size + 512,), byte, dtype=torch.uint8, device="cuda")
    return t, t[256:256 + size]


def guards(t, byte):
    return bool((t[:256] == byte).all() and (t[-256:] == byte).all())


def stream():
    return torch.cuda.current_stream().cuda_stream


@pytest.mark.parametrize("byte", FILLS)
def test_orthogonalize(ops, lib, byte):
    torch.manual_seed(1)
    shapes = [(70, 33), (130, 300), (1, 5), (513, 257)]
    g = [torch.randn(*s, device="cuda") for s in shapes]
    want = ops.orthogonalize(g)
    n = len(g)
    rows, cols = ((ctypes.c_int64 * n)(*(s[i] for s in shapes)) for i in range(2))
    need = lib.novak_orthogonalize_bytes(rows, cols, n)
    base, work = filled(need, byte)
    out = [torch.empty_like(w) for w in want]
    coefficients = [x for c in ops.NEWTON_SCHULZ for x in c]
    assert lib.novak_orthogonalize((ctypes.c_void_p * n)(*(t.data_ptr() for t in g)), cols, 0,
                                   (ctypes.c_void_p * n)(*(t.data_ptr() for t in out)), cols, rows, cols, n,
                                   (ctypes.c_double * len(coefficients))(*coefficients), len(ops.NEWTON_SCHULZ), 1e-7,
                                   work.data_ptr(), need, stream()) == B.NOVAK_OK
    assert all(torch.equal(a, b) for a, b in zip(out, want)) and guards(base, byte)


@pytest.mark.parametrize("byte", FILLS)
@pytest.mark.parametrize("tokens,vocab,dim", [(1, 1, 1), (197, 1003, 771), (5000, 40, 64)])
def test_embedding_grad(ops, lib, byte, tokens, vocab, dim):
    torch.manual_seed(2)
    ids = torch.randint(-1, vocab + 1, (tokens,), device="cuda")
    dout = torch.randn(tokens, dim, device="cuda")
    want = ops.embedding_grad(dout, ids, vocab, 1.5)
    need = lib.novak_embedding_grad_bytes(tokens, vocab, dim)
    base, work = filled(need, byte)
    out = torch.full((vocab, dim), 9.0, device="cuda")
    assert lib.novak_embedding_grad(dout.data_ptr(), dim, 0, ids.data_ptr(), B.NOVAK_ID_I64, 1.5, out.data_ptr(), dim, 0, 0,
                                    work.data_ptr(), need, tokens, vocab, dim, stream()) == B.NOVAK_OK
    assert torch.equal(out, want) and guards(base, byte)


@pytest.mark.parametrize("byte", FILLS)
@pytest.mark.parametrize("rows,width", [(1, 8), (700, 96), (33, 4096)])
def test_rms_norm_backward(ops, lib, byte, rows, width):
    torch.manual_seed(3)
    x, w, dy = torch.randn(rows, width, device="cuda"), torch.randn(width, device="cuda"), torch.randn(rows, width, device="cuda")
    _, _, rstd, kept = ops.rms_norm(x, w, checkpoint=True)
    dx, dw = ops.rms_norm_backward(dy, kept, rstd, w)
    need = lib.novak_rms_norm_backward_bytes(rows, width)
    base, work = filled(need, byte)
    got, dgamma = torch.empty_like(dx), torch.empty_like(dw)
    assert lib.novak_rms_norm_backward(dy.data_ptr(), width, None, 0, None, 0, 0, rstd.data_ptr(), kept.codes_ptr, kept.exps_ptr,
                                       w.data_ptr(), 0, got.data_ptr(), width, dgamma.data_ptr(), 0, work.data_ptr(), need, rows,
                                       width, stream()) == B.NOVAK_OK
    assert torch.equal(got, dx) and torch.equal(dgamma, dw) and guards(base, byte)


def test_two_of_each_at_a_time(ops):
    """Calls of two streams that run beside one another, each with its own results: the same as alone."""
    torch.manual_seed(4)
    ids = [torch.randint(500, (3000,), device="cuda") for _ in range(2)]
    dout = [torch.randn(3000, 256, device="cuda") for _ in range(2)]
    g = [torch.randn(1500, 700, device="cuda") for _ in range(2)]
    gamma = torch.randn(256, device="cuda")

    def work(i):
        out = [ops.embedding_grad(dout[i], ids[i], 500), ops.orthogonalize(g[i])]
        y, h, rstd, kept = ops.rms_norm(dout[i], gamma, residual=dout[1 - i], checkpoint=True)
        return out + [y, h, *ops.rms_norm_backward(y, kept, rstd, gamma, dh=dout[i])]
    want = [work(i) for i in range(2)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[], []]
    for _ in range(10):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(work(i))
    torch.cuda.synchronize()
    for i in range(2):
        for out in got[i]:
            assert all(torch.equal(a, b) for a, b in zip(out, want[i]))
    assert ops.wait_failures() == 0


def test_two_graphs(ops):
    """Two captured calls replayed side by side: each has its own workspace."""
    torch.manual_seed(5)
    ids = [torch.randint(300, (2000,), device="cuda") for _ in range(2)]
    dout = [torch.randn(2000, 128, device="cuda") for _ in range(2)]
    g = [torch.randn(600, 900, device="cuda") for _ in range(2)]
    want = [(ops.embedding_grad(dout[i], ids[i], 300), ops.orthogonalize(g[i])) for i in range(2)]
    graphs, out = [], []
    for i in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out.append((ops.embedding_grad(dout[i], ids[i], 300), ops.orthogonalize(g[i])))
        graphs.append(graph)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(5):
        for s, graph in zip(streams, graphs):
            with torch.cuda.stream(s):
                graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for i in range(2) for a, b in zip(out[i], want[i]))
