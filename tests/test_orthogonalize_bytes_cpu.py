"""What the orthogonalised updates ask for as a workspace."""
import pytest

from paper_2601_07876_b200 import binding as B
from test_stream_ops_cpu import MUON, P, doubles, pointers, sizes


@pytest.fixture(scope="module")
def lib():
    return B.load_library()


def ask(lib, *shapes):
    return lib.novak_orthogonalize_bytes(sizes(*(r for r, _ in shapes)), sizes(*(c for _, c in shapes)), len(shapes))


@pytest.mark.parametrize("shape", [(1, 1), (64, 64), (17, 1000), (1000, 17), (1, 28000), (128, 512), (64, 4096)])
def test_matrices_that_stay_in_shared_memory_need_next_to_nothing(lib, shape):
    assert 0 < ask(lib, shape) <= 4096 and ask(lib, *[shape] * 5000) == ask(lib, shape)
    large = [(300, 300), (2048, 100)]
    assert ask(lib, *large, *[shape] * 100) == ask(lib, *[shape] * 100, *large) == ask(lib, *large) > 4 * 300 * 300


def test_nothing_needs_nothing(lib):
    assert ask(lib) == 0 and ask(lib, (0, 5), (5, 0)) == 0 and ask(lib, (0, 5), (5, 4)) > 0


def test_many_matrices_go_through_one_workspace_in_groups(lib):
    one = ask(lib, (4096, 4096))
    assert 10 * 4096 ** 2 <= one < 10.2 * 4096 ** 2
    for n in (7, 24, 400):                              # 6.7e9 elements
        assert 5 * one < ask(lib, *[(4096, 4096)] * n) <= 1 << 30
    assert ask(lib, *[(4096, 4096)] * 3) > 2.9 * one
    huge = ask(lib, (65536, 16384))                     # too large for a group of the usual size: one of its own
    assert ask(lib, *[(4096, 4096)] * 30, (65536, 16384), *[(4096, 4096)] * 30) == huge > 1 << 30


def test_operands_of_two_parts_take_more(lib):
    def fine(*shapes):
        return lib.novak_orthogonalize_fine_bytes(sizes(*(r for r, _ in shapes)), sizes(*(c for _, c in shapes)), len(shapes))
    assert 16 * 4096 ** 2 <= fine((4096, 4096)) < 16.2 * 4096 ** 2
    assert fine((64, 64)) == ask(lib, (64, 64)) and fine() == 0 and fine(*[(4096, 4096)] * 24) <= 1 << 30
    assert fine((65536 + 1, 4)) == 0


@pytest.mark.parametrize("change", [dict(work=None), dict(bytes=1000), dict(type=2), dict(n=-1), dict(steps=0), dict(eps=-1.0)])
def test_refusals_with_operands_of_two_parts(lib, change):
    base = dict(g=pointers(P, P), gs=sizes(9, 9), type=0, out=pointers(P, P), os=sizes(9, 9), rows=sizes(4, 5), cols=sizes(9, 9), n=2,
                abc=doubles(*MUON), steps=1, eps=1e-7, work=P, bytes=1 << 40, stream=None)
    assert lib.novak_orthogonalize_fine(*{**base, **change}.values()) == B.NOVAK_EINVAL and lib.novak_ops_error()
    change = {k: v for k, v in change.items() if k != "n"} or dict(n=-1)
    base = dict(theta=pointers(P), g=pointers(P), type=0, m=pointers(P), rows=sizes(4), cols=sizes(9), n=1, momentum=0.9, nesterov=1,
                step=doubles(0.1), decay=1.0, abc=doubles(*MUON), steps=1, eps=1e-7, work=P, bytes=1 << 40, stream=None)
    assert lib.novak_orthogonal_step_fine(*{**base, **change}.values()) == B.NOVAK_EINVAL       # (theta and m are one, too)
