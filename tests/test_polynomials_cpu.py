"""Which polynomials the orthogonalised updates take: the checks of the C entry point (made before any CUDA work)
against values on a fine grid."""
import random

import pytest

from paper_2601_07876_b200 import binding as B
from test_stream_ops_cpu import call, doubles


@pytest.fixture(scope="module")
def lib():
    return B.load_library()


def answer(lib, *coefficients):
    """"held" where the polynomials are refused, "work" where the missing workspace is all that is wrong."""
    assert call(lib, "novak_orthogonalize", abc=doubles(*coefficients), steps=len(coefficients) // 3, bytes=0) == B.NOVAK_EINVAL
    text = lib.novak_ops_error().decode()
    return "held" if "held" in text else "work" if "work" in text else text


@pytest.mark.parametrize("c", [0.0, 1e-18, -1e-18, 1e-300, 5e-324, 1e-6, -1e-6])
def test_a_vanishing_term_hides_no_maximum(lib, c):
    """12 x - 12 x^3 gets to 4.62 at x = 0.577, and to 0.24 at the ends."""
    assert answer(lib, 12.0, -12.0, c) == "held"
    assert answer(lib, 12.0, -12.0, c, 16.0, 0.0, 0.0) == "held"
    assert answer(lib, 1.5, -0.5, c) == "work"


def test_coefficients_whose_squares_overflow(lib):
    top = 1.01 ** 2
    assert answer(lib, 1e200, -1e200 / top, 0.0) == "held"
    assert answer(lib, 1e300, -2e300 / top, 1e300 / top ** 2) == "held"


def test_no_coefficients_at_all(lib):
    assert answer(lib, 0.0, 0.0, 0.0) == "work" and answer(lib, 0.0, 0.0, 0.0, 3.9, 0.0, 0.0) == "work"


def test_any_ratio_of_coefficients_against_a_grid(lib):
    """One step from [0, 1.01]: values of up to 4 and products of up to 15 are held."""
    rng = random.Random(5)
    grid = [1.01 * i / 4000 for i in range(4001)]
    seen = {"held": 0, "work": 0}
    for _ in range(1500):
        a, b, c = (rng.choice([-1, 1]) * 10 ** rng.uniform(-20, 1.5) if rng.random() < 0.6 else rng.uniform(-15, 15) for _ in range(3))
        value = max(abs(x * (a + x * x * (b + x * x * c))) for x in grid)
        product = max(abs(x * x * (b + x * x * c)) for x in grid)
        if abs(value - 4) < 0.01 or abs(product - 15) < 0.01:
            continue                                    # (nearer to the border than the grid is fine)
        want = "work" if value < 4 and product < 15 else "held"
        seen[want] += 1
        assert answer(lib, a, b, c) == want, (a, b, c, value, product)
    assert min(seen.values()) > 200
