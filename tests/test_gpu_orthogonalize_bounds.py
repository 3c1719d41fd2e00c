"""How far orthogonalised updates are from the definition in 64 bits: what include/novak.h promises of them, over many
matrices of every size and of unlike kinds."""
import math

import pytest
import torch

import stream_reference as S
from test_gpu_ops import gen
from test_gpu_orthogonalize import far, spectrum

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16

# Sides of up to 64, or 128 where the other one is up to 512: operands of two fp16 parts, sums in fp32.  With u = 2^-23
# (half a step of a first part is 2^-12 of it, of a second part 2^-12 of that, of a sum 2^-24): a step adds 5.6 u of X's norm
# (orthogonal_tolerance has the terms), and in the directions in which X is small all that is there is multiplied
# by 3.4445 with every step left: the rounding of G itself by 3.4445^5 = 485, the steps' by 3.4445^4 + ... + 1 = 198.
# That is (485 + 5.6 * 198) u = 1.9e-4, which takes nearly all of G in one direction.
TWO_PARTS = (485 + 5.6 * 198) * 2.0 ** -23
# Where that is not so: what is added where singular values end (11 u a step in all, without a mean), and three times
# as much for the growth on the way there.
TWO_PARTS_DENSE = 3 * 5 * 11 * 2.0 ** -23


@pytest.fixture(scope="module")
def ops():
    from paper_2601_07876_b200 import ops
    return ops


def unrounded(ops, g):
    """X before it is rounded to bf16, of many gradients: the step of parameters of zeros."""
    theta, m = ([torch.zeros(x.shape, device="cuda") for x in g] for _ in range(2))
    ops.orthogonal_step(theta, g, m, [-1.0] * len(g), momentum=0.0, nesterov=False)
    return theta


def few(rows, cols, seed):
    """A gradient carried by a few elements."""
    g = gen(seed)
    x = torch.zeros(rows, cols)
    n = 1 + seed % 4
    x[torch.randint(rows, (n,), generator=g), torch.randint(cols, (n,), generator=g)] = 1 + torch.randn(n, generator=g).abs()
    return x.cuda()


def kinds(rows, cols, count):
    for kind in ("gauss", "low rank", "rank one", "unlike features"):
        yield kind, [spectrum(rows, cols, kind, 1000 * rows + i) for i in range(count)]
    yield "few", [few(rows, cols, i) for i in range(count)]


@pytest.mark.parametrize("rows,cols,count", [(1, 1, 40), (1, 9, 40), (2, 2, 400), (2, 9, 400), (9, 2, 100), (3, 5, 200), (8, 8, 200), (12, 30, 100),
                                             (15, 15, 100), (17, 1000, 20), (32, 32, 50), (33, 70, 30), (70, 33, 30), (64, 64, 20), (64, 500, 10),
                                             (96, 100, 10), (128, 128, 10), (128, 400, 5), (500, 80, 5)])
def test_small_matrices_are_as_good_as_fp32(ops, rows, cols, count):
    for kind, g in kinds(rows, cols, count):
        for a, x in zip(g, unrounded(ops, g)):
            want = S.orthogonalized(a)
            assert far(x, want) <= (TWO_PARTS if kind in ("rank one", "low rank") else TWO_PARTS_DENSE), kind


# Larger ones: operands of 11 bits.  The plain sum of what roundings can do (orthogonal_tolerance), 11 u a step with u = 2^-12,
# holds whatever G is; twice their mean square where so many elements carry G that means hold.
ANY = 5 * 11 * 2.0 ** -12


@pytest.mark.parametrize("rows,cols,count", [(65, 600, 8), (129, 129, 20), (200, 300, 20), (300, 200, 20), (256, 300, 20), (700, 257, 5), (768, 768, 3)])
def test_larger_matrices(ops, rows, cols, count):
    unlike = [spectrum(rows, cols, "unlike features", 77 + i).abs().pow(3.0) for i in range(count)]      # of a few rows and columns
    for kind, g in [*kinds(rows, cols, count), ("very unlike features", unlike)]:
        for a, x in zip(g, unrounded(ops, g)):
            means = kind not in ("few", "very unlike features")
            assert far(x, S.orthogonalized(a)) <= (S.orthogonal_tolerance(rows, cols) if means else ANY), kind


@pytest.mark.parametrize("rows,cols", [(200, 300), (300, 200), (768, 768)])
def test_a_gradient_of_low_rank_keeps_its_second_part_to_the_end(ops, rows, cols):
    """Without it the last step would add 3.4445 u, a times the first part's rounding, in the directions in which B has
    nothing.  With it there are the products' roundings, 5.6 u / sqrt(3) in the mean of a step where singular values
    end, which is the last step's alone here; a tenth is allowed on top."""
    for kind in ("low rank", "rank one"):
        g = [spectrum(rows, cols, kind, 5 + i) for i in range(4)]
        for a, x in zip(g, unrounded(ops, g)):
            assert far(x, S.orthogonalized(a)) <= 1.1 * 5.6 * 2.0 ** -12 / math.sqrt(3), kind
