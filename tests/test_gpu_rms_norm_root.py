"""The root-mean-square norm's reciprocal root, to the bit."""
import pytest
import torch

from test_gpu_ops import TYPES, gen, vector

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ops():
    from paper_2601_07876_b200 import ops
    return ops


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", [1, 31, 768, 771, 4096, 9000])
@pytest.mark.parametrize("eps", [0.0, 1e-6, 0.5])
def test_each_operation_of_rstd_is_correctly_rounded(ops, cols, eps, dtype):
    """Rows of whole numbers whose squares' sum is below 2^24: exact in fp32 in any order.  Then the mean, eps and the
    reciprocal root, a rounding each (from 64 bits: a double rounding would take a tie in 29 bits)."""
    g = gen(cols)
    x = torch.randint(-30, 31, (500, cols), generator=g).to(dtype).cuda()
    x[:, 0] = 7
    total = x.cpu().double().square().sum(1)
    assert float(total.max()) < 2 ** 24
    mean = (total / cols).float()
    want = (1.0 / (mean + torch.tensor(eps, dtype=torch.float32)).double().sqrt()).float()
    residual = torch.zeros_like(x)
    for kw in (dict(), dict(residual=residual)):
        assert torch.equal(ops.rms_norm(x, vector(cols, torch.float32, 1), eps=eps, **kw)[2].cpu(), want)
