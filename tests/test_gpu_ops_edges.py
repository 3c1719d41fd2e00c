"""The training operators where memory ends and numbers do: what stands behind their vectors, infinities, sums that
overflow."""
import math

import pytest
import torch

import ops_reference as R
from test_gpu_ops import BF16, F32, TYPES, check_layer_norm, gen, matrix

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ops():
    from paper_2601_07876_b200 import ops
    return ops


# ---- what stands behind a vector --------------------------------------------------
def slice_of_nans(n, dtype, offset, values):
    """A vector of these values, NaNs before and behind it."""
    buf = torch.full((offset + n + 64,), math.nan, dtype=dtype, device="cuda")
    buf[offset:offset + n] = values.to(dtype)
    return buf[offset:offset + n]


@pytest.mark.parametrize("param", TYPES)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", [7, 96, 257, 771, 1001, 1031, 2048, 4099, 8190, 20001])
def test_nothing_behind_weight_and_bias_is_read(ops, cols, dtype, param):
    rows, g = 9, gen(cols)
    x, dy = matrix(rows, cols, dtype, cols), matrix(rows, cols, dtype, cols + 1, scale=1e-3)
    values, shift = 1 + 0.2 * torch.randn(cols, generator=g), torch.randn(cols, generator=g)
    for offset in (0, 1):
        w, b = slice_of_nans(cols, param, offset, values), slice_of_nans(cols, param, offset, shift)
        y, mean, rstd, kept = ops.layer_norm(x, w, b, checkpoint=True)
        check_layer_norm(ops, x, w, b, 1e-5, y, mean, rstd, kept)
        from_x = (x.cpu().double() - mean.cpu().double()[:, None]) * rstd.cpu().double()[:, None]
        for saved, ref, err in ((kept, R.act8_values(kept.codes, kept.exps, cols), 0.0), (x, from_x, 3 * R.U)):
            got = ops.layer_norm_backward(dy, saved, rstd, w, mean=mean)
            want = R.layer_norm_backward(dy, ref, rstd, w)
            bounds = R.layer_norm_backward_bounds(dy, ref, rstd, w, dtype, F32, err)
            for a, c, bound, what in zip(got, want, bounds, ("dx", "dw", "db")):
                R.assert_within(a, c, bound, what)


# ---- a form's shape ---------------------------------------------------------------
def test_unpacking_writes_nothing_but_the_forms_elements(ops):
    kept = ops.act8_pack(matrix(300, 64, F32, 1))
    again = ops.Act8(kept.codes, kept.exps, 64, shape=(3, 100, 64))
    assert torch.equal(ops.act8_unpack(again).view(300, 64), ops.act8_unpack(kept))
    for out in (torch.zeros(1, 64, device="cuda"), torch.zeros(64, 300, device="cuda").t(), torch.zeros(301, 64, device="cuda")):
        with pytest.raises(ValueError, match="elements"):
            ops._calls.unpack(kept, out)
        assert not out.any()


# ---- infinities through the activation functions -------------------------------------
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kind", ["gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("cols", [96, 33])
def test_infinities_and_nans_through_the_activations(ops, cols, kind, dtype):
    """f(inf) = inf.  f(-inf) is -inf times 0 by each of the formulas, a NaN; the slopes at the infinities are NaNs too
    or their limits, 1 and 0.  Neighbours see nothing of it."""
    u = matrix(5, cols, dtype, 1)
    clean, _, _ = ops.activation(u, kind, save_input=False)
    slope = ops.activation_backward(torch.ones_like(u), u, kind)
    at = {(0, 3): math.inf, (1, 8): -math.inf, (2, cols - 1): math.nan, (4, 0): math.inf}
    for place, value in at.items():
        u[place] = value
    a, _, kept_a = ops.activation(u, kind, save_output=True)
    du = ops.activation_backward(torch.ones_like(u), u, kind)
    for place, value in at.items():
        if value == math.inf:
            assert a[place] == math.inf
        else:
            assert torch.isnan(a[place])
        limit = 1.0 if value == math.inf else 0.0
        assert torch.isnan(du[place]) or (du[place] == limit and not math.isnan(value))
    others = torch.ones(5, cols, dtype=torch.bool, device="cuda")
    for place in at:
        others[place] = False
    assert torch.equal(a[others], clean[others]) and torch.equal(du[others], slope[others])
    blocks = torch.nn.functional.pad(~torch.isfinite(a), (0, -cols % 32)).view(5, -1, 32).any(2)
    assert torch.equal(kept_a.exps == 255, blocks)


# ---- sums that overflow ----------------------------------------------------------------
@pytest.mark.parametrize("cols,offset", [(8, 0), (40, 0), (40, 1), (1024, 0), (4096, 0), (9000, 0)])
def test_a_deviation_that_overflows_is_the_same_nan_in_both_results(ops, cols, offset):
    """fp32's largest numbers: the first element's deviation from the mean is an infinity, the root's reciprocal 0, and
    xhat a NaN there and 0 in the others.  Its block of the 8-bit form stands for NaNs."""
    buf = torch.zeros(offset + 2 * cols, device="cuda")
    x = buf[offset:].view(2, cols)
    top = 3.4028234e38
    x[0, 0], x[0, 1:] = top, -1.01 * top / (cols - 1)       # (no part of their sum overflows; the mean is below 0)
    x[1] = torch.linspace(-1, 1, cols, device="cuda")
    w = torch.ones(cols, device="cuda")
    y, _, _, kept = ops.layer_norm(x, w, checkpoint=True)
    value = ops.act8_unpack(kept, dtype=F32)
    bad = torch.isnan(y)
    assert bad[0, 0] and not bad[0, 1:].any() and not bad[1].any()
    blocks = torch.nn.functional.pad(bad, (0, -cols % 32)).view(2, -1, 32).any(2)
    assert torch.equal(kept.exps == 255, blocks)
    assert torch.equal(torch.isnan(value), blocks.repeat_interleave(32, 1)[:, :cols])


# ---- a form's buffer -------------------------------------------------------------------
def test_a_form_from_its_buffer_is_the_form(ops):
    x = matrix(30, 70, F32, 1)
    kept = ops.act8_pack(x.view(3, 10, 70) if x.is_contiguous() else x)
    by_parts = ops.Act8(kept.codes.clone(), kept.exps.clone(), 70)
    for form in (kept, by_parts):
        copy = ops.Act8.from_buffer(form.buffer.clone(), 70, shape=(3, 10, 70))
        assert copy.rows == 30 and torch.equal(copy.codes, kept.codes) and torch.equal(copy.exps, kept.exps)
        assert torch.equal(ops.act8_unpack(copy).view(30, 70), ops.act8_unpack(kept).view(30, 70))
    for cols, shape in ((64, None), (70, (3, 11, 70)), (70, (30, 64))):
        with pytest.raises(ValueError):
            ops.Act8.from_buffer(kept.buffer[:-1] if shape is None else kept.buffer, cols, shape)


# ---- bits -------------------------------------------------------------------------------
def off(got, want):
    return float((got.cpu().double() - want).norm() / want.norm())


@pytest.mark.parametrize("lo,hi", [(-1, 1), (-0.01, 0.01), (-3, 3), (0, 6), (-4, -1), (-6, -3)])
def test_gelu_in_fp32_is_as_good_as_the_formula_in_fp32(ops, lo, hi):
    """Against the definition in 64 bits, over 2^18 numbers: no further off in the norm than u (1 + erf) / 2 and its
    slope by one fp32 operation after another; a tenth more is allowed for the sample."""
    u = (lo + (hi - lo) * torch.rand(256, 1024, generator=gen(2), dtype=torch.float64)).float().cuda()
    cdf = 0.5 * (1 + torch.erf(u * math.sqrt(0.5)))
    want = R.act("gelu", u)
    assert off(ops.activation(u, "gelu")[0], want) <= 1.1 * off(u * cdf, want)
    want = R.act_slope("gelu", u)
    plain = cdf + u * torch.exp(-0.5 * u * u) * (1 / math.sqrt(2 * math.pi))
    assert off(ops.activation_backward(torch.ones_like(u), u, "gelu"), want) <= 1.1 * off(plain, want)


# ---- more rows than a grid's second dimension holds --------------------------------------
@pytest.mark.parametrize("cols", [33, 40])
def test_more_rows_than_the_grid_has_places_for(ops, cols):
    """1.1 million rows, 16 to a CTA: the CTAs go on with further rows.  Rows know nothing of one another, so that the
    last ones on their own give the same bits."""
    rows, part = 1_100_000, slice(1_000_000, None)
    g = torch.Generator(device="cuda").manual_seed(1)
    u = torch.empty(rows, cols, device="cuda").normal_(generator=g).to(BF16)
    da = torch.empty(rows, cols, device="cuda").normal_(generator=g).to(BF16)
    a, kept_u, kept_a = ops.activation(u, "gelu", save_output=True)
    du, back = ops.activation_backward(da, kept_u, "gelu"), ops.act8_unpack(kept_a)
    few, few_u, few_a = ops.activation(u[part].contiguous(), "gelu", save_output=True)
    assert torch.equal(a[part], few) and torch.equal(kept_u.codes[part], few_u.codes)
    assert torch.equal(kept_a.exps[part], few_a.exps) and torch.equal(back[part], ops.act8_unpack(few_a))
    assert torch.equal(du[part], ops.activation_backward(da[part].contiguous(), few_u, "gelu"))
    assert torch.equal(ops.act8_pack(u).codes, kept_u.codes)
