"""Refusals of the training operators' Python side that need no GPU."""
import pytest
import torch


@pytest.mark.parametrize("shape", [(1, 64), (300, 32), (300,), (), (2, 100, 64), (299, 64), (3, 100, 63), (-300, 64)])
def test_a_form_is_refused_a_shape_that_is_not_its_own(shape):
    """Unpacking writes a tensor of this shape: it has to hold the form's elements."""
    from paper_2601_07876_b200 import ops
    codes, exps = torch.zeros(300, 64, dtype=torch.int8), torch.zeros(300, 2, dtype=torch.uint8)
    with pytest.raises(ValueError, match="fold"):
        ops.Act8(codes, exps, 64, shape=shape)
