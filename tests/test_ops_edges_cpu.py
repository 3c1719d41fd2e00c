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


@pytest.mark.parametrize("cols", [0, -5, -100, 64])
def test_a_form_is_refused_a_buffer_that_is_not_its_own(cols):
    from paper_2601_07876_b200 import ops
    with pytest.raises(ValueError, match="buffer"):
        ops.Act8.from_buffer(torch.zeros(66 * 4 + 1, dtype=torch.uint8), cols)
    for wrong in (torch.zeros(66), torch.zeros(4, 66, dtype=torch.uint8), torch.zeros(132, dtype=torch.uint8)[::2]):
        with pytest.raises(TypeError):
            ops.Act8.from_buffer(wrong, cols)


def test_no_workspace_is_asked_for_what_will_be_refused():
    """A caller is to see the reason, not an allocation that fails first."""
    from paper_2601_07876_b200 import binding as B
    lib = B.load_library()
    base = dict(dy=1 << 20, stride=4096, type=0, rows=1000, n_out=4096, n_in=4096)
    ask = lib.novak_linear_weight_grad_bytes
    assert ask(*base.values()) > 0
    for change in (dict(n_in=(1 << 22) + 1), dict(n_out=(1 << 22) + 1, stride=(1 << 22) + 1), dict(rows=1 << 31),
                   dict(rows=-1), dict(n_in=0), dict(n_out=0), dict(type=2)):
        assert ask(*{**base, **change}.values()) == 0, change
    assert ask(*{**base, "n_in": 1 << 22}.values()) > 0
