"""What the bindings say of a tensor of another shape (CPU only)."""
import pytest
import torch

from paper_2607_28848_amd import _marshal


@pytest.mark.parametrize("shape", [(6, 4, 32), (5, 4, 64), (6, 255), (6,), (), (1, 6, 4, 64)])
def test_the_shape_that_was_given_is_named(shape):
    with pytest.raises(ValueError) as e:
        _marshal.view(torch.zeros(shape), 6, 4, 64, torch.float32, "K_out")
    assert str(e.value) == "K_out must be [6][4][64], got %s" % (shape,)
