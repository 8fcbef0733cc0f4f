"""What the binding of the layers in front of the LM head refuses by itself, whatever the device: an operand that a result needs and that is not given."""
import pytest
import torch

from paper_2603_16435_amd import binding

DY, X, STATS, GAMMA = torch.zeros(4, 8), torch.zeros(4, 16), torch.zeros(4, 2), torch.ones(8)


def _rows(rows, cols):
    return binding.F8Rows(torch.zeros(rows, 128, dtype=torch.uint8), torch.zeros(rows, 4, dtype=torch.uint8), cols)


@pytest.mark.parametrize("kept, w, want, says", [
    (None, None, {}, "packed transpose"), (None, None, dict(want_dx=False), "kept"), (None, None, dict(want_dw=False), "packed transpose"),
    (None, binding.F8Weight(_rows(8, 16), _rows(16, 8)), {}, "kept"), (_rows(4, 16), binding.F8Weight(_rows(8, 16)), {}, "packed transpose"),
    (_rows(4, 16), None, dict(want_dw=False), "packed transpose"), (X, binding.F8Weight(_rows(8, 16), _rows(16, 8)), {}, "kept"),
    (_rows(4, 16), binding.F8Weight(_rows(8, 16), _rows(16, 8)), dict(want_dx=False, want_dw=False), "neither")])
def test_linear_backward_names_what_is_missing(kept, w, want, says):
    with pytest.raises(ValueError, match=says):
        binding.rl_f8_linear_backward(DY, kept, w, **want)


@pytest.mark.parametrize("x", [None, "x", binding.F8Weight(_rows(4, 8))])
def test_layer_norm_backward_wants_x_or_its_checkpoint(x):
    with pytest.raises(ValueError, match="x must be"):
        binding.rl_layer_norm_backward(DY, x, STATS, GAMMA)
