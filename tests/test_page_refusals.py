"""Refusals of the paged and rotary calls that come before anything looks at a device (no GPU needed)."""
import pytest
import torch


def test_a_negative_number_of_new_tokens_is_refused():
    """As by the C call; left out it means any number."""
    import paper_2501_06480_amd as fwa
    pool, i = torch.zeros(2, 16, 2, 64), torch.int32
    args = (torch.zeros(4, 128), pool, pool.clone(), torch.zeros(1, 2, dtype=i), torch.zeros(2, dtype=i), torch.zeros(1, dtype=i), 2, 0.1)
    for most in (-1, -5):
        with pytest.raises(ValueError, match="most_new"):
            fwa.fwa_page_forward(*args, most_new=most)
    for most in (None, 3):
        with pytest.raises(TypeError):  # not on a GPU
            fwa.fwa_page_forward(*args, most_new=most)


def test_frequencies_that_want_a_gradient_are_refused():
    """They would be left without one in silence."""
    from paper_2501_06480_amd import autograd
    x, positions, f = torch.zeros(1, 4, 128), torch.zeros(4, 1, dtype=torch.int32), torch.nn.Parameter(torch.ones(32))
    with pytest.raises(NotImplementedError, match="frequencies"):
        autograd.rotary(x, 2, positions, f)
    with torch.no_grad(), pytest.raises(TypeError):  # not on a GPU
        autograd.rotary(x, 2, positions, f)
    with pytest.raises(TypeError):
        autograd.rotary(x, 2, positions, f.detach())


def test_frequencies_that_are_no_tensor_are_refused_as_such():
    from paper_2501_06480_amd import autograd
    x, positions = torch.zeros(1, 4, 128), torch.zeros(4, 1, dtype=torch.int32)
    for f in (None, [1.0] * 32):
        with pytest.raises(TypeError):
            autograd.rotary(x, 2, positions, f)
