"""The gradient of an output that is a part of a larger one and starts at any element of it."""
import pytest
import torch

from test_gpu_sequence import BF16, F32, device, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("native", [True, False])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_output_whose_gradient_starts_at_an_odd_element(native, dtype):
    from paper_2501_06480_amd import autograd
    x, t, _ = make(dtype, 2, 40, 40, 2, 2, 32)
    xd, td = device(x), device(t)
    leaves = [xd[n].requires_grad_(True) for n in "qkv"] + [td["table"].requires_grad_(True)]

    def call():
        if native:
            return autograd.sequence_attention(*leaves[:3], 2, 0.2, td["table"], td["buckets"])
        return autograd._SequenceAttention.apply(*leaves, td["buckets"], None, None, None, 2, 0.2, False)
    want = torch.autograd.grad(call(), leaves, xd["d_o"])
    flat = torch.cat([torch.zeros(1, dtype=dtype, device="cuda"), call().flatten()])
    got = torch.autograd.grad(flat, leaves, torch.cat([torch.zeros(1, dtype=dtype, device="cuda"), xd["d_o"].flatten()]))
    for a, b in zip(got, want):
        assert torch.equal(a, b)
