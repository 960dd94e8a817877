"""The gradient of a bias by buckets that is a part of a larger one and starts at any element of it."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("native", [True, False])
@pytest.mark.parametrize("dtype", [None, torch.bfloat16])
def test_bias_whose_gradient_starts_at_an_odd_element(native, dtype):
    """Biases of two tables of odd size next to each other: the gradient of the second is contiguous and not aligned."""
    from paper_2501_06480_amd import autograd, binding
    g = torch.Generator().manual_seed(1)
    L, buckets = 49, binding.log_buckets(16, 40).cuda()
    tables = [torch.randn(3, 16, generator=g).cuda().requires_grad_(True) for _ in range(2)]
    make_bias = (lambda t: autograd.bucket_bias(t, buckets, L, dtype=dtype)) if native else (lambda t: autograd._BucketBias.apply(t, buckets, L, L, 0, dtype))
    both = torch.cat([make_bias(t) for t in tables])
    w = torch.randn(both.shape, generator=g).to(both.dtype).cuda()
    got = torch.autograd.grad(both, tables, w)
    for x, part in zip(got, (w[:3], w[3:])):
        assert torch.equal(x, binding.fwa_bucket_scatter(part.float().clone(), buckets, 16))
