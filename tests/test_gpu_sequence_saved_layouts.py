"""Saved tensors that a hook hands back in another layout than the calls take."""
import pytest
import torch

from test_gpu_sequence import BF16, device, make

pytestmark = pytest.mark.gpu


def other_layout(y):
    """the same values with the axes in memory the other way round, one element into their storage"""
    if y.dim() == 1:
        wide = torch.zeros(2 * y.numel() + 1, dtype=y.dtype, device=y.device)[1::2]
        return wide.copy_(y)
    shape = tuple(reversed(y.shape))
    room = torch.zeros(y.numel() + 1, dtype=y.dtype, device=y.device)[1:].view(shape)
    return room.permute(*reversed(range(y.dim()))).copy_(y)


@pytest.mark.parametrize("native", [True, False])
@pytest.mark.parametrize("which", [None, 0, 1, 2, 3, 4, 5, 6, 7, 8, 9])
def test_saved_tensors_that_come_back_in_another_layout(native, which):
    from paper_2501_06480_amd import autograd
    x, t, _ = make(BF16, 2, 70, 70, 4, 2, 32)
    xd, td = device(x), device(t)
    td["q_lengths"], td["k_lengths"], td["q_start"] = (torch.tensor(y, dtype=torch.int32, device="cuda") for y in ([70, 50], [70, 61], [0, 3]))
    leaves = [xd[n].requires_grad_(True) for n in "qkv"] + [td["table"].requires_grad_(True)]

    def call():
        if native:
            return autograd.sequence_attention(*leaves[:3], 4, 0.2, td["table"], td["buckets"], td["q_lengths"], td["k_lengths"], td["q_start"], True)
        return autograd._SequenceAttention.apply(*leaves, td["buckets"], td["q_lengths"], td["k_lengths"], td["q_start"], 4, 0.2, True)
    want = torch.autograd.grad(call(), leaves, xd["d_o"])
    packed = []

    def pack(y):
        packed.append(y)
        return len(packed) - 1, y.detach()

    def unpack(entry):
        return other_layout(entry[1]) if which in (None, entry[0]) else entry[1]
    with torch.autograd.graph.saved_tensors_hooks(pack, unpack):
        o = call()
    assert len(packed) == 10
    got = torch.autograd.grad(o, leaves, xd["d_o"])
    for a, b in zip(got, want):
        assert torch.equal(a, b)


@pytest.mark.parametrize("native", [True, False])
def test_map_that_comes_back_in_another_layout(native):
    from paper_2501_06480_amd import autograd, binding
    buckets = binding.log_buckets(16, 40).cuda()
    table = torch.randn(3, 16, generator=torch.Generator().manual_seed(2)).cuda().requires_grad_(True)
    call = (lambda: autograd.bucket_bias(table, buckets, 30)) if native else (lambda: autograd._BucketBias.apply(table, buckets, 30, 30, 0, None))
    w = torch.randn(3, 30, 30, generator=torch.Generator().manual_seed(3)).cuda()
    want, = torch.autograd.grad(call(), table, w)
    with torch.autograd.graph.saved_tensors_hooks(lambda y: y.detach(), other_layout):
        bias = call()
    got, = torch.autograd.grad(bias, table, w)
    assert torch.equal(got, want)
