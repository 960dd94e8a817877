"""A training step captured into a graph: rotated queries and keys through the attention of whole sequences, and the gradients back through the rotation, replayed with other data and
positions against the eager step."""
import pytest
import torch

from test_gpu_rotary import BF16, F32, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_captured_forward_and_backward(dtype):
    from paper_2501_06480_amd import autograd
    N, L, H, KV, d = 2, 50, 4, 2, 64
    _, positions, f, axis, g = make(dtype, N, L, H, d, (20, 8))
    positions, f, axis = positions.cuda(), f.cuda(), axis.cuda()
    data = [torch.randn(N, L, h * d, generator=g).to(dtype).cuda() for h in (H, KV, KV, H)]

    def step(q, k, v, dy):
        q, k, v = (t.detach().requires_grad_(True) for t in (q, k, v))  # leaves of this step alone
        rq, rk = (autograd.rotary(t, h, positions, f, axis) for t, h in ((q, H), (k, KV)))
        o = autograd.sequence_attention(rq, rk, v, H, d ** -0.5, causal=True)
        return (o.detach(), *torch.autograd.grad(o, (q, k, v), dy))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(*data)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        captured = step(*data)
    for turn in range(3):
        for t in data:
            t.copy_(torch.randn(t.shape, generator=g))
        positions.copy_(torch.randint(0, 9000, positions.shape, generator=g, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in captured]
        for t in captured:
            t.fill_(7.0)
        for a, b in zip(got, step(*data)):
            assert torch.equal(a, b), turn
