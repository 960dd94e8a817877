"""The bias by buckets and its gradient against 64 bits: the gather to the bit, the scatter within the rounding of its sums."""
import pytest
import torch

import sequence_reference as ref

pytestmark = pytest.mark.gpu

SHAPES = [  # heads, Lq, Lk, columns, far, q_start
    (1, 1, 1, 1, 0, 0), (3, 49, 49, 32, 128, 0), (2, 7, 300, 8, 16, 0), (5, 130, 3, 32, 64, -5), (12, 64, 257, 16, 1, 190),
    (2, 1, 9000, 32, 128, 8999), (4, 515, 515, 64, 2000, 0), (1, 33, 65, 300, 8192, 1 << 40), (2, 100, 100, 7, 20, -(1 << 33)), (33, 40, 31, 4, 5, 3),
    (2, 4100, 5, 32, 300, 17),
]


def make(heads, Lq, Lk, nb, far, seed=0):
    g = torch.Generator().manual_seed(1000 * heads + Lq + 7 * Lk + seed)
    table = torch.randn(heads, nb, generator=g)
    buckets = torch.randint(0, nb, (2 * far + 1,), generator=g, dtype=torch.int32)
    return g, table, buckets


def cut(q_start):
    return max(-(1 << 29), min(1 << 29, q_start))


@pytest.mark.parametrize("heads,Lq,Lk,nb,far,q0", SHAPES)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_gather_is_the_table_to_the_bit(heads, Lq, Lk, nb, far, q0, dtype):
    import paper_2501_06480_amd as fwa
    _, table, buckets = make(heads, Lq, Lk, nb, far)
    got = fwa.fwa_bucket_gather(table.cuda(), buckets.cuda(), Lq, Lk, q0, dtype)
    want = ref.bias(table, buckets, Lq, Lk, cut(q0)).float().to(dtype)
    assert torch.equal(got.cpu(), want)


@pytest.mark.parametrize("heads,Lq,Lk,nb,far,q0", SHAPES)
def test_scatter_adds_up_every_pair_once(heads, Lq, Lk, nb, far, q0):
    import paper_2501_06480_amd as fwa
    g, _, buckets = make(heads, Lq, Lk, nb, far)
    x = torch.randn(heads, Lq, Lk, generator=g)
    xd, bd = x.cuda(), buckets.cuda()
    got = fwa.fwa_bucket_scatter(xd, bd, nb, q0)
    # a term passes through at most 9 additions of a diagonal, a few dozen of the lines and distances, 6 of the lanes
    tol = 96 * ref.U32 * ref.by_bucket(x.abs(), buckets, nb, cut(q0)) + (Lq / 32 + Lk / 64) * ref.U32 * ref.by_bucket(x.abs(), buckets, nb, cut(q0))
    ref.check(got, ref.by_bucket(x, buckets, nb, cut(q0)), tol, "dtable")
    assert torch.equal(got, fwa.fwa_bucket_scatter(xd, bd, nb, q0))


def test_entries_outside_the_table_add_nothing_and_get_nothing():
    import paper_2501_06480_amd as fwa
    g, table, buckets = make(3, 50, 70, 8, 30)
    buckets[::5] = -1
    buckets[::7] = 8
    buckets[11] = 1 << 30
    x = torch.randn(3, 50, 70, generator=g)
    assert torch.equal(fwa.fwa_bucket_gather(table.cuda(), buckets.cuda(), 50, 70).cpu(), ref.bias(table, buckets, 50, 70).float())
    want = ref.by_bucket(x, buckets, 8)
    ref.check(fwa.fwa_bucket_scatter(x.cuda(), buckets.cuda(), 8), want, 96 * ref.U32 * ref.by_bucket(x.abs(), buckets, 8), "dtable")


def test_nothing_is_written_outside_and_zero_sizes():
    import paper_2501_06480_amd as fwa
    _, table, buckets = make(2, 5, 7, 8, 4)
    room = torch.full((2 * 5 * 7 + 8,), 3.0, device="cuda")
    fwa.fwa_bucket_gather(table.cuda(), buckets.cuda(), 5, 7, out=room[:70].view(2, 5, 7))
    assert torch.equal(room[70:], torch.full((8,), 3.0, device="cuda"))
    assert fwa.fwa_bucket_gather(table.cuda(), buckets.cuda(), 0, 7).shape == (2, 0, 7)
    assert torch.equal(fwa.fwa_bucket_scatter(torch.empty(2, 5, 0, device="cuda"), buckets.cuda(), 8), torch.zeros(2, 8, device="cuda"))


@pytest.mark.parametrize("native", [True, False])
def test_bias_of_a_window_attention_with_the_gradient_of_its_table(native):
    """bucket_bias -> window_attention -> gradient of the table: the operators as a step of windows of a 1-D sequence uses them."""
    from paper_2501_06480_amd import autograd, binding
    g = torch.Generator().manual_seed(5)
    N, L, heads = 6, 100, 4
    buckets = binding.log_buckets(16, 40)
    table = (torch.randn(heads, 16, generator=g) * 0.3)
    q, k, v, d_o = (torch.randn(N, L, 32 * heads, generator=g).bfloat16() for _ in range(4))
    td = table.cuda().requires_grad_(True)
    make_bias = autograd.bucket_bias if native else lambda t, b, n: autograd._BucketBias.apply(t, b, n, n, 0, None)
    bias = make_bias(td, buckets.cuda(), L)
    o = autograd.window_attention(q.cuda(), k.cuda(), v.cuda(), heads, 32 ** -0.5, bias)
    dtable, = torch.autograd.grad(o, td, d_o.cuda())
    want = ref.attention(q, k, v, heads, 32 ** -0.5, table, buckets, d_o=d_o)
    ref.check(o, want["o"], want["o_tol"] + 1e-2, "o")
    # the gradient of the bias comes from the window kernels, which hold each of its elements to 1e-2
    count = ref.by_bucket(torch.ones(heads, L, L), buckets, 16)
    ref.check(dtable, want["dtable"], 1e-2 * count, "dtable")
