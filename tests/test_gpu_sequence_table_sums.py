"""The gradient of the table of many heads and several sequences of different lengths (128 rows a workgroup), and of a window attention's bias, each against
64 bits and the bound of its own sums."""
import pytest
import torch

import sequence_reference as ref
from test_gpu_sequence import BF16, F16, F32, device, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,N,L,H,KV,d,causal,far", [
    (BF16, 3, 300, 32, 32, 64, False, 40), (BF16, 4, 290, 24, 6, 128, True, 40), (F16, 3, 300, 30, 10, 64, True, 128),
    (BF16, 5, 170, 28, 28, 32, False, 500), (F32, 3, 260, 30, 30, 32, False, 8),
])
def test_table_of_many_heads_and_several_sequences(dtype, N, L, H, KV, d, causal, far):
    import paper_2501_06480_amd as fwa
    x, t, g = make(dtype, N, L, L, H, KV, d, far=far)
    t["causal"] = causal
    t["k_lengths"] = t["q_lengths"] = torch.randint(1, L + 1, (N,), generator=g, dtype=torch.int32)
    t["q_lengths"][N - 1] = L  # the last waves' rows exist in one sequence at least
    xd, td = device(x), device(t)
    o, stats = fwa.fwa_sequence_forward(xd["q"], xd["k"], xd["v"], H, d ** -0.5, want_stats=True, **td)
    dt = fwa.fwa_sequence_backward(xd["q"], xd["k"], xd["v"], o, stats, xd["d_o"], H, d ** -0.5, want_dtable=True, **td)[3]
    G = H // KV
    for kv in (0, KV - 1):
        hs, ks = slice(kv * G * d, (kv + 1) * G * d), slice(kv * d, (kv + 1) * d)
        want = ref.attention(x["q"][..., hs], x["k"][..., ks], x["v"][..., ks], G, d ** -0.5, t["table"][kv * G:(kv + 1) * G], t["buckets"],
                             t["q_lengths"], t["k_lengths"], None, causal, x["d_o"][..., hs])
        assert float(want["dtable"].abs().max()) > 4 * float(want["dtable_tol"].max())  # the bound tells something
        ref.check(dt[kv * G:(kv + 1) * G], want["dtable"], want["dtable_tol"], f"dtable {kv}")


def test_table_of_a_window_attention_is_the_sum_of_its_bias_gradient():
    """The dense gradient as the window attention hands it over, added up in 64 bits."""
    from paper_2501_06480_amd import autograd, binding
    g = torch.Generator().manual_seed(6)
    N, L, heads = 6, 100, 4
    buckets = binding.log_buckets(16, 40)
    table = (torch.randn(heads, 16, generator=g) * 0.3).cuda().requires_grad_(True)
    q, k, v, d_o = (torch.randn(N, L, 32 * heads, generator=g).bfloat16().cuda() for _ in range(4))
    bias = autograd.bucket_bias(table, buckets.cuda(), L)
    o = autograd.window_attention(q, k, v, heads, 32 ** -0.5, bias)
    dbias, dtable = torch.autograd.grad(o, (bias, table), d_o)
    x = dbias.cpu()
    sizes = ref.by_bucket(x.abs(), buckets, 16)
    # a term passes through at most 9 additions of a diagonal, a few dozen of the lines and distances, 6 of the lanes
    ref.check(dtable, ref.by_bucket(x, buckets, 16), (96 + L / 32 + L / 64) * ref.U32 * sizes, "dtable")
    want = ref.attention(q.cpu(), k.cpu(), v.cpu(), heads, 32 ** -0.5, table.detach().cpu(), buckets, d_o=d_o.cpu())
    # each dS is a few roundings of bf16 (2^-8) off, of independent signs: a dozen of them in norm
    far_off = (dtable.detach().cpu().double() - want["dtable"]).abs()
    assert float((far_off ** 2).sum().sqrt()) < 0.05 * float((want["dtable"] ** 2).sum().sqrt())
