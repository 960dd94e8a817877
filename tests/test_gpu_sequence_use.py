"""The bias by buckets and the attention of whole sequences as programs use them: through autograd, on streams of their own, captured in graphs,
against long strided caches, a prompt and its new tokens one after the other."""
import pytest
import torch

import sequence_reference as ref
from test_gpu_sequence import BF16, F16, F32, device, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("native", [True, False])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_autograd_gives_the_gradients_of_the_call(native, dtype):
    import paper_2501_06480_amd as fwa
    from paper_2501_06480_amd import autograd
    x, t, _ = make(dtype, 2, 150, 150, 4, 2, 64)
    t["causal"] = True
    t["k_lengths"] = t["q_lengths"] = torch.tensor([150, 101], dtype=torch.int32)
    xd, td = device(x), device(t)
    o, stats = fwa.fwa_sequence_forward(xd["q"], xd["k"], xd["v"], 4, 0.125, want_stats=True, **td)
    want = fwa.fwa_sequence_backward(xd["q"], xd["k"], xd["v"], o, stats, xd["d_o"], 4, 0.125, want_dtable=True, **td)
    leaves = [y.clone().requires_grad_(True) for y in (xd["q"], xd["k"], xd["v"], td["table"])]
    rest = {n: y for n, y in td.items() if n != "table"}
    if native:
        got = autograd.sequence_attention(*leaves[:3], 4, 0.125, table=leaves[3], **rest)
    else:
        got = autograd._SequenceAttention.apply(*leaves, td["buckets"], td["q_lengths"], td["k_lengths"], None, 4, 0.125, True)
    assert torch.equal(got, o)
    got.backward(xd["d_o"])
    for y, w in zip(leaves, want):
        assert torch.equal(y.grad, w)
    # only what is asked for, from an expanded gradient
    q = leaves[0].detach().requires_grad_(True)
    one, = torch.autograd.grad(autograd.sequence_attention(q, xd["k"], xd["v"], 4, 0.125, **td).sum(), q)
    assert one.shape == q.shape and torch.isfinite(one.float()).all()


def test_without_a_table_the_other_gradients_have_the_same_bits():
    import paper_2501_06480_amd as fwa
    for L, H in ((300, 2), (2100, 20)):  # waves that share out keys, and rows
        x, t, _ = make(BF16, 1, L, L, H, 2, 64)
        xd, td = device(x), device(t)
        o, stats = fwa.fwa_sequence_forward(xd["q"], xd["k"], xd["v"], H, 0.125, want_stats=True, **td)
        a = fwa.fwa_sequence_backward(xd["q"], xd["k"], xd["v"], o, stats, xd["d_o"], H, 0.125, want_dtable=True, **td)
        b = fwa.fwa_sequence_backward(xd["q"], xd["k"], xd["v"], o, stats, xd["d_o"], H, 0.125, want_dtable=False, **td)
        for y, z in zip(a[:3], b[:3]):
            assert torch.equal(y, z), L


@pytest.mark.parametrize("dtype,N,L,H,KV,d,causal", [(BF16, 2, 700, 40, 40, 64, False), (F16, 1, 900, 40, 8, 128, True), (F32, 1, 520, 70, 70, 32, True),
                                                     (BF16, 3, 450, 24, 24, 32, False), (F32, 1, 300, 90, 30, 128, False)])
def test_many_heads_take_the_rows_form(dtype, N, L, H, KV, d, causal):
    """More than a workgroup of 128 rows for each CU: checked for two heads of the first and the last sequence, of one group each."""
    import paper_2501_06480_amd as fwa
    x, t, g = make(dtype, N, L, L, H, KV, d)
    t["causal"] = causal
    t["k_lengths"] = t["q_lengths"] = torch.randint(L // 2, L + 1, (N,), generator=g, dtype=torch.int32)
    xd, td = device(x), device(t)
    o, stats = fwa.fwa_sequence_forward(xd["q"], xd["k"], xd["v"], H, d ** -0.5, want_stats=True, **td)
    dq, dk, dv, dt = fwa.fwa_sequence_backward(xd["q"], xd["k"], xd["v"], o, stats, xd["d_o"], H, d ** -0.5, want_dtable=True, **td)
    G = H // KV
    for n, kv in ((0, 0), (N - 1, KV - 1)):
        hs = slice(kv * G * d, (kv + 1) * G * d)
        ks = slice(kv * d, (kv + 1) * d)
        part = {"q": x["q"][n:n + 1, :, hs], "k": x["k"][n:n + 1, :, ks], "v": x["v"][n:n + 1, :, ks], "d_o": x["d_o"][n:n + 1, :, hs]}
        want = ref.attention(part["q"], part["k"], part["v"], G, d ** -0.5, t["table"][kv * G:(kv + 1) * G], t["buckets"], t["q_lengths"][n:n + 1],
                             t["k_lengths"][n:n + 1], None, causal, part["d_o"])
        for got, name, at in ((o, "o", hs), (dq, "dq", hs), (dk, "dk", ks), (dv, "dv", ks)):
            ref.check(got[n:n + 1, :, at], want[name], want[name + "_tol"], f"{name} {n} {kv}")
        if N == 1:
            ref.check(dt[kv * G:(kv + 1) * G], want["dtable"], want["dtable_tol"], f"dtable {kv}")


def test_a_prompt_and_its_new_tokens_one_by_one():
    """The output of a causal sequence, and the same from a prompt and single tokens against a cache that grows: one bias, one set of positions."""
    import paper_2501_06480_amd as fwa
    N, L, H, KV, d, room = 2, 90, 4, 2, 64, 128
    x, t, _ = make(F32, N, L, L, H, KV, d)
    xd, td = device(x), device(t)
    whole = fwa.fwa_sequence_forward(xd["q"], xd["k"], xd["v"], H, 0.125, causal=True, **td)
    cache = torch.full((2, N, room, KV * d), float("nan"), device="cuda")  # behind the lengths nothing is read
    cache[0, :, :70], cache[1, :, :70] = xd["k"][:, :70], xd["v"][:, :70]
    lengths = torch.full((N,), 70, dtype=torch.int32, device="cuda")
    parts = [fwa.fwa_sequence_forward(xd["q"][:, :70].contiguous(), cache[0], cache[1], H, 0.125, k_lengths=lengths, causal=True, **td)]
    for i in range(70, L):
        cache[0, :, i], cache[1, :, i] = xd["k"][:, i], xd["v"][:, i]
        start = lengths.clone()
        lengths += 1
        parts.append(fwa.fwa_sequence_forward(xd["q"][:, i:i + 1].contiguous(), cache[0], cache[1], H, 0.125, k_lengths=lengths, q_start=start, **td))
    # the same sums in another order: fp32 rounding
    assert float((torch.cat(parts, 1) - whole).abs().max()) <= 64 * ref.U32 * float(x["v"].abs().max()) * 8


def test_a_cache_whose_rows_pass_4_gib():
    """Keys 128 KiB apart: offsets inside one sequence pass 32 bits; the same bits as from a dense copy."""
    import paper_2501_06480_amd as fwa
    L, ld, d, H = 36000, 65536, 64, 1
    free = torch.cuda.mem_get_info()[0]
    if free < 14 << 30:
        pytest.skip("needs 14 GB of device memory")
    wide = torch.zeros(1, L, ld, dtype=BF16, device="cuda")
    g = torch.Generator().manual_seed(3)
    k, v = (torch.randn(1, L, d, generator=g).bfloat16().cuda() for _ in range(2))
    wide[..., :d], wide[..., d:2 * d] = k, v
    x, t, _ = make(BF16, 1, 150, 1, H, H, d)
    td = device(t)
    q, d_o = x["q"].cuda(), x["d_o"].cuda()
    start = torch.tensor([L - 150], dtype=torch.int32, device="cuda")
    results = []
    for kk, vv in ((k, v), (wide[..., :d], wide[..., d:2 * d])):
        o, stats = fwa.fwa_sequence_forward(q, kk, vv, H, 0.125, want_stats=True, q_start=start, causal=True, **td)
        out = None
        if kk is not k:
            room = torch.zeros(1, L, ld, dtype=BF16, device="cuda")
            out = (torch.empty_like(q), room[..., :d], room[..., d:2 * d])
        results.append((o,) + fwa.fwa_sequence_backward(q, kk, vv, o, stats, d_o, H, 0.125, q_start=start, causal=True, want_dtable=True, out=out, **td))
    for a, b in zip(*results):
        assert torch.equal(a, b)


def test_calls_on_another_stream():
    import paper_2501_06480_amd as fwa
    x, t, _ = make(BF16, 2, 300, 300, 4, 4, 64)
    xd, td = device(x), device(t)
    o, stats = fwa.fwa_sequence_forward(xd["q"], xd["k"], xd["v"], 4, 0.125, want_stats=True, **td)
    want = fwa.fwa_sequence_backward(xd["q"], xd["k"], xd["v"], o, stats, xd["d_o"], 4, 0.125, want_dtable=True, **td)
    bias = fwa.fwa_bucket_gather(td["table"], td["buckets"], 60)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    o2, s2 = fwa.fwa_sequence_forward(xd["q"], xd["k"], xd["v"], 4, 0.125, want_stats=True, stream=side, **td)
    got = fwa.fwa_sequence_backward(xd["q"], xd["k"], xd["v"], o2, s2, xd["d_o"], 4, 0.125, want_dtable=True, stream=side, **td)
    bias2 = fwa.fwa_bucket_gather(td["table"], td["buckets"], 60, stream=side)
    dt2 = fwa.fwa_bucket_scatter(bias2, td["buckets"], 16, stream=side)
    side.synchronize()
    assert torch.equal(o, o2) and torch.equal(bias, bias2)
    assert torch.equal(dt2, fwa.fwa_bucket_scatter(bias, td["buckets"], 16))
    for a, b in zip(want, got):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype,N,Lq,Lk,H,KV,d", [(BF16, 2, 260, 260, 4, 2, 64), (F32, 1, 1, 2000, 8, 8, 32)])
def test_captured_calls_replay_as_they_run(dtype, N, Lq, Lk, H, KV, d):
    """Forward, backward, gather and scatter in one graph; inputs, lengths and table change between the replays."""
    import paper_2501_06480_amd as fwa
    x, t, g = make(dtype, N, Lq, Lk, H, KV, d)
    t["k_lengths"] = torch.full((N,), Lk, dtype=torch.int32)
    xd, td = device(x), device(t)

    def run(stream=None):
        o, stats = fwa.fwa_sequence_forward(xd["q"], xd["k"], xd["v"], H, 0.2, want_stats=True, stream=stream, **td)
        grads = fwa.fwa_sequence_backward(xd["q"], xd["k"], xd["v"], o, stats, xd["d_o"], H, 0.2, want_dtable=True, stream=stream, **td)
        bias = fwa.fwa_bucket_gather(td["table"], td["buckets"], 100, stream=stream)
        return (o,) + grads + (bias, fwa.fwa_bucket_scatter(bias, td["buckets"], 16, stream=stream))

    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        captured = run(torch.cuda.current_stream())
    for seed in range(3):
        for n in ("q", "k", "v", "d_o"):
            xd[n].copy_(torch.randn(x[n].shape, generator=g).to(dtype))
        td["table"].copy_(torch.randn(t["table"].shape, generator=g))
        td["k_lengths"].copy_(torch.randint(1, Lk + 1, (N,), generator=g, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        got = [y.clone() for y in captured]
        for y in captured:
            y.fill_(7.0)
        for a, b in zip(got, run()):
            assert torch.equal(a, b), seed


def test_refusals_of_the_bindings():
    import paper_2501_06480_amd as fwa
    x, t, _ = make(BF16, 2, 40, 50, 4, 2, 64)
    xd, td = device(x), device(t)
    q, k, v = xd["q"], xd["k"], xd["v"]
    f = lambda *a, **kw: fwa.fwa_sequence_forward(*a, 4, 0.1, **kw)  # noqa: E731
    for bad in (lambda: f(q, k, v[:, :49]), lambda: f(q, k.float(), v), lambda: f(q, k[..., :100], v[..., :100]), lambda: f(q[0], k, v),
                lambda: f(q, k, v, table=td["table"]), lambda: f(q, k, v, table=td["table"][:2], buckets=td["buckets"]),
                lambda: f(q, k, v, table=td["table"], buckets=td["buckets"].long()), lambda: f(q, k, v, table=td["table"], buckets=td["buckets"][:-1]),
                lambda: f(q, k, v, k_lengths=torch.ones(2, dtype=torch.int64, device="cuda")), lambda: f(q, k, v, q_start=torch.ones(3, dtype=torch.int32, device="cuda")),
                lambda: f(q[:, ::2], k, v, out=torch.empty_like(q)), lambda: f(q.transpose(0, 1), k, v),
                lambda: fwa.fwa_sequence_forward(q, k, v, 3, 0.1),
                lambda: fwa.fwa_bucket_gather(td["table"], td["buckets"], 5, 5, out=torch.empty(4, 5, 6, device="cuda")),
                lambda: fwa.fwa_bucket_scatter(td["table"], td["buckets"], 8)):
        with pytest.raises((TypeError, ValueError)):
            bad()
    with pytest.raises(TypeError):
        f(q, k, v, k_lengths=torch.ones(2, dtype=torch.int32))
    with pytest.raises(TypeError):
        f(q, k, v, table=td["table"].double(), buckets=td["buckets"])
    with pytest.raises(fwa.FwaError):  # head width 48
        fwa.fwa_sequence_forward(q[..., :192].contiguous(), k[..., :96].contiguous(), v[..., :96].contiguous(), 4, 0.1)
    o, stats = f(q, k, v, want_stats=True)
    with pytest.raises(fwa.FwaError):  # an output on top of an input
        f(q, k, v, out=q)
    with pytest.raises(ValueError):
        fwa.fwa_sequence_backward(q, k, v, o, stats[:, :2], xd["d_o"], 4, 0.1)
    with pytest.raises(ValueError):
        fwa.fwa_sequence_backward(q, k, v, o, stats, xd["d_o"], 4, 0.1, want_dtable=True)
    with pytest.raises(fwa.FwaError):
        fwa.fwa_sequence_backward(q, k, v, o, stats, xd["d_o"], 4, 0.1, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
