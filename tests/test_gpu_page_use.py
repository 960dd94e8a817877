"""The operators on a paged cache as programs use them, one behind the other: prompts in chunks and single tokens against the attention of whole sequences, long caches whose
keys all workgroups share out, captured steps that replay with other lengths, streams, caches beyond 4 GiB."""
import pytest
import torch

import page_reference as ref
from test_gpu_page_forward import BF16, F16, F32, compare, device, make, run

pytestmark = pytest.mark.gpu


def shared_out(dtype, news, lengths, H, KV, d, size, width, seed=0):
    """A table far wider than the sequences need, its other entries no pages: as much room as a server gives each of its sequences"""
    x, g = make(dtype, news, lengths, H, KV, d, size, seed=seed)
    wide = torch.full((len(news), width), -1, dtype=torch.int32)
    wide[:, :x["page_table"].shape[1]] = x["page_table"]
    x["page_table"] = wide
    return x, g


@pytest.mark.parametrize("dtype,d", [(BF16, 64), (F32, 32), (F16, 128), (BF16, 32), (F32, 128), (F32, 64)])
@pytest.mark.parametrize("H,KV", [(4, 4), (8, 1), (6, 3)])
def test_all_keys_shared_out(dtype, d, H, KV):
    """Lengths from none to thousands beside each other, sequences without a new token at both ends and between; rooms so wide that the even share is taken."""
    import paper_2501_06480_amd as fwa
    news = [0, 1, 1, 0, 1, 2, 1, 1, 0]
    lengths = [500, 2900, 0, 77, 16, 1213, 31, 600, 3]
    x, _ = shared_out(dtype, news, lengths, H, KV, d, 16, 8192)
    code = {F32: 0, BF16: 1, F16: 2}[dtype]
    need = fwa.fwa_page_forward_workspace_bytes(7, 9, H, KV, d, 16, 8192, 2, code)
    assert need > 512 // KV * KV * 2 * 32 * d * 4  # two blocks of rows for each of all workgroups
    compare(x, H, d ** -0.5, f"{dtype} {d} {H}/{KV}", most_new=2)
    x["page_table"][1, 3:9] = 0x7fffffff
    x["page_table"][4] = -1
    o, stats = compare(x, H, d ** -0.5, f"{dtype} {d} {H}/{KV} holes", most_new=2)
    again, more = run(device(x), H, d ** -0.5, most_new=2)
    assert torch.equal(again, o) and torch.equal(more, stats)


def test_more_sequences_than_lanes_shared_out():
    g = torch.Generator().manual_seed(9)
    lengths = torch.randint(0, 700, (150,), generator=g).tolist()
    news = [1 if i % 5 else 0 for i in range(150)]
    x, _ = shared_out(BF16, news, lengths, 2, 1, 64, 16, 4096)
    compare(x, 2, 0.125, "150 sequences", most_new=1)
    x, _ = shared_out(F16, [1], [3000], 4, 1, 128, 16, 30000)  # one sequence, all workgroups
    compare(x, 4, 0.1, "one sequence", most_new=1)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype,H,KV,d,news,width,most", [(BF16, 4, 2, 64, [1, 1, 0, 1], 200, 1), (F16, 8, 1, 128, [3, 3, 3], 300, 3), (BF16, 4, 2, 64, [1, 2, 0, 1], 8192, 2),
                                                          (F32, 2, 2, 32, [40, 40], 200, 40), (BF16, 4, 1, 128, [1, 150, 60, 0], 200, None)])
def test_the_workspace_ends_where_the_query_says(dtype, H, KV, d, news, width, most, causal):
    """Each way of sharing out keys, in a workspace of not a byte more than asked for, with a mark behind it."""
    import paper_2501_06480_amd as fwa
    T, N, code = sum(news), len(news), {F32: 0, BF16: 1, F16: 2}[dtype]
    x, _ = shared_out(dtype, news, [700, 33, 5, 1500][:N], H, KV, d, 16, width)
    need = fwa.fwa_page_forward_workspace_bytes(T, N, H, KV, d, 16, width, T if most is None else most, code)
    assert need > 0
    whole = torch.full((need + 4096,), 0xa5, dtype=torch.uint8, device="cuda")
    y = device(x)
    o, stats = run(y, H, 0.1, most_new=most, causal=causal, workspace=whole[:need])
    assert bool((whole[need:] == 0xa5).all())
    again, more = run(y, H, 0.1, most_new=most, causal=causal)
    assert torch.equal(o, again) and torch.equal(stats, more)
    with pytest.raises(fwa.FwaError):
        run(y, H, 0.1, most_new=most, causal=causal, workspace=whole[:need - 1])


def cache(pages, size, KV, d, dtype):
    return [torch.full((pages, size, KV, d), float("nan"), dtype=dtype, device="cuda") for _ in range(2)]


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_a_prompt_in_chunks_and_its_new_tokens(dtype):
    """Two sequences side by side, their prompts in chunks of different lengths and single tokens, in pages handed out as they are needed: the outputs of the
    rotation and the attention of whole sequences."""
    import paper_2501_06480_amd as fwa
    N, H, KV, d, size, L = 2, 4, 2, 64, 16, 150
    g = torch.Generator().manual_seed(4)
    q, k, v = (torch.randn(N, L, h * d, generator=g).to(dtype).cuda() for h in (H, KV, KV))
    f, axis = fwa.rotary_frequencies((32,), device="cuda")
    positions = torch.arange(L, dtype=torch.int32, device="cuda")[:, None]
    rq, rk = (fwa.fwa_rotary(t, h, positions, f, axis) for t, h in ((q, H), (k, KV)))
    whole = fwa.fwa_sequence_forward(rq, rk, v, H, 0.125, causal=True)
    pages = 24
    k_pages, v_pages = cache(pages, size, KV, d, dtype)  # rows that no token has hold NaN
    table = torch.full((N, 10), -1, dtype=torch.int32, device="cuda")
    free = torch.randperm(pages, generator=g).tolist()
    held = [0, 0]
    got = [[], []]
    while min(held) < L:
        news = [min(L - h, int(torch.randint(0, 50, (1,), generator=g)) if h < 120 else 1) for h in held]
        for n in range(N):
            for index in range(-(-held[n] // size), -(-(held[n] + news[n]) // size)):
                table[n, index] = free.pop()
        rows = [(n, i) for n in range(N) for i in range(held[n], held[n] + news[n])]
        if rows:
            at = tuple(torch.tensor(t, device="cuda") for t in zip(*rows))
            tables = (table, torch.tensor([0, news[0], sum(news)], dtype=torch.int32, device="cuda"), torch.tensor(held, dtype=torch.int32, device="cuda"))
            fused = torch.cat([t[at] for t in (q, k, v)], 1)
            pq, pk, pv = fused[:, :H * d], fused[:, H * d:(H + KV) * d], fused[:, (H + KV) * d:]
            turned = fwa.fwa_page_append(pk, pv, k_pages, v_pages, *tables, frequencies=f, axis_of=axis, q=pq)
            assert torch.equal(turned, rq[at])  # the same rotation, bit for bit
            o = fwa.fwa_page_forward(turned, k_pages, v_pages, *tables, H, 0.125, most_new=max(news))
            for n in range(N):
                got[n].append(o[sum(news[:n]):sum(news[:n + 1])])
        held = [h + x for h, x in zip(held, news)]
    # each side: a score is off by (d + 8) half steps of the sum of its magnitudes, its exponent and the sums by a few more, twice that of the output; 16-bit data: P and the output
    # are rounded, half a step each
    most = 0.125 * float((rq.float().view(N, L, H, d).abs().sum(-1).amax() * rk.float().abs().max()))
    bound = 2 * (2 * ((d + 8) * most + 100) * ref.U32 + (0 if dtype == F32 else 2 * ref.U[dtype])) * float(v.abs().max())
    assert float((torch.stack([torch.cat(t) for t in got]).float() - whole.float()).abs().max()) <= bound


def test_captured_steps_replay_with_other_lengths():
    """A step of a server in one graph: append, attention, and the lengths one further; pages come along between the replays.  Another graph with the same workspace, one
    behind the other."""
    import paper_2501_06480_amd as fwa
    N, H, KV, d, size, width = 3, 8, 2, 64, 16, 300
    g = torch.Generator().manual_seed(6)
    f, axis = fwa.rotary_frequencies((16, 16), device="cuda")
    fused = torch.randn(N, (H + 2 * KV) * d, generator=g).bfloat16().cuda()
    q, k, v = fused[:, :H * d], fused[:, H * d:(H + KV) * d], fused[:, (H + KV) * d:]
    positions = torch.randint(0, 999, (N, 2), generator=g, dtype=torch.int32).cuda()
    k_pages, v_pages = (torch.randn(60, size, KV, d, generator=g).bfloat16().cuda() for _ in range(2))
    table = torch.full((N, width), -1, dtype=torch.int32, device="cuda")
    table[:, :20] = torch.randperm(60, generator=g).to(torch.int32).view(N, 20)
    offsets = torch.arange(N + 1, dtype=torch.int32, device="cuda")
    lengths = torch.tensor([0, 130, 40], dtype=torch.int32, device="cuda")
    ws = torch.empty(fwa.fwa_page_forward_workspace_bytes(N, N, H, KV, d, size, width, 1, 1), dtype=torch.uint8, device="cuda")
    assert ws.numel() > 0
    turned, out, other = (torch.empty(N, H * d, dtype=BF16, device="cuda") for _ in range(3))

    def step(o, stream=None):
        tables = (k_pages, v_pages, table, offsets, lengths)
        fwa.fwa_page_append(k, v, *tables, frequencies=f, positions=positions, axis_of=axis, q=q, q_out=turned, stream=stream)
        fwa.fwa_page_forward(turned, *tables, H, 0.125, most_new=1, out=o, workspace=ws, stream=stream)

    step(out)
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for graph, o in zip(graphs, (out, other)):
        with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
            step(o, torch.cuda.current_stream())
            lengths.add_(1)
    lengths.copy_(torch.tensor([0, 130, 40]))
    clean = [k_pages.clone(), v_pages.clone()]
    seen = []
    for i in range(4):
        fused.copy_(torch.randn(fused.shape, generator=g))
        seen.append(fused.clone())
        graphs[i % 2].replay()
        torch.cuda.synchronize()
        got = (out, other)[i % 2].clone()
        after = [k_pages.clone(), v_pages.clone(), lengths.clone()]
        (out, other)[i % 2].fill_(7.0)
        ws.fill_(0xff)  # what it holds does not matter
        k_pages.copy_(clean[0]), v_pages.copy_(clean[1])
        lengths.sub_(1)
        want = torch.empty_like(out)
        step(want)
        lengths.add_(1)
        assert torch.equal(got, want), i
        assert torch.equal(after[0], k_pages) and torch.equal(after[1], v_pages) and after[2].tolist() == [i + 1, 131 + i, 41 + i]
        clean = [k_pages.clone(), v_pages.clone()]


def test_calls_on_another_stream():
    for dtype, news, lengths, wide in ((BF16, [1, 1, 1], [900, 20, 300], 0), (F16, [1, 80, 3], [90, 20, 300], 0), (F32, [1, 1], [800, 9], 4000)):
        x, _ = make(dtype, news, lengths, 4, 2, 64, 16, wider=wide) if not wide else shared_out(dtype, news, lengths, 4, 2, 64, 16, wide)
        y = device(x)
        want, stats = run(y, 4, 0.125, most_new=max(news))
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        got, more = run(y, 4, 0.125, most_new=max(news), stream=side)
        side.synchronize()
        assert torch.equal(got, want) and torch.equal(more, stats)


def test_pages_behind_4_gib():
    """Pages 96 MiB apart in a buffer of 9 GB: append and attention, the same bits as in a dense cache."""
    import paper_2501_06480_amd as fwa
    if torch.cuda.mem_get_info()[0] < 14 << 30:
        pytest.skip("needs 14 GB of device memory")
    H, KV, d, size, pages, apart = 4, 2, 64, 32, 90, 48 << 20
    room = torch.zeros(pages * apart, dtype=BF16, device="cuda")
    far = [torch.as_strided(room, (pages, size, KV, d), (apart, KV * d, d, 1), i * size * KV * d) for i in range(2)]
    near = [torch.zeros(pages, size, KV, d, dtype=BF16, device="cuda") for _ in range(2)]
    g = torch.Generator().manual_seed(8)
    table = torch.randperm(pages, generator=g).to(torch.int32).view(2, 45).cuda()
    f, axis = fwa.rotary_frequencies((32,), device="cuda")
    lengths, held = torch.zeros(2, dtype=torch.int32, device="cuda"), [0, 0]
    for news in ([1000, 700], [1, 1], [300, 1]):
        T = sum(news)
        fused = torch.randn(T, (H + 2 * KV) * d, generator=g).bfloat16().cuda()
        offsets = torch.tensor([0, news[0], T], dtype=torch.int32, device="cuda")
        results = []
        for k_pages, v_pages in (near, far):
            q = fwa.fwa_page_append(fused[:, H * d:(H + KV) * d], fused[:, (H + KV) * d:], k_pages, v_pages, table, offsets, lengths, frequencies=f, axis_of=axis, q=fused[:, :H * d])
            results.append(fwa.fwa_page_forward(q, k_pages, v_pages, table, offsets, lengths, H, 0.125, most_new=max(news)))
        assert torch.equal(results[0], results[1])
        lengths += torch.tensor(news, dtype=torch.int32, device="cuda")
    for a, b in zip(near, far):
        assert torch.equal(a, b)
    assert int((room != 0).sum()) == sum(int((t != 0).sum()) for t in near)
