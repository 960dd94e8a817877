"""Append of new tokens to a paged cache against 64 bits (tests/page_reference.py): every row of the cache is looked at, so one that should have been left
alone and was not is found."""
import pytest
import torch

import page_reference as ref

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32


def make(dtype, news, lengths, H, KV, d, size, extra=2, by_heads=False, sections=None, spare=(0, 0), seed=0, positions=False):
    """`spare`: rows in front of the first sequence and behind the last"""
    from paper_2501_06480_amd import binding
    g = torch.Generator().manual_seed(seed + sum(news) + 7 * d + size)
    N, T = len(news), sum(news) + sum(spare)
    width = max([1] + [-(-(n + l) // size) for n, l in zip(news, lengths)])
    pages = N * width + extra
    x = {"fused": torch.randn(T, (H + 2 * KV) * d, generator=g).to(dtype)}
    shape = (pages, KV, size, d) if by_heads else (pages, size, KV, d)
    for n in ("k_pages", "v_pages"):
        x[n] = torch.randn(shape, generator=g).to(dtype)
    x["page_table"] = torch.randperm(pages, generator=g)[:N * width].to(torch.int32).view(N, width)
    x["offsets"] = torch.tensor([spare[0] + sum(news[:i]) for i in range(N + 1)], dtype=torch.int32)
    x["lengths"] = torch.tensor(lengths, dtype=torch.int32)
    if sections is not None:
        x["frequencies"], x["axis_of"] = binding.rotary_frequencies(sections)
        if positions or len(sections) > 1:
            x["positions"] = torch.randint(0, 3000, (T, len(sections)), generator=g, dtype=torch.int32)
    return x, g


def device(x, by_heads=False):
    y = {n: t.cuda() for n, t in x.items()}
    if by_heads:
        for n in ("k_pages", "v_pages"):
            y[n] = y[n].transpose(1, 2)
    return y


def split(fused, H, KV, d):
    return fused[:, :H * d], fused[:, H * d:(H + KV) * d], fused[:, (H + KV) * d:]


def call(y, H, KV, d, with_q=True, interleaved=False, **kw):
    import paper_2501_06480_amd as fwa
    q, k, v = split(y["fused"], H, KV, d)
    return fwa.fwa_page_append(k, v, y["k_pages"], y["v_pages"], y["page_table"], y["offsets"], y["lengths"], y.get("frequencies"), y.get("positions"),
                               y.get("axis_of"), interleaved, q=q if with_q else None, **kw)


def expected(x, H, KV, d, by_heads=False, interleaved=False):
    """k and v pools, queries, each with its bounds; rows of the queries that are written"""
    q, k, v = split(x["fused"], H, KV, d)
    T = q.shape[0]
    rows = torch.zeros(T, dtype=torch.bool)
    places = torch.zeros(T, 1, dtype=torch.int32)
    for n, a, count, length in ref.new_tokens(x["offsets"], x["lengths"], T):
        rows[a:a + count] = True
        places[a:a + count, 0] = torch.arange(length, length + count)
    at = x.get("positions", places)
    pools = [x[n].transpose(1, 2) if by_heads else x[n] for n in ("k_pages", "v_pages")]
    if "frequencies" in x:
        (kr, k_tol), (qr, q_tol) = (ref.rotate(t, h, at, x["frequencies"], x.get("axis_of"), interleaved) for t, h in ((k, KV), (q, H)))
    else:
        kr, qr = k.double(), q.double()
        k_tol, q_tol = torch.zeros_like(kr), torch.zeros_like(qr)
    tables = (x["page_table"], x["offsets"], x["lengths"])
    kp, written = ref.append(kr, pools[0].double(), *tables)
    kt, _ = ref.append(k_tol, torch.zeros(pools[0].shape, dtype=torch.float64), *tables)
    vp, _ = ref.append(v.double(), pools[1].double(), *tables)
    return kp, kt, vp, qr, q_tol, rows, written


def compare(x, H, KV, d, what, by_heads=False, interleaved=False, with_q=True):
    want = expected(x, H, KV, d, by_heads, interleaved)
    y = device(x, by_heads)
    q_out = torch.full((x["fused"].shape[0], H * d), 7.0, dtype=x["fused"].dtype, device="cuda") if with_q else None
    got = call(y, H, KV, d, with_q, interleaved, q_out=q_out)
    kp, kt, vp, qr, q_tol, rows, _ = want
    ref.check(y["k_pages"], kp, kt, what + " keys")
    assert torch.equal(y["v_pages"].cpu().double(), vp), what + " values"
    assert torch.equal(y["fused"].cpu(), x["fused"])
    if with_q:
        assert got is q_out
        ref.check(got.cpu()[rows], qr[rows], q_tol[rows], what + " queries")
        assert bool((got.cpu()[~rows] == 7.0).all())
    else:
        assert got is None
    return y, got


CASES = [  # dtype, new tokens, older ones, H, KV, d, page, by_heads, sections, interleaved, with_q
    (BF16, [1] * 5, [0, 15, 16, 100, 31], 8, 2, 128, 16, False, (64,), False, True),
    (F16, [130], [7], 4, 4, 64, 32, True, (10, 11, 11), False, True),
    (F32, [3, 0, 17, 1, 0, 40], [5, 9, 0, 47, 2, 90], 3, 1, 32, 48, False, (16,), True, True),
    (BF16, [33, 65], [0, 0], 12, 12, 64, 64, True, (32,), True, False),
    (F16, [50, 1], [100, 3], 2, 1, 128, 16, False, (20, 20), False, True),   # vectors of 4
    (BF16, [50, 1], [100, 3], 2, 1, 128, 16, False, (13, 8), True, True),     # single elements
    (F32, [9, 9], [20, 20], 2, 2, 64, 256, False, None, False, True),         # no rotation
    (BF16, [1], [0], 1, 1, 32, 16, False, (8,), False, True),
    (F32, [70], [1000], 4, 2, 128, 16, True, (64,), False, True),
]


@pytest.mark.parametrize("dtype,news,lengths,H,KV,d,size,by_heads,sections,interleaved,with_q", CASES)
def test_append(dtype, news, lengths, H, KV, d, size, by_heads, sections, interleaved, with_q):
    x, _ = make(dtype, news, lengths, H, KV, d, size, by_heads=by_heads, sections=sections)
    compare(x, H, KV, d, f"{dtype} {news} {d}", by_heads, interleaved, with_q)


def test_pages_that_are_none_and_places_without_a_page():
    """Entries outside the pages, lengths below zero and beyond the table, rows outside the offsets: nothing is stored, queries are rotated all the same."""
    x, _ = make(BF16, [20, 20, 20, 5, 5], [0, 30, 10, 3, 0], 2, 2, 64, 16, sections=(32,), spare=(3, 9))
    x["page_table"][0, 1] = -1
    x["page_table"][1, 2] = x["k_pages"].shape[0]
    x["page_table"][1, 3:] = 0x7fffffff
    x["page_table"][2, 0] = -0x80000000
    x["lengths"][3] = x["page_table"].shape[1] * 16 - 2  # three of five beyond the table
    x["lengths"][4] = -5                                  # counts as 0
    compare(x, 2, 2, 64, "no pages")
    x["lengths"][0] = 0x7fffffff  # cut off; the position of the rotation with it
    y = device(x)
    before = y["k_pages"].clone()
    call(y, 2, 2, 64)
    x["lengths"][0] = 1 << 29
    _, _, _, _, _, _, written = expected(x, 2, 2, 64)
    assert torch.equal(y["k_pages"].cpu()[~written], before.cpu()[~written])


def test_offsets_of_all_kinds():
    """Empty sequences at both ends and between, offsets beyond the rows; more sequences than a workgroup has threads."""
    x, g = make(F16, [0, 0, 4, 0, 0, 7, 0], [1, 2, 3, 4, 5, 6, 7], 1, 1, 32, 16, sections=(16,))
    compare(x, 1, 1, 32, "empty")
    x["offsets"][-1] += 5  # beyond the rows
    x["offsets"][0] -= 3
    y = device(x)
    call(y, 1, 1, 32)
    torch.cuda.synchronize()
    news = torch.randint(0, 3, (700,), generator=g).tolist()
    lengths = torch.randint(0, 30, (700,), generator=g).tolist()
    x, _ = make(BF16, news, lengths, 2, 1, 32, 16, sections=(16,))
    compare(x, 2, 1, 32, "many")


def test_cache_of_one_buffer_and_queries_in_place():
    """Keys and values of one buffer [pages, 2, page, kv, d], and [pages, page, 2, kv, d]; queries rotated where they stand in the fused projection."""
    H, KV, d, size = 4, 2, 64, 16
    x, g = make(BF16, [5, 20], [30, 2], H, KV, d, size, sections=(32,))
    kp, kt, vp, qr, q_tol, rows, _ = expected(x, H, KV, d)
    y = device(x)
    for dim in (1, 2):
        both = torch.stack([x["k_pages"], x["v_pages"]], dim).cuda()
        y["k_pages"], y["v_pages"] = both.unbind(dim)
        fused = x["fused"].cuda()
        q = fused[:, :H * d]
        y["fused"] = fused
        got = call(y, H, KV, d, q_out=q)
        assert got.data_ptr() == fused.data_ptr()
        ref.check(fused[:, :H * d], qr, q_tol, "in place")
        assert torch.equal(fused[:, H * d:].cpu(), x["fused"][:, H * d:])
        ref.check(y["k_pages"], kp, kt, "keys")
        assert torch.equal(y["v_pages"].cpu().double(), vp)


def test_streams_and_graphs():
    H, KV, d = 4, 2, 64
    x, g = make(BF16, [3, 4, 5], [20, 0, 9], H, KV, d, 16, sections=(16, 16))
    y = device(x)
    clean = [y["k_pages"].clone(), y["v_pages"].clone()]
    want_q = call(y, H, KV, d)
    want = [y["k_pages"].clone(), y["v_pages"].clone()]
    y["k_pages"].copy_(clean[0]), y["v_pages"].copy_(clean[1])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got_q = call(y, H, KV, d, stream=side)
    side.synchronize()
    assert torch.equal(got_q, want_q) and torch.equal(y["k_pages"], want[0]) and torch.equal(y["v_pages"], want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        out = call(y, H, KV, d, stream=torch.cuda.current_stream())
    for _ in range(3):
        y["fused"].copy_(torch.randn(x["fused"].shape, generator=g).to(BF16))
        y["lengths"].copy_(torch.randint(0, 20, (3,), generator=g, dtype=torch.int32))
        y["offsets"][1:3] += torch.tensor([-1, 1], dtype=torch.int32, device="cuda")
        y["k_pages"].copy_(clean[0]), y["v_pages"].copy_(clean[1])
        graph.replay()
        torch.cuda.synchronize()
        got = [out.clone(), y["k_pages"].clone(), y["v_pages"].clone()]
        out.fill_(7.0)
        y["k_pages"].copy_(clean[0]), y["v_pages"].copy_(clean[1])
        q = call(y, H, KV, d)
        for a, b in zip(got, (q, y["k_pages"], y["v_pages"])):
            assert torch.equal(a, b)


def test_refusals():
    import paper_2501_06480_amd as fwa
    H, KV, d = 2, 2, 64
    x, _ = make(BF16, [3, 4], [20, 0], H, KV, d, 16, sections=(16, 16))
    y = device(x)
    q, k, v = split(y["fused"], H, KV, d)
    f = lambda k=k, v=v, **kw: fwa.fwa_page_append(k, v, *(kw.pop(n, y[n]) for n in ("k_pages", "v_pages", "page_table", "offsets", "lengths")), **kw)  # noqa: E731
    for bad in (lambda: f(k=k[:, :64]), lambda: f(v=v[:5]), lambda: f(k=k.float()), lambda: f(k_pages=y["k_pages"][:-1]), lambda: f(v_pages=y["v_pages"].float()),
                lambda: f(v_pages=y["v_pages"].transpose(1, 2).contiguous().transpose(1, 2)), lambda: f(page_table=y["page_table"].long()),
                lambda: f(page_table=y["page_table"][:1]), lambda: f(offsets=y["offsets"][:2]), lambda: f(lengths=y["lengths"][:1]),
                lambda: f(positions=y["positions"]), lambda: f(frequencies=y["frequencies"], positions=y["positions"][:2]),
                lambda: f(frequencies=y["frequencies"], axis_of=y["axis_of"][:3]), lambda: f(q_out=torch.empty_like(q)), lambda: f(q=q[:5]),
                lambda: f(q=q, q_out=torch.empty(7, 64, dtype=BF16, device="cuda")), lambda: f(lengths=y["lengths"].cpu()), lambda: f(k=k[None], v=v[None]),
                lambda: f(k_pages=y["k_pages"][..., ::2], v_pages=y["v_pages"][..., ::2])):
        with pytest.raises((TypeError, ValueError)):
            bad()
    with pytest.raises(fwa.FwaError):  # keys on top of values
        f(v_pages=y["k_pages"])
    with pytest.raises(fwa.FwaError):  # a cache that reaches an element twice
        f(k_pages=y["k_pages"][:1].expand(4, -1, -1, -1), v_pages=y["v_pages"][:1].expand(4, -1, -1, -1))
    with pytest.raises(fwa.FwaError):  # pages of 8 rows
        f(k_pages=y["k_pages"][:, :8].contiguous(), v_pages=y["v_pages"][:, :8].contiguous())
