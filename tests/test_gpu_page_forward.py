"""Attention over a paged cache against 64 bits (tests/page_reference.py): single tokens, chunks and whole prompts, alone and mixed, pages that end inside
a tile, both layouts, pages that are none, rows of no sequence, rows without a key."""
import math

import pytest
import torch

import page_reference as ref

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32


def make(dtype, news, lengths, H, KV, d, size, by_heads=False, spare=(0, 0), extra=2, seed=0, wider=0):
    g = torch.Generator().manual_seed(seed + sum(news) + 7 * d + size + H)
    N, T = len(news), sum(news) + sum(spare)
    width = max([1] + [-(-(n + l) // size) for n, l in zip(news, lengths)]) + wider
    pages = N * width + extra
    x = {"q": torch.randn(T, H * d, generator=g).to(dtype)}
    for n in ("k_pages", "v_pages"):
        x[n] = torch.randn(pages, size, KV, d, generator=g).to(dtype)
    x["page_table"] = torch.randperm(pages, generator=g)[:N * width].to(torch.int32).view(N, width)
    x["offsets"] = torch.tensor([spare[0] + sum(news[:i]) for i in range(N + 1)], dtype=torch.int32)
    x["lengths"] = torch.tensor(lengths, dtype=torch.int32)
    return x, g


def device(x, by_heads=False):
    y = {n: t.cuda() for n, t in x.items()}
    if by_heads:
        for n in ("k_pages", "v_pages"):
            y[n] = y[n].transpose(1, 2).contiguous().transpose(1, 2)
    return y


def run(y, H, scale, **kw):
    import paper_2501_06480_amd as fwa
    return fwa.fwa_page_forward(y["q"], y["k_pages"], y["v_pages"], y["page_table"], y["offsets"], y["lengths"], H, scale, want_stats=True, **kw)


def compare(x, H, scale, what, by_heads=False, most_new=None, causal=True):
    before = torch.full_like(x["q"], 7.0)
    o, stats = run(device(x, by_heads), H, scale, most_new=most_new, causal=causal, out=before.cuda())
    want = ref.attention(x["q"], x["k_pages"], x["v_pages"], x["page_table"], x["offsets"], x["lengths"], H, scale, causal, most_new)
    ref.check_attention(o, stats, before, want, what)
    return o, stats


CASES = [  # dtype, new tokens, older ones, H, KV, d, page, by_heads, causal
    (BF16, [1], [0], 1, 1, 64, 16, False, True),
    (BF16, [1, 1, 1, 1], [0, 15, 16, 700], 8, 2, 128, 16, False, True),
    (F16, [4], [700], 12, 12, 64, 64, False, True),
    (F32, [1, 1], [333, 40], 4, 4, 32, 16, True, True),
    (F32, [1, 2], [65, 300], 8, 1, 128, 48, False, True),
    (F32, [3, 1], [65, 300], 4, 2, 64, 32, False, True),
    (BF16, [32], [1000], 1, 1, 32, 16, False, True),     # as many rows as the form for few has
    (BF16, [33], [1000], 1, 1, 32, 16, False, True),     # one more
    (BF16, [200], [0], 4, 2, 64, 16, False, True),
    (F16, [129, 129], [70, 0], 4, 1, 128, 48, True, True),
    (BF16, [300], [450], 3, 3, 128, 256, False, True),
    (F32, [100, 100], [33, 200], 2, 2, 32, 16, False, True),
    (F32, [70], [130], 2, 1, 64, 80, True, True),
    (F32, [40], [90], 3, 1, 128, 16, False, True),
    (BF16, [65, 1, 200, 1, 17, 0, 1], [1, 700, 0, 33, 500, 12, 0], 4, 2, 64, 16, False, True),   # a mixed batch
    (F16, [1, 150, 2, 90], [300, 20, 31, 0], 8, 1, 32, 32, True, True),
    (F32, [1, 65, 2], [300, 20, 31], 6, 2, 32, 48, False, True),
    (BF16, [50, 64], [20, 100], 4, 4, 64, 16, False, False),
    (F16, [2, 1], [20, 100], 4, 4, 128, 16, False, False),
]


@pytest.mark.parametrize("dtype,news,lengths,H,KV,d,size,by_heads,causal", CASES)
def test_attention(dtype, news, lengths, H, KV, d, size, by_heads, causal):
    x, _ = make(dtype, news, lengths, H, KV, d, size)
    what = f"{dtype} {news} {lengths} {H}/{KV} d{d}"
    compare(x, H, d ** -0.5, what, by_heads, max(news), causal)
    compare(x, H, d ** -0.5, what + " most unknown", by_heads, None, causal)


@pytest.mark.parametrize("dtype,d", [(BF16, 64), (F32, 32), (F16, 128), (BF16, 32), (F32, 128)])
@pytest.mark.parametrize("new,H,KV", [(1, 4, 4), (1, 8, 1), (4, 8, 2), (1, 64, 2), (20, 6, 3), (60, 4, 2)])
def test_long_caches_are_shared_out(dtype, d, new, H, KV):
    """Caches of different lengths behind a wide table: several workgroups have a block's keys, and sequences too short for that do without."""
    import paper_2501_06480_amd as fwa
    lengths = [1500 - new, 0, 700, 30]
    x, _ = make(dtype, [new] * 4, lengths, H, KV, d, 16, wider=100)
    code = {F32: 0, BF16: 1, F16: 2}[dtype]
    assert fwa.fwa_page_forward_workspace_bytes(4 * new, 4, H, KV, d, 16, x["page_table"].shape[1], new, code) > 0
    compare(x, H, d ** -0.5, f"{dtype} d{d} {new} {H}/{KV}", most_new=new)


@pytest.mark.parametrize("dtype,H,KV,d,size,causal", [(BF16, 4, 2, 64, 16, True), (F16, 4, 1, 128, 48, True), (F32, 2, 2, 32, 16, True), (F32, 2, 1, 128, 16, True),
                                                      (BF16, 6, 3, 32, 32, False), (BF16, 8, 1, 128, 16, True)])
@pytest.mark.parametrize("news,lengths", [([1, 150, 1, 40, 0, 260, 1], [900, 1500, 0, 2000, 700, 10, 3000]), ([300, 1], [2500, 100]), ([0, 0, 130], [50, 0, 4000]),
                                          ([1] * 60 + [70, 0, 1, 33], [0, 1, 400, 90] * 15 + [1200, 10, 1600, 0])])
def test_chunks_of_different_lengths(dtype, H, KV, d, size, causal, news, lengths):
    """Up to 64 sequences of which each brings what it has, behind wide tables: blocks are cut into parts of about one length, some into one, some into many."""
    x, _ = make(dtype, news, lengths, H, KV, d, size, spare=(2, 3), wider=3000 // size)
    for n, column in ((len(news) - 1, 3), (1, 0)):
        x["page_table"][n, column] = -1
    got = compare(x, H, d ** -0.5, f"{dtype} {news[:7]} {H}/{KV} d{d}", size == 48, None, causal)
    again = run(device(x), H, d ** -0.5, most_new=None, causal=causal, out=torch.full_like(x["q"], 7.0).cuda())
    rows = slice(2, x["q"].shape[0] - 3)
    assert torch.equal(got[0], again[0]) and torch.equal(got[1][rows], again[1][rows])


@pytest.mark.parametrize("dtype,H,KV,d,new,length", [(BF16, 1, 1, 64, 40, 6000), (F16, 2, 1, 128, 70, 4000), (F32, 1, 1, 128, 35, 2500), (F32, 3, 1, 32, 20, 5000), (BF16, 1, 1, 32, 140, 3000)])
def test_many_parts_of_few_blocks(dtype, H, KV, d, new, length):
    """Few rows too many for the form for few, against a long cache: a block in dozens of parts, of one sequence and beside a short one."""
    x, _ = make(dtype, [new], [length], H, KV, d, 16)
    compare(x, H, d ** -0.5, f"{dtype} {new} on {length} d{d}", most_new=new)
    x, _ = make(dtype, [new, 7], [length, 300], H, KV, d, 16)
    compare(x, H, d ** -0.5, f"{dtype} {new} and 7 on {length} d{d}", most_new=new)


@pytest.mark.parametrize("H,KV,d", [(2, 1, 32), (6, 3, 64), (2, 2, 128)])
@pytest.mark.parametrize("news,lengths,wider", [([32, 32], [500, 20], 0), ([30, 1, 0, 20], [300, 1500, 9, 0], 0), ([17, 32, 5], [0, 900, 3000], 100), ([3] * 66 + [31], [0, 40, 100] * 22 + [200], 0)])
def test_two_blocks_of_few_fp32_rows(H, KV, d, news, lengths, wider):
    """32 to 64 rows of a sequence, in two blocks whose waves share out the keys: alone, beside others of one block, with and without parts, more sequences than lanes."""
    x, _ = make(F32, news, lengths, H, KV, d, 16, spare=(1, 2), wider=wider)
    compare(x, H, d ** -0.5, f"{news[:4]} {H}/{KV} d{d}", most_new=max(news))
    compare(x, H, d ** -0.5, f"{news[:4]} {H}/{KV} d{d} all", most_new=max(news), causal=False)


def test_mixed_batches_of_many_sequences():
    """More sequences than lanes: their blocks are found by a search of two steps."""
    g = torch.Generator().manual_seed(5)
    news = [1 if i % 9 else int(torch.randint(1, 90, (1,), generator=g)) for i in range(150)]
    for i in (0, 1, 40, 77, 78, 149):
        news[i] = 0
    lengths = torch.randint(0, 60, (150,), generator=g).tolist()
    x, _ = make(BF16, news, lengths, 2, 1, 32, 16)
    compare(x, 2, 0.2, "many", most_new=90)
    x, _ = make(F16, [1] * 300, torch.randint(0, 60, (300,), generator=g).tolist(), 2, 2, 64, 16)
    compare(x, 2, 0.2, "tokens", most_new=1)


def test_pages_that_are_none_are_not_seen():
    """Entries outside the pages at the front, in the middle and at the end, whole sequences of them: rows that see nothing give zeros."""
    for dtype, H, KV, d, news, lengths in ((BF16, 4, 2, 64, [1, 1, 1, 1], [300, 300, 300, 20]), (F32, 2, 1, 32, [90, 40, 70, 20], [100, 60, 0, 0]),
                                           (F16, 2, 2, 128, [3, 100, 1, 40], [500, 60, 30, 0])):
        x, _ = make(dtype, news, lengths, H, KV, d, 16)
        pages = x["k_pages"].shape[0]
        x["page_table"][0, 0], x["page_table"][0, 3], x["page_table"][0, 4] = -1, pages, 0x7fffffff
        x["page_table"][1, 1:3] = -0x80000000
        x["page_table"][2] = -1
        x["page_table"][3, 1] = -1
        o, stats = compare(x, H, d ** -0.5, f"none {dtype}", most_new=max(news))
        a, b = int(x["offsets"][2]), int(x["offsets"][3])
        assert float(o[a:b].abs().max()) == 0.0 and bool(torch.isinf(stats[a:b, :, 0]).all()) and float(stats[a:b, :, 1].abs().max()) == 0.0


def test_a_cache_without_pages_and_tables_without_entries():
    x, _ = make(BF16, [3, 70], [0, 10], 2, 2, 64, 16)
    for shrink in ({"k_pages": x["k_pages"][:0], "v_pages": x["v_pages"][:0]}, {"page_table": x["page_table"][:, :0].contiguous()}):
        y = device({**x, **shrink})
        o, stats = run(y, 2, 0.1)
        assert float(o.abs().max()) == 0.0 and bool(torch.isinf(stats[..., 0]).all())


def test_what_no_key_has_does_not_matter():
    """NaN in all rows of the cache that no sequence sees, within the last pages of the sequences and in pages of nobody; the same bits as without."""
    for dtype, H, KV, d, news, lengths, size in ((BF16, 4, 1, 64, [1, 1, 1], [37, 500, 0], 16), (F16, 2, 2, 128, [100, 37, 1], [5, 90, 200], 48),
                                                 (F32, 2, 1, 32, [70, 1], [3, 100], 64)):
        x, _ = make(dtype, news, lengths, H, KV, d, size)
        clean, stats = compare(x, H, d ** -0.5, f"{dtype}", most_new=max(news))
        held = torch.zeros(x["k_pages"].shape[:2], dtype=torch.bool)
        for n, (new, length) in enumerate(zip(news, lengths)):
            for t in range(new + length):
                held[int(x["page_table"][n, t // size]), t % size] = True
        for n in ("k_pages", "v_pages"):
            x[n][~held] = float("nan")
        o, again = run(device(x), H, d ** -0.5, most_new=max(news))
        assert torch.equal(o, clean) and torch.equal(again, stats)


def test_rows_of_no_sequence_and_offsets_of_all_kinds():
    x, _ = make(BF16, [5, 0, 70, 1, 0], [20, 7, 33, 0, 9], 2, 1, 64, 16, spare=(4, 11))
    compare(x, 2, 0.125, "spare rows")
    compare(x, 2, 0.125, "fewer counted", most_new=40)
    x["lengths"][:] = torch.tensor([-3, 0, -0x80000000, 0x7fffffff, 5])  # below zero: none; beyond the table: what it has room for
    compare(x, 2, 0.125, "lengths")
    x["offsets"][-1] = 1 << 30
    x["offsets"][0] = -(1 << 30)
    o, _ = run(device(x), 2, 0.125)
    torch.cuda.synchronize()
    x["offsets"][:] = torch.tensor([90, 3, 40, 10, 0, 80])  # falling: whatever rows come out, no access leaves the tensors
    run(device(x), 2, 0.125)
    torch.cuda.synchronize()
    y = device(x)
    y["offsets"].zero_()
    assert bool((run(y, 2, 0.125, out=torch.full_like(y["q"], 7.0))[0] == 7.0).all())
    for n in (0,):
        empty = {**y, "q": y["q"][:0]}
        assert run(empty, 2, 0.125)[0].shape == (0, 128)
    assert run(y, 2, 0.125, most_new=0)[0].shape == y["q"].shape


@pytest.mark.parametrize("scale", [0.0, -0.3, 4.0])
def test_scales(scale):
    for dtype, news in ((BF16, [3, 80]), (F32, [1, 50])):
        x, _ = make(dtype, news, [40, 9], 2, 1, 64, 16)
        x["page_table"][0, 1] = -1
        compare(x, 2, scale, f"scale {scale}", most_new=max(news))


def test_large_scores_and_one_key_above_all():
    """Scores in the hundreds, one key far above the others at the end of the keys: the reference moves in the last tile."""
    for dtype in (BF16, F16, F32):
        x, _ = make(dtype, [1, 100], [300, 200], 2, 2, 64, 16)
        x["q"] *= 4
        for n, total in ((0, 301), (1, 300)):
            t = total - 1
            x["k_pages"][int(x["page_table"][n, t // 16]), t % 16] *= 6
        compare(x, 2, 0.5, f"{dtype} large", most_new=100)


def test_views_of_a_fused_projection_and_a_wider_output():
    H, KV, d = 4, 2, 64
    x, g = make(BF16, [1, 40, 1], [100, 20, 7], H, KV, d, 16)
    y = device(x)
    want, stats = run(y, H, 0.125, most_new=40)
    wide = torch.full((42, 2 * H * d), 7.0, dtype=BF16, device="cuda")
    fused = torch.randn(42, 3 * H * d, device="cuda").to(BF16)
    fused[:, H * d:2 * H * d] = y["q"]
    y["q"] = fused[:, H * d:2 * H * d]
    got, again = run(y, H, 0.125, most_new=40, out=wide[:, H * d:])
    assert torch.equal(got, want) and torch.equal(stats, again) and bool((wide[:, :H * d] == 7.0).all())


def test_refusals():
    import paper_2501_06480_amd as fwa
    x, _ = make(BF16, [3, 40], [20, 0], 4, 2, 64, 16)
    y = device(x)
    f = lambda H=4, **kw: fwa.fwa_page_forward(*(kw.pop(n, y[n]) for n in ("q", "k_pages", "v_pages", "page_table", "offsets", "lengths")), H, 0.1, **kw)  # noqa: E731
    for bad in (lambda: f(H=3), lambda: f(H=8), lambda: f(q=y["q"].float()), lambda: f(q=y["q"][None]), lambda: f(k_pages=y["k_pages"][:3]),
                lambda: f(v_pages=y["v_pages"].transpose(1, 2).contiguous().transpose(1, 2)), lambda: f(page_table=y["page_table"][:1]),
                lambda: f(page_table=y["page_table"].t().contiguous().t() if y["page_table"].shape[1] > 1 else y["page_table"].long()), lambda: f(offsets=y["offsets"][1:]),
                lambda: f(lengths=y["lengths"].long()), lambda: f(out=torch.empty_like(y["q"][:5])), lambda: f(q=y["q"].cpu()), lambda: f(H=0)):
        with pytest.raises((TypeError, ValueError)):
            bad()
    with pytest.raises(fwa.FwaError):  # an output on top of an input
        f(out=y["q"])
    with pytest.raises(fwa.FwaError):  # head width 32 of 48
        f(q=y["q"][:, :192].contiguous(), k_pages=y["k_pages"][..., :48].contiguous(), v_pages=y["v_pages"][..., :48].contiguous())
    z, _ = make(BF16, [1], [3000], 4, 2, 64, 16)
    z = device(z)
    with pytest.raises(fwa.FwaError):
        fwa.fwa_page_forward(*(z[n] for n in ("q", "k_pages", "v_pages", "page_table", "offsets", "lengths")), 4, 0.1,
                             workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    assert math.isfinite(float(f()[0].float().abs().max()))
