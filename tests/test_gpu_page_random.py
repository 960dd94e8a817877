"""Drawn calls of the operators on a paged cache and of the rotation against 64 bits: sizes, spreads of new tokens, layouts, strides and pages that are none, as they come."""
import random

import pytest
import torch

import page_reference as ref
import test_gpu_page_append as append
import test_gpu_page_forward as forward
from test_gpu_page_forward import BF16, F16, F32

pytestmark = pytest.mark.gpu


def sizes(seed):
    r = random.Random(seed)
    d, kv = r.choice((32, 64, 128)), r.choice((1, 1, 2, 3, 5))
    group = r.choice((1, 1, 2, 3, 4, 7, 8))
    N = r.choice((1, 1, 2, 3, 7, 70))
    spread = r.choice(("one", "few", "chunks", "mixed"))
    most = {"one": 1, "few": r.randint(1, 40 // group + 1), "chunks": r.randint(1, 300 if N < 7 else 40), "mixed": r.randint(1, 200 if N < 7 else 30)}[spread]
    news = [1 if spread == "one" or (spread == "mixed" and r.random() < 0.7) else r.randint(0, most) for _ in range(N)]
    cached = r.choice((0, 20, 300, 1500 if N < 7 else 100))
    return r, r.choice((F32, BF16, BF16, F16)), news, [r.randint(0, cached) for _ in range(N)], kv * group, kv, d, r.choice((16, 16, 32, 48, 64, 112, 256))


@pytest.mark.parametrize("seed", range(40))
def test_drawn_attention(seed):
    r, dtype, news, lengths, H, KV, d, size = sizes(seed)
    if sum(news) == 0:
        news[0] = 1
    x, _ = forward.make(dtype, news, lengths, H, KV, d, size, seed=seed, spare=(r.randint(0, 3), r.randint(0, 5)), wider=r.choice((0, 0, 5, 300)) if len(news) < 70 else 0)
    for _ in range(r.choice((0, 0, 0, 4))):
        x["page_table"][r.randrange(len(news)), r.randrange(x["page_table"].shape[1])] = r.choice((-1, 1 << 30, x["k_pages"].shape[0]))
    print(seed, dtype, news[:8], lengths[:8], H, KV, d, size, flush=True)
    forward.compare(x, H, r.choice((d ** -0.5, -0.2, 0.5)), f"{seed}", r.random() < 0.5, r.choice((None, max(news), max(1, max(news) // 2))), r.random() < 0.8)


@pytest.mark.parametrize("seed", range(100, 130))
def test_drawn_append(seed):
    r, dtype, news, lengths, H, KV, d, size = sizes(seed)
    if sum(news) == 0:
        news[0] = 1
    pairs = d // 2 if r.random() < 0.6 else r.randint(1, d // 2)
    cut = r.randint(0, pairs)
    sections = r.choice((None, (pairs,), (cut, pairs - cut)))
    by_heads = r.random() < 0.5
    x, _ = append.make(dtype, news, lengths, H, KV, d, size, by_heads=by_heads, sections=sections, spare=(r.randint(0, 3), r.randint(0, 5)), seed=seed, positions=r.random() < 0.5)
    x["page_table"][r.randrange(len(news)), r.randrange(x["page_table"].shape[1])] = r.choice((-1, 1 << 30))
    print(seed, dtype, news[:8], lengths[:8], H, KV, d, size, sections, flush=True)
    append.compare(x, H, KV, d, f"{seed}", by_heads, r.random() < 0.5, r.random() < 0.7)


@pytest.mark.parametrize("seed", range(200, 230))
def test_drawn_rotation(seed):
    import paper_2501_06480_amd as fwa
    r = random.Random(seed)
    d, heads, N, L = r.choice((r.randint(1, 80), 64, 128, 72, 512)), r.randint(1, 9), r.randint(1, 4), r.choice((1, 3, 50, 401))
    dtype, pairs, axes = r.choice((F32, BF16, F16)), r.randint(0, d // 2), r.randint(1, 4)
    while heads * d % (4 if dtype == F32 else 8):
        heads += 1
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(N, L, heads * d, generator=g).to(dtype)
    positions = torch.randint(-5000, 1 << 20, r.choice(((L, axes), (N, L, axes))), generator=g, dtype=torch.int32)
    f, axis = torch.rand(pairs, generator=g), torch.randint(-1, axes + 1, (pairs,), generator=g, dtype=torch.int32)
    interleaved, inverse = r.random() < 0.5, r.random() < 0.5
    print(seed, dtype, d, heads, N, L, pairs, axes, interleaved, flush=True)
    got = fwa.fwa_rotary(x.cuda(), heads, positions.cuda(), f.cuda(), axis.cuda(), interleaved, inverse)
    ref.check(got, *ref.rotate(x, heads, positions, f, axis, interleaved, inverse), f"{seed}")
