"""Attention of whole sequences at drawn sizes, types, head layouts, lengths, starts, maps and scales against 64 bits."""
import math
import random

import pytest
import torch

from test_gpu_sequence import BF16, F16, F32, compare

pytestmark = pytest.mark.gpu


def drawn(seed):
    r = random.Random(seed)
    size = lambda most: int(round(math.exp(r.uniform(0.0, math.log(most)))))  # noqa: E731
    dtype, d = r.choice((BF16, F16, F32)), r.choice((32, 64, 128))
    kv, group = r.randint(1, 4), r.choice((1, 1, 2, 3, 8))
    N, Lq = r.randint(1, 4), size(400)
    Lk = Lq if r.random() < 0.4 else size(500)
    g = torch.Generator().manual_seed(seed)
    x = {n: torch.randn(N, L, h * d, generator=g).to(dtype) for n, L, h in (("q", Lq, kv * group), ("k", Lk, kv), ("v", Lk, kv), ("d_o", Lq, kv * group))}
    t = {"causal": r.random() < 0.5}
    if r.random() < 0.8:
        nb, far = r.randint(1, 40), r.choice((0, 1, 2, 17, 63, 64, 128, 1000, 8192))
        t["table"] = torch.randn(kv * group, nb, generator=g) * r.choice((0.1, 1.0, 20.0))
        t["buckets"] = torch.randint(0, nb, (2 * far + 1,), generator=g, dtype=torch.int32)
    for name, most in (("q_lengths", Lq), ("k_lengths", Lk)):
        if r.random() < 0.5:
            t[name] = torch.randint(0, most + 2, (N,), generator=g, dtype=torch.int32)
    if r.random() < 0.5:
        t["q_start"] = torch.randint(-Lq - 5, Lk + 40, (N,), generator=g, dtype=torch.int32)
    scale = d ** -0.5 * r.choice((1.0, 1.0, 0.3, -1.0))
    return x, t, kv * group, scale, f"seed {seed}: {dtype} N{N} {Lq}x{Lk} {kv * group}/{kv} d{d} {sorted(t)}"


@pytest.mark.parametrize("seed", range(60))
def test_drawn_calls(seed):
    x, t, heads, scale, what = drawn(seed)
    print(what, flush=True)
    compare(x, t, heads, scale, what)


@pytest.mark.parametrize("far", [0, 1, 2, 31, 32, 33, 63, 64, 65])
@pytest.mark.parametrize("dtype,d", [(BF16, 64), (F32, 32)])
def test_ends_of_the_map_at_the_edges_of_tiles(far, dtype, d):
    """Distances cut off inside the first tiles, at their edges and one beyond: each pair counts in one column once."""
    g = torch.Generator().manual_seed(far)
    N, L, H = 2, 200, 2
    x = {n: torch.randn(N, L, H * d, generator=g).to(dtype) for n in ("q", "k", "v", "d_o")}
    t = {"table": torch.randn(H, 2 * far + 1, generator=g), "buckets": torch.arange(2 * far + 1, dtype=torch.int32),
         "q_start": torch.tensor([0, 37], dtype=torch.int32)}
    compare(x, t, H, d ** -0.5, f"far {far}")


def test_entries_of_the_map_outside_the_table():
    g = torch.Generator().manual_seed(1)
    x = {n: torch.randn(1, 140, 64, generator=g).bfloat16() for n in ("q", "k", "v", "d_o")}
    b = torch.randint(-3, 12, (41,), generator=g, dtype=torch.int32)
    b[0], b[40] = 9, -1
    compare(x, {"table": torch.randn(2, 8, generator=g), "buckets": b}, 2, 0.2, "outside")


def test_a_nan_in_the_table_reaches_the_rows_that_read_it():
    import paper_2501_06480_amd as fwa
    g = torch.Generator().manual_seed(2)
    q, k, v = (torch.randn(1, 100, 32, generator=g).cuda() for _ in range(3))
    table = torch.randn(1, 3, generator=g)
    table[0, 2] = float("nan")  # keys five or more in front
    buckets = torch.tensor([0, 0, 0, 0, 0, 1, 1, 1, 1, 1, 2], dtype=torch.int32)
    o = fwa.fwa_sequence_forward(q, k, v, 1, 0.2, table=table.cuda(), buckets=buckets.cuda())
    assert torch.isnan(o[:, :95]).all() and torch.isfinite(o[:, 95:]).all()
