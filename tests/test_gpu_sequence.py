"""Attention of whole sequences and its gradients against 64 bits (tests/sequence_reference.py, whose bounds follow from the
arithmetic): lengths from one to several tiles, odd sizes, shared key heads, padding, rows without a key, strides, few rows."""
import math

import pytest
import torch

import sequence_reference as ref

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32


def make(dtype, N, Lq, Lk, H, KV, d, nb=16, far=40, table=True, seed=0):
    from paper_2501_06480_amd import binding
    g = torch.Generator().manual_seed(seed + Lq * 31 + Lk * 7 + H + d)
    x = {n: torch.randn(N, L, h * d, generator=g).to(dtype) for n, L, h in (("q", Lq, H), ("k", Lk, KV), ("v", Lk, KV), ("d_o", Lq, H))}
    t = {}
    if table:
        t = {"table": torch.randn(H, nb, generator=g), "buckets": binding.log_buckets(nb, far)}
    return x, t, g


def device(t):
    return {n: x.cuda() if torch.is_tensor(x) else x for n, x in t.items()}


def run(x, t, H, scale, backward=True):
    import paper_2501_06480_amd as fwa
    xd, td = device(x), device(t)
    o, stats = fwa.fwa_sequence_forward(xd["q"], xd["k"], xd["v"], H, scale, want_stats=True, **td)
    got = {"o": o, "lse": stats.sum(-1) * math.log(2.0)}
    if backward:
        dtable = td.get("table") is not None
        got["dq"], got["dk"], got["dv"], dt = fwa.fwa_sequence_backward(xd["q"], xd["k"], xd["v"], o, stats, xd["d_o"], H, scale, want_dtable=dtable, **td)
        if dtable:
            got["dtable"] = dt
    return got


def compare(x, t, H, scale, what, backward=True):
    want = ref.attention(x["q"], x["k"], x["v"], H, scale, d_o=x["d_o"] if backward else None, **t)
    got = run(x, t, H, scale, backward)
    for n, y in got.items():
        ref.check(y, want[n], want[n + "_tol"], f"{what} {n}")
    return got


CASES = [  # dtype, N, Lq, Lk, H, KV, d, causal, ragged, table
    (F32, 1, 1, 1, 1, 1, 32, False, False, True),
    (F32, 2, 33, 65, 2, 1, 32, False, False, True),
    (F32, 2, 130, 130, 3, 3, 64, True, True, True),
    (F32, 1, 70, 200, 2, 2, 128, False, True, True),
    (F32, 2, 5, 129, 4, 2, 64, False, False, False),
    (BF16, 1, 1, 1, 2, 1, 64, False, False, True),
    (BF16, 1, 2, 3, 1, 1, 32, True, False, True),
    (BF16, 2, 31, 33, 4, 2, 32, False, True, True),
    (BF16, 2, 64, 64, 2, 2, 64, True, False, True),
    (BF16, 1, 128, 128, 2, 1, 128, False, False, False),
    (BF16, 2, 129, 191, 4, 1, 64, False, True, True),
    (BF16, 1, 300, 300, 3, 3, 32, True, True, True),
    (BF16, 1, 515, 515, 4, 2, 128, True, False, True),
    (BF16, 1, 700, 90, 2, 2, 64, False, False, True),
    (F16, 1, 1, 5, 2, 2, 128, False, False, True),
    (F16, 2, 100, 333, 4, 4, 64, False, True, True),
    (F16, 1, 257, 257, 6, 2, 128, True, False, True),
    (F16, 1, 400, 400, 2, 1, 32, False, False, True),
]


@pytest.mark.parametrize("dtype,N,Lq,Lk,H,KV,d,causal,ragged,table", CASES)
def test_forward_and_gradients(dtype, N, Lq, Lk, H, KV, d, causal, ragged, table):
    x, t, g = make(dtype, N, Lq, Lk, H, KV, d, table=table)
    t["causal"] = causal
    if ragged:
        t["k_lengths"] = torch.randint(1, Lk + 1, (N,), generator=g, dtype=torch.int32)
        if Lq == Lk:
            t["q_lengths"] = t["k_lengths"].clone()
    compare(x, t, H, d ** -0.5, f"{dtype} {Lq}x{Lk} {H}/{KV} d{d}")


@pytest.mark.parametrize("dtype,d", [(BF16, 64), (F32, 32), (F16, 128), (BF16, 32), (F32, 128)])
@pytest.mark.parametrize("Lq,H,KV", [(1, 4, 4), (1, 8, 1), (4, 8, 2), (3, 64, 2), (20, 6, 3)])
def test_few_rows_against_a_long_cache(dtype, d, Lq, H, KV):
    """New tokens at the end of caches of different lengths: rows of a group packed, keys shared out and joined."""
    import paper_2501_06480_amd as fwa
    N, Lk = 3, 1500
    x, t, _ = make(dtype, N, Lq, Lk, H, KV, d)
    t["k_lengths"] = torch.tensor([1500, Lq, 700], dtype=torch.int32)
    t["q_start"] = t["k_lengths"] - Lq
    t["causal"] = Lq > 1
    code = {F32: 0, BF16: 1, F16: 2}[dtype]
    assert fwa.fwa_sequence_forward_workspace_bytes(N, Lq, Lk, H, KV, d, code) > 0  # the split form
    compare(x, t, H, d ** -0.5, f"decode {dtype} d{d} {Lq} {H}/{KV}")


def test_what_lies_behind_the_lengths_does_not_matter():
    """NaN and infinities behind the lengths; lengths of zero, below zero and beyond the rows; the same results as without."""
    N, L, H, d = 5, 150, 2, 64
    x, t, _ = make(BF16, N, L, L, H, H, d)
    t["k_lengths"] = torch.tensor([150, 77, 0, -3, 1000], dtype=torch.int32)
    t["q_lengths"] = torch.tensor([150, 70, 20, 0, 149], dtype=torch.int32)
    clean = compare(x, t, H, d ** -0.5, "ragged")
    for n, y in x.items():
        for b in range(N):
            length = min(max(int(t["q_lengths" if n in ("q", "d_o") else "k_lengths"][b]), 0), L)
            y[b, length:] = float("nan")
            y[b, length::3] = float("inf")
    again = run(x, t, H, d ** -0.5)
    for n in clean:
        assert torch.equal(clean[n], again[n]), n
    assert float(clean["o"][2].abs().max()) == 0.0 and float(clean["dq"][2].abs().max()) == 0.0
    assert torch.isinf(clean["lse"][2]).all()


@pytest.mark.parametrize("start", [-70, -1000, 60, 5000, -(1 << 31), (1 << 31) - 1])
def test_starts_before_and_behind_the_keys(start):
    """Causal rows in front of the first key see nothing; far behind it they see all."""
    x, t, _ = make(BF16, 2, 140, 150, 2, 1, 64)
    t["q_start"] = torch.tensor([start, 3], dtype=torch.int32)
    t["causal"] = True
    compare(x, t, 2, 0.125, f"start {start}")


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_tables_that_shut_pairs_out(dtype):
    """-inf and the lowest finite value in the table: a band of keys, rows without any, rows of nothing but the lowest value."""
    lowest = torch.finfo(torch.float32).min
    for kind, fill in (("-inf", -math.inf), ("lowest", lowest)):
        x, t, _ = make(dtype, 1, 200, 200, 2, 2, 32, nb=9, far=4)
        t["buckets"] = torch.tensor([0, 1, 1, 2, 3, 4, 5, 6, 7], dtype=torch.int32)
        t["table"][:, 0] = fill   # keys 4 and more behind
        t["table"][:, 7] = fill   # keys 4 and more in front
        compare(x, t, 2, 32 ** -0.5, f"band {kind}")
        t["table"][1] = fill      # the second head: nothing at all
        if kind == "-inf":
            got = compare(x, t, 2, 32 ** -0.5, "no key")
            assert float(got["o"][..., 32:].abs().max()) == 0.0
        else:
            import paper_2501_06480_amd as fwa
            xd, td = device(x), device(t)
            o = fwa.fwa_sequence_forward(xd["q"], xd["k"], xd["v"], 2, 32 ** -0.5, **td)
            mean = x["v"][..., 32:].double().mean(1, keepdim=True).expand(-1, 200, -1)
            # scores vanish beside such a bias: the mean of the values, rounded once (weights of one are exact)
            ref.check(o[..., 32:], mean, 2 * ref.U[dtype] * mean.abs() + 1e-5, "uniform")


@pytest.mark.parametrize("scale", [0.0, -0.3, 4.0])
def test_scales(scale):
    x, t, _ = make(BF16, 1, 150, 170, 2, 2, 64)
    compare(x, t, 2, scale, f"scale {scale}")


def test_large_scores_keep_their_rows_apart():
    """Scores up to several hundred, rising along the keys: the running reference moves at every tile."""
    x, t, _ = make(F32, 1, 96, 400, 1, 1, 32)
    x["k"] = x["k"] * torch.linspace(0.1, 20.0, 400)[None, :, None]
    compare(x, t, 1, 1.0, "rising")


def test_one_key_gives_gradients_of_exactly_zero():
    x, t, _ = make(BF16, 2, 40, 1, 2, 2, 64)
    got = run(x, t, 2, 0.125)
    for n in ("dq", "dk", "dtable"):
        assert float(got[n].abs().max()) == 0.0, n


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_views_of_fused_projections_are_read_and_written_in_place(dtype):
    """q, k, v as the parts of one [N, L, (heads + 2 kv) d] tensor, the gradients into parts of another."""
    import paper_2501_06480_amd as fwa
    N, L, H, KV, d = 2, 150, 4, 2, 64
    x, t, _ = make(dtype, N, L, L, H, KV, d)
    t["causal"] = True
    parts = [0, H * d, (H + KV) * d, (H + 2 * KV) * d]
    fused = torch.cat([x["q"], x["k"], x["v"]], 2).cuda()
    q, k, v = (fused[..., a:b] for a, b in zip(parts, parts[1:]))
    td = device(t)
    o, stats = fwa.fwa_sequence_forward(q, k, v, H, 0.125, want_stats=True, **td)
    room = torch.full_like(fused, 7.0)
    out = tuple(room[..., a:b] for a, b in zip(parts, parts[1:]))
    wide = torch.zeros(N, L, 2 * H * d, dtype=dtype, device="cuda")
    wide[..., :H * d] = x["d_o"].cuda()
    fwa.fwa_sequence_backward(q, k, v, o, stats, wide[..., :H * d], H, 0.125, out=out, **td)
    plain = run(x, t, H, 0.125)
    assert torch.equal(o, plain["o"])
    for got, n in zip(out, ("dq", "dk", "dv")):
        assert torch.equal(got, plain[n]), n


def test_rows_around_the_outputs_are_left_as_they_were():
    import paper_2501_06480_amd as fwa
    x, t, _ = make(BF16, 1, 37, 70, 2, 2, 32)
    xd, td = device(x), device(t)
    room = torch.full((1, 40, 96), 7.0, dtype=BF16, device="cuda")
    fwa.fwa_sequence_forward(xd["q"], xd["k"], xd["v"], 2, 0.2, out=room[:, :37, :64], **td)
    assert float((room[:, 37:] - 7.0).abs().max()) == 0.0 and float((room[:, :, 64:] - 7.0).abs().max()) == 0.0


def test_the_same_bits_every_time():
    x, t, _ = make(BF16, 2, 300, 300, 8, 2, 64)
    a, b = run(x, t, 8, 0.125), run(x, t, 8, 0.125)
    for n in a:
        assert torch.equal(a[n], b[n]), n


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_lengths_of_zero(dtype):
    x, t, _ = make(dtype, 2, 40, 0, 2, 1, 64)
    got = run(x, t, 2, 0.125)
    assert all(float(got[n].abs().max()) == 0.0 for n in ("o", "dq", "dtable"))
    x, t, _ = make(dtype, 2, 0, 40, 2, 1, 64)
    got = run(x, t, 2, 0.125)
    assert all(float(got[n].abs().max()) == 0.0 for n in ("dk", "dv", "dtable")) and got["o"].shape == (2, 0, 128)
    x, t, _ = make(dtype, 0, 40, 40, 2, 1, 64)
    got = run(x, t, 2, 0.125)
    assert float(got["dtable"].abs().max()) == 0.0


def test_gradients_against_differences():
    """Directional derivatives of sum(o * d_o) in fp32 by central differences of the 64-bit reference's inputs."""
    x, t, g = make(F32, 1, 60, 80, 2, 1, 32)
    got = run(x, t, 2, 0.2)
    f = lambda y: float((ref.attention(y["q"], y["k"], y["v"], 2, 0.2, y["table"], t["buckets"])["o"] * x["d_o"].double()).sum())  # noqa: E731
    base = {"q": x["q"], "k": x["k"], "v": x["v"], "table": t["table"]}
    base = {n: y.double() for n, y in base.items()}
    ref.U[torch.float64], ref.STEP[torch.float64] = 2.0 ** -53, 0.0
    for n in base:
        step = torch.randn(base[n].shape, generator=g).double()
        h = 1e-5
        plus, minus = ({**base, n: base[n] + s * h * step} for s in (1, -1))
        numeric = (f(plus) - f(minus)) / (2 * h)
        mine = got["dtable" if n == "table" else "d" + n].double().cpu()
        # differences: h^2 times a third derivative, and 1e-16 / h of the sum's magnitude; the gradients: fp32
        assert abs(float((mine * step).sum()) - numeric) <= 1e-4 * float((mine.abs() * step.abs()).sum()) ** 0.5 + 1e-4, n
