"""Attention beyond one window: a learned relative position bias by buckets and the attention over whole sequences that
reads it, with the gradients of both.

A case is one call of these operators as a program makes it (sequences padded to one length, as [N, L, heads * d]):

  gather   the bias of all pairs written out from a table by buckets, for windows of a 1-D sequence or a whole one
  scatter  its gradient: the sums of a bias gradient over the pairs of each bucket
  forward  attention of a whole sequence (encoders, prompts)
  train    the same through autograd: output, gradients of queries, keys, values and of the table
  decode   one or a few new tokens per sequence against a cache of keys and values

``buckets`` maps the distance key - query, cut off at -far and far, to a column of the table ([2 far + 1] int32); here it
is the usual map: exact for short distances, then logarithmic up to ``far``.
"""
import math

import torch

own = False  # set from outside: the framework's operators instead of their plain form

TORCH = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}


def _bias_case(op, heads, Lq, Lk, nb=32, far=128, both=True, dtype="f32", name=None):
    c = {"op": op, "dtype": dtype, "heads": heads, "Lq": Lq, "Lk": Lk, "nb": nb, "far": far, "both": both}
    return c if name is None else dict(c, name=name)


def _case(op, dtype, N, Lq, Lk, heads, kv, d, causal=False, ragged=False, nb=32, far=128, name=None):
    c = {"op": op, "dtype": dtype, "N": N, "Lq": Lq, "Lk": Lk, "heads": heads, "kv": kv, "d": d, "causal": causal, "ragged": ragged,
         "nb": nb, "far": far}
    return c if name is None else dict(c, name=name)


def listed():
    return [
        # the bias of 49-token windows of a 1-D sequence, 12 heads: the smallest call, all launch and latency
        _bias_case("gather", 12, 49, 49, name="gather_window"),
        # the bias of a whole sequence, written out for code that wants it dense
        _bias_case("gather", 16, 2048, 2048, name="gather_sequence"),
        # the gradient of a window attention's bias, summed by buckets
        _bias_case("scatter", 6, 196, 196, name="scatter_window"),
        # odd lengths, a causal map over a wide range: every entry of the gradient read once
        _bias_case("scatter", 12, 1500, 2047, nb=64, far=1024, both=False, name="scatter_sequence"),
        # an encoder in evaluation, padded batch of sequences of different lengths
        _case("forward", "bf16", 4, 2048, 2048, 16, 16, 64, ragged=True, name="forward_encoder"),
        # a prompt of a decoder with shared key heads, half precision, odd length
        _case("forward", "f16", 1, 4001, 4001, 16, 4, 128, causal=True, name="forward_prompt"),
        # a short fp32 sequence with heads of width 32: few rows, latency and fp32 products
        _case("forward", "f32", 2, 333, 333, 6, 6, 32, name="forward_f32_short"),
        # an encoder in training: the largest of the common shapes, with the gradient of the table
        _case("train", "bf16", 4, 2048, 2048, 12, 12, 64, ragged=True, name="train_encoder"),
        # a decoder in training: shared key heads, causal, odd length, wide heads
        _case("train", "bf16", 2, 1023, 1023, 16, 4, 128, causal=True, name="train_decoder"),
        # fp32 training of short sequences with heads of width 32
        _case("train", "f32", 4, 515, 515, 3, 3, 32, ragged=True, name="train_f32"),
        # serving: one new token for each of 16 sequences against long caches of shared key heads
        _case("decode", "bf16", 16, 1, 8192, 32, 8, 128, ragged=True, name="decode_batch"),
        # one sequence, four drafted tokens, a short cache: latency
        _case("decode", "f16", 1, 4, 700, 12, 12, 64, ragged=True, name="decode_one"),
    ]


MOST_PAIRS = {"forward": 4 * 16 * 2048 * 2048 * 64, "train": 4 * 12 * 2048 * 2048 * 64}
MOST_CACHE = 16 * 8192 * 8 * 128
MOST_BIAS = 16 * 2048 * 2048


def draw(rng):
    """Another call of the same ranges: sequences of 1 to 8192 tokens, caches up to 32768, 1 to 32 heads of width 32, 64 or
    128 that share keys or do not, the three types (fp32 up to a quarter of the work), tables of 8 to 128 buckets."""
    log = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))  # noqa: E731
    op = rng.choice(("gather", "scatter", "forward", "forward", "train", "train", "decode"))
    while True:
        nb, far = rng.choice((8, 16, 32, 32, 64, 128)), rng.choice((64, 128, 128, 300, 1024, 2000))
        if far < nb:
            continue
        if op in ("gather", "scatter"):
            Lq = log(1, 4096)
            Lk = Lq if rng.random() < 0.6 else log(1, 4096)
            c = _bias_case(op, rng.randint(1, 32), Lq, Lk, nb, far, rng.random() < 0.5,
                           "bf16" if op == "gather" and rng.random() < 0.3 else "f32")
            if c["heads"] * Lq * Lk <= MOST_BIAS:
                return c
            continue
        d, kv, group = rng.choice((32, 64, 64, 128)), log(1, 32), rng.choice((1, 1, 2, 4, 8))
        if kv * group > 32:
            continue
        dtype = rng.choice(("bf16", "bf16", "f16", "f32"))
        if op == "decode":
            Lk = log(1, 32768)
            c = _case(op, dtype, log(1, 32), min(rng.choice((1, 1, 1, 2, 5)), Lk), Lk, kv * group, kv, d, False, rng.random() < 0.7, nb, far)
            if c["N"] * Lk * kv * d * SIZE[dtype] <= MOST_CACHE * 2:
                return c
            continue
        L = log(1, 8192) if rng.random() < 0.3 else log(64, 4096)
        same = op == "train" or rng.random() < 0.8
        c = _case(op, dtype, log(1, 16), L, L if same else log(1, 4096), kv * group, kv, d, rng.random() < 0.5 and same, rng.random() < 0.5, nb, far)
        if c["N"] * c["heads"] * L * c["Lk"] * d * (4 if dtype == "f32" else 1) <= MOST_PAIRS[op]:
            return c


def _bucket_map(nb, far, both, device):
    """Column of the table for each distance -far .. far: half of the columns for keys behind the query and half for keys
    in front of it (or all for those behind, ``both`` false); the first half of them one distance each, the others
    logarithmic up to ``far``."""
    def column(n, cols):
        exact = cols // 2
        if n < exact or exact == 0:
            return min(n, cols - 1)
        steps = cols - exact
        t = 0  # the largest t with exact * (far / exact)^(t / steps) <= n, in whole numbers
        while t + 1 < steps and exact ** (steps - t - 1) * far ** (t + 1) <= n ** steps:
            t += 1
        return exact + t
    if both:
        half = nb // 2
        cols = [column(-r, half) if r <= 0 else half + column(r, half) for r in range(-far, far + 1)]
    else:
        cols = [column(max(-r, 0), nb) for r in range(-far, far + 1)]
    return torch.tensor(cols, dtype=torch.int32, device=device)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))

    def normal(*shape, dtype=torch.float32, std=1.0):
        return (torch.randn(*shape, generator=g, device="cuda") * std).to(dtype)

    s = dict(case)
    s["table"] = normal(case["heads"], case["nb"], std=0.5)
    s["buckets"] = _bucket_map(case["nb"], case["far"], case.get("both", not case.get("causal", False)), "cuda")
    if case["op"] == "gather":
        return s
    if case["op"] == "scatter":
        s["dbias"] = normal(case["heads"], case["Lq"], case["Lk"], std=0.01)
        return s
    dtype, N, Lq, Lk, H, kv, d = TORCH[case["dtype"]], case["N"], case["Lq"], case["Lk"], case["heads"], case["kv"], case["d"]
    s["q"], s["k"], s["v"] = (normal(N, L, h * d, dtype=dtype) for L, h in ((Lq, H), (Lk, kv), (Lk, kv)))
    s["scale"] = d ** -0.5
    s["k_lengths"] = s["q_lengths"] = s["q_start"] = None
    if case["ragged"]:  # the first sequence fills its room, the others half to all of it
        lengths = torch.randint((Lk + 1) // 2, Lk + 1, (N,), generator=g, device="cuda", dtype=torch.int32)
        lengths[0] = Lk
        s["k_lengths"] = lengths
        if Lq == Lk:
            s["q_lengths"] = lengths
    if case["op"] == "decode":  # the new tokens are the last ones of the cache
        lengths = s["k_lengths"] if s["k_lengths"] is not None else torch.full((N,), Lk, dtype=torch.int32, device="cuda")
        s["q_start"] = torch.clamp(lengths - Lq, min=0)
        s["causal"] = Lq > 1
    if case["op"] == "train":
        s["d_o"] = normal(N, Lq, H * d, dtype=dtype)
        for name in ("q", "k", "v", "table"):
            s[name].requires_grad_(True)
    return s


def run(s):
    if own:
        return _own(s)
    with torch.no_grad():
        if s["op"] == "gather":
            return _plain_bias(s["table"], s["buckets"], s["Lq"], s["Lk"], None)[0].to(TORCH[s["dtype"]])
        if s["op"] == "scatter":
            return _plain_by_bucket(s["dbias"][None], s["buckets"], s["nb"], None)
        return _plain_attention(s)


def _own(s):
    from paper_2501_06480_amd import autograd, binding
    if s["op"] == "gather":
        return binding.fwa_bucket_gather(s["table"], s["buckets"], s["Lq"], s["Lk"], dtype=TORCH[s["dtype"]])
    if s["op"] == "scatter":
        return binding.fwa_bucket_scatter(s["dbias"], s["buckets"], s["nb"])
    terms = {n: s[n] for n in ("table", "buckets", "q_lengths", "k_lengths", "q_start", "causal")}
    if s["op"] == "train":
        o = autograd.sequence_attention(s["q"], s["k"], s["v"], s["heads"], s["scale"], **terms)
        return (o.detach(),) + torch.autograd.grad(o, (s["q"], s["k"], s["v"], s["table"]), s["d_o"])
    return binding.fwa_sequence_forward(s["q"], s["k"], s["v"], s["heads"], s["scale"], **terms)


def _distances(Lq, Lk, q_start, device):
    """key - query for every pair, [N or 1, Lq, Lk]"""
    at = torch.arange(Lq, device=device)[None]
    if q_start is not None:
        at = at + q_start[:, None]
    return torch.arange(Lk, device=device) - at[:, :, None]


def _plain_bias(table, buckets, Lq, Lk, q_start):
    """[N or 1, heads, Lq, Lk]"""
    far = buckets.numel() // 2
    column = buckets[_distances(Lq, Lk, q_start, table.device).clamp(-far, far) + far].long()
    return table[:, column].transpose(0, 1)


def _plain_by_bucket(ds, buckets, nb, q_start):
    """Sums of ds [N, heads, Lq, Lk] over the pairs of each bucket, added up in 64 bits: [heads, nb]"""
    N, H, Lq, Lk = ds.shape
    far = buckets.numel() // 2
    # each row shifted one place further than the row below it: a column then holds the pairs of one distance
    wide = torch.zeros(N, H, Lq, Lk + Lq, device=ds.device)
    wide[..., :Lk] = ds.flip(2)
    each = wide.view(N, H, -1)[..., : Lq * (Lk + Lq - 1)].view(N, H, Lq, Lk + Lq - 1).sum(2, dtype=torch.float64)
    at = torch.arange(-(Lq - 1), Lk, device=ds.device)[None].expand(N, -1)
    if q_start is not None:
        at = at - q_start[:, None]
    column = buckets[at.clamp(-far, far) + far].long()
    out = torch.zeros(H, nb, dtype=torch.float64, device=ds.device)
    out.scatter_add_(1, column.reshape(1, -1).expand(H, -1), each.transpose(0, 1).reshape(H, -1))
    return out.float()


def _plain_attention(s):
    N, Lq, Lk, H, kv, d = s["N"], s["Lq"], s["Lk"], s["heads"], s["kv"], s["d"]
    G, dtype, dev = H // kv, s["q"].dtype, s["q"].device
    q = s["q"].float().view(N, Lq, kv, G, d).permute(0, 2, 3, 1, 4).reshape(N, kv, G * Lq, d)
    k, v = (s[n].float().view(N, Lk, kv, d).transpose(1, 2).contiguous() for n in "kv")
    x = torch.matmul(q, k.transpose(-1, -2).contiguous()).view(N, H, Lq, Lk)
    x.mul_(s["scale"])
    x.add_(_plain_bias(s["table"], s["buckets"], Lq, Lk, s["q_start"]))
    distance = _distances(Lq, Lk, s["q_start"], dev)
    shut = torch.zeros_like(distance, dtype=torch.bool)
    if s["causal"]:
        shut = distance > 0
    if s["k_lengths"] is not None:
        shut = shut | (torch.arange(Lk, device=dev) >= s["k_lengths"][:, None, None])
    if s["q_lengths"] is not None:
        shut = shut | (torch.arange(Lq, device=dev) >= s["q_lengths"][:, None])[:, :, None]
    x.masked_fill_(shut[:, None], -math.inf)
    top = x.amax(-1, keepdim=True)
    x.sub_(torch.where(top == -math.inf, torch.zeros_like(top), top)).exp_()
    total = x.sum(-1, keepdim=True)
    p = x.div_(torch.where(total > 0, total, torch.ones_like(total)))  # rows without a key: zeros
    rows = lambda t: t.view(N, kv, G, Lq, d).permute(0, 3, 1, 2, 4).reshape(N, Lq, H * d).to(dtype)  # noqa: E731
    p = p.view(N, kv, G * Lq, Lk)
    o = rows(torch.matmul(p, v))
    if s["op"] != "train":
        return o
    g = s["d_o"].float().view(N, Lq, kv, G, d).permute(0, 2, 3, 1, 4).reshape(N, kv, G * Lq, d)
    keys = lambda t: t.transpose(1, 2).reshape(N, Lk, kv * d).to(dtype)  # noqa: E731
    dv = keys(torch.matmul(p.transpose(-1, -2), g))
    ds = torch.matmul(g, v.transpose(-1, -2).contiguous())
    ds.sub_((ds * p).sum(-1, keepdim=True)).mul_(p)
    dtable = _plain_by_bucket(ds.view(N, H, Lq, Lk), s["buckets"], s["nb"], s["q_start"])
    ds.mul_(s["scale"])
    return o, rows(torch.matmul(ds, k)), keys(torch.matmul(ds.transpose(-1, -2), q)), dv, dtable


def exact(case, seed):
    """The same from the definition in 64 bits, a head of a sequence at a time."""
    s = prepare(case, seed)
    Lq, Lk, H, dev = s["Lq"], s["Lk"], s["heads"], s["table"].device
    table, far = s["table"].detach().double(), case["far"]

    def columns(start):
        i = torch.arange(start, start + Lq, device=dev).view(-1, 1)
        j = torch.arange(Lk, device=dev).view(1, -1)
        return s["buckets"].long()[torch.minimum(torch.maximum(j - i, torch.tensor(-far, device=dev)), torch.tensor(far, device=dev)) + far], j > i

    if s["op"] == "gather":
        c, _ = columns(0)
        return torch.stack([table[h][c] for h in range(H)])
    if s["op"] == "scatter":
        c, _ = columns(0)
        return torch.stack([torch.bincount(c.reshape(-1), weights=s["dbias"][h].double().reshape(-1), minlength=s["nb"]) for h in range(H)])
    N, d, G = s["N"], s["d"], H // s["kv"]
    train = s["op"] == "train"
    out = {n: torch.zeros(t.shape, dtype=torch.float64, device=dev) for n, t in (("q", s["q"]), ("k", s["k"]), ("v", s["v"]), ("o", s["q"]), ("table", table))}
    for n in range(N):
        start = 0 if s["q_start"] is None else int(s["q_start"][n])
        lq = Lq if s["q_lengths"] is None else int(s["q_lengths"][n])
        lk = Lk if s["k_lengths"] is None else int(s["k_lengths"][n])
        c, ahead = columns(start)
        c, ahead = c[:lq, :lk], ahead[:lq, :lk]
        for h in range(H):
            at, kat = slice(h * d, (h + 1) * d), slice(h // G * d, (h // G + 1) * d)
            q, k, v = s["q"].detach()[n, :lq, at].double(), s["k"].detach()[n, :lk, kat].double(), s["v"].detach()[n, :lk, kat].double()
            x = s["scale"] * (q @ k.t()) + table[h][c]
            if s["causal"]:
                x = x.masked_fill(ahead, -math.inf)
            p = torch.softmax(x, 1)  # every row has a key in these cases: its own, or the cache's first
            out["o"][n, :lq, at] = p @ v
            if train:
                g = s["d_o"][n, :lq, at].double()
                dp = g @ v.t()
                ds = p * (dp - (dp * p).sum(1, keepdim=True))
                out["q"][n, :lq, at] = s["scale"] * (ds @ k)
                out["k"][n, :lk, kat] += s["scale"] * (ds.t() @ q)
                out["v"][n, :lk, kat] += p.t() @ g
                out["table"][h] += torch.bincount(c.reshape(-1), weights=ds.reshape(-1), minlength=s["nb"])
    return (out["o"], out["q"], out["k"], out["v"], out["table"]) if train else out["o"]


def work(case):
    """Inputs read once, outputs written once; products of the pairs that are not shut out (ragged: three quarters of each
    length on average), four matrix products for a forward and its gradients' five with one repeated: 4 and 14 flops a
    channel of a pair."""
    H, Lq, Lk = case["heads"], case["Lq"], case["Lk"]
    if case["op"] == "gather":
        return {"bytes": H * Lq * Lk * SIZE[case["dtype"]] + 4 * H * case["nb"], "flops": 0}
    if case["op"] == "scatter":
        return {"bytes": 4 * H * Lq * Lk + 4 * H * case["nb"], "flops": H * Lq * Lk}
    N, kv, d, size = case["N"], case["kv"], case["d"], SIZE[case["dtype"]]
    part = (1 + 0.75 * (N - 1)) / N if case["ragged"] else 1.0
    rows = part if Lq == Lk else 1.0
    pairs = N * H * Lq * Lk * rows * part * (0.5 if case["causal"] else 1.0)
    q, k = N * Lq * H * d * size, N * Lk * kv * d * size * part
    if case["op"] == "train":
        return {"bytes": 4 * q + 4 * k + 8 * H * case["nb"], "flops": 14 * d * pairs}
    return {"bytes": 2 * q + 2 * k + 4 * H * case["nb"], "flops": 4 * d * pairs}
