"""64-bit reference of the bias by buckets and of the attention of whole sequences (plain torch on the CPU), and what the
kernels' arithmetic may be off by.

u is half a step of the data's type (2^-8 bf16, 2^-11 half), e = U32 half a step of fp32, 2^-24.  16-bit data: a probability is rounded once
in front of the product with V (u of each term), the output once (u of the output); backward the same for P, dS and the four
gradients, and delta = sum(d_o * o) takes over what the stored output is off by.  fp32 data and everything else is fp32: a score
is a sum of d products (d e of the sum of their magnitudes), an exponent of magnitude x has an error of about x e, and sums of
n terms in blocks stay within a few dozen e of the sum of magnitudes.  Half data below 2^-14 have an absolute step: half of
it is 2^-25.  Below 2^-126, the smallest normal fp32 number, a probability may be taken as zero: up to TINY of each, times what it is
multiplied with."""
import math

import torch

U = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
U32 = 2.0 ** -24
TINY = 2.0 ** -126
STEP = {torch.float32: TINY, torch.bfloat16: TINY, torch.float16: 2.0 ** -25}


def columns(buckets, Lq, Lk, q_start):
    far = buckets.numel() // 2
    d = torch.arange(Lk)[None, :] - torch.arange(Lq)[:, None] - q_start
    return buckets.long()[d.clamp(-far, far) + far]


def bias(table, buckets, Lq, Lk, q_start=0):
    """[heads, Lq, Lk]; an entry outside the table adds nothing"""
    c = columns(buckets, Lq, Lk, q_start)
    inside = (c >= 0) & (c < table.shape[1])
    return torch.where(inside, table.double()[:, c.clamp(0, table.shape[1] - 1)], 0.0)


def by_bucket(x, buckets, nb, q_start=0):
    """sums of x [heads, Lq, Lk] over the pairs of each bucket"""
    c = columns(buckets, x.shape[1], x.shape[2], q_start).reshape(-1)
    ok = (c >= 0) & (c < nb)
    out = torch.zeros(x.shape[0], nb, dtype=torch.float64)
    out.index_add_(1, c[ok], x.reshape(x.shape[0], -1)[:, ok].double())
    return out


def attention(q, k, v, heads, scale, table=None, buckets=None, q_lengths=None, k_lengths=None, q_start=None, causal=False, d_o=None):
    """dict of the outputs in 64 bits and, under the same names with _tol, of what each element may be off by."""
    dtype = q.dtype
    u, step = U[dtype], STEP[dtype]
    N, Lq, C = q.shape
    d = C // heads
    Lk, kv = k.shape[1], k.shape[2] // d
    G = heads // kv
    r = {n: torch.zeros(t.shape, dtype=torch.float64) for n, t in (("o", q), ("dq", q), ("dk", k), ("dv", v))}
    r["lse"] = torch.full((N, heads, Lq), -math.inf, dtype=torch.float64)
    for n in ("o", "dq", "dk", "dv"):
        r[n + "_tol"] = torch.zeros_like(r[n])
    r["lse_tol"] = torch.zeros(N, heads, Lq, dtype=torch.float64)
    if table is not None:
        r["dtable"], r["dtable_tol"] = (torch.zeros(table.shape, dtype=torch.float64) for _ in range(2))
    get = lambda t, n, other: other if t is None else min(max(int(t[n]), 0), other)  # noqa: E731
    for n in range(N):
        lq, lk, start = get(q_lengths, n, Lq), get(k_lengths, n, Lk), 0 if q_start is None else int(q_start[n])
        for h in range(heads):
            a, b = slice(h * d, h * d + d), slice(h // G * d, h // G * d + d)
            Q, K, V = q[n, :lq, a].double(), k[n, :lk, b].double(), v[n, :lk, b].double()
            s = scale * (Q @ K.T)
            mag = abs(scale) * (Q.abs() @ K.abs().T)
            if table is not None:
                B = bias(table, buckets, lq, lk, start)[h]
                s = s + B
                mag = mag + B.abs().nan_to_num(posinf=0.0)
            if causal:
                s = s.masked_fill(torch.arange(lk)[None] > torch.arange(lq)[:, None] + start, -math.inf)
            top = s.amax(1, keepdim=True) if lk else torch.full((lq, 1), -math.inf, dtype=torch.float64)
            p = torch.where(top == -math.inf, 0.0, torch.exp(s - torch.where(top == -math.inf, 0.0, top)))
            l = p.sum(1, keepdim=True)
            p = p / torch.where(l > 0, l, 1.0)
            any_key = (l > 0).squeeze(1)
            # relative error of a probability before it is rounded: the score's, the exponent's, the row sum's
            rel = (d + 8) * U32 * mag.clamp(max=1e6) + 16 * U32 * (1 + (s - top).abs().nan_to_num(nan=0.0, posinf=0.0).clamp(max=200.0))
            rel = rel + (p * rel).sum(1, keepdim=True) + 32 * U32
            r["lse"][n, h, :lq] = torch.where(any_key, (top + torch.log(torch.where(l > 0, l, 1.0))).squeeze(1), torch.tensor(-math.inf).double())
            r["lse_tol"][n, h, :lq] = (p * rel).sum(1) + 4 * U32 * top.abs().squeeze(1).nan_to_num(posinf=0.0) + 1e-6
            round_p = u if dtype != torch.float32 else 0.0
            o = p @ V
            o_tol = (p * (rel + round_p)) @ V.abs() + step * V.abs().sum(0, keepdim=True) + u * o.abs() + 64 * U32 * (p @ V.abs())
            o_tol = o_tol * any_key[:, None]
            r["o"][n, :lq, a] = o
            r["o_tol"][n, :lq, a] = o_tol + step
            if d_o is None:
                continue
            g = d_o[n, :lq, a].double()
            dp, dp_mag = g @ V.T, g.abs() @ V.abs().T
            delta = (p * dp).sum(1, keepdim=True)
            ds = p * (dp - delta)
            delta_tol = (g.abs() * o_tol).sum(1, keepdim=True) + (d + 8) * U32 * (g.abs() * o.abs()).sum(1, keepdim=True)
            exact_delta = (p * dp_mag * (rel + 64 * U32)).sum(1, keepdim=True)  # where it is formed from dP itself
            delta_tol = torch.maximum(delta_tol, exact_delta)
            ds_tol = rel * p * (dp.abs() + delta.abs()) + (d + 8) * U32 * p * dp_mag
            ds_tol = ds_tol + TINY * (dp.abs() + delta.abs())
            dsr = ds_tol + p * delta_tol + round_p * (ds.abs() + p * delta_tol)
            r["dq"][n, :lq, a] = scale * (ds @ K)
            r["dq_tol"][n, :lq, a] = abs(scale) * (dsr @ K.abs() + 64 * U32 * ds.abs() @ K.abs() + step * K.abs().sum(0, keepdim=True)) + step
            r["dk"][n, :lk, b] += scale * (ds.T @ Q)
            r["dk_tol"][n, :lk, b] += abs(scale) * (dsr.T @ Q.abs() + 64 * U32 * ds.abs().T @ Q.abs() + step * Q.abs().sum(0, keepdim=True)) + step
            r["dv"][n, :lk, b] += p.T @ g
            r["dv_tol"][n, :lk, b] += (p * (rel + round_p + 64 * U32)).T @ g.abs() + step * g.abs().sum(0, keepdim=True) + step
            if table is not None:
                r["dtable"][h] += by_bucket(ds[None], buckets, table.shape[1], start)[0]
                each = ds_tol + p * exact_delta + 64 * U32 * p * (dp.abs() + delta.abs())
                r["dtable_tol"][h] += by_bucket(each[None], buckets, table.shape[1], start)[0]
    for n in ("dq", "dk", "dv"):
        r[n + "_tol"] += u * r[n].abs()
    return r


def check(got, want, tol, what):
    got = got.detach().double().cpu()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    finite = torch.isfinite(want)
    assert torch.equal(torch.isfinite(got), finite), (what, "finite in other places")
    assert torch.equal(got[~finite], want[~finite]), what
    over = (got - want).abs()[finite] - tol.expand_as(want)[finite]
    worst = float(over.max()) if over.numel() else 0.0
    assert worst <= 0.0, (what, "beyond the bound by", worst, "largest error", float((got - want).abs()[finite].max()))
