"""64-bit reference of the rotary positions and of the operators on a paged cache (plain torch on the CPU), and what the kernels' arithmetic may be off by.

U and U32 are half a step of the data's type and of fp32, as in sequence_reference.  Rotation: the angle is reduced to a part of a turn in 64 bits (the frequency in
turns and the product round once each, 2^-53 of the whole turns: at most 2^-51 of the angle) and rounded to fp32 there (half a turn at most, so 2^-25
turns, 2 pi 2^-25 < 4 U32 of the angle); cosine and sine add two steps of fp32 (4 U32 of a value up to 1): 8 U32 a factor; the two products
and the sum round once each, 2 U32 of each term; the result once to its type.
Attention: as in sequence_reference (scores, exponents and sums in fp32, P rounded once to 16-bit data in front of its product, the output once)."""
import math

import torch

from sequence_reference import STEP, U, U32, check  # noqa: F401


def rotate(x, heads, positions, frequencies, axis_of=None, interleaved=False, inverse=False):
    """x [..., L, heads * d], positions [..., L, axes] -> y in 64 bits and what it may be off by"""
    d, P = x.shape[-1] // heads, frequencies.numel()
    axis = torch.zeros(P, dtype=torch.long) if axis_of is None else axis_of.long()
    inside = (axis >= 0) & (axis < positions.shape[-1])
    angle = positions.double()[..., axis.clamp(0, positions.shape[-1] - 1)] * frequencies.double() * inside
    angle = (-angle if inverse else angle).expand(*x.shape[:-1], P).unsqueeze(-2)
    y = x.double().reshape(*x.shape[:-1], heads, d).clone()
    tol = torch.zeros_like(y)
    i, j = (slice(0, 2 * P, 2), slice(1, 2 * P, 2)) if interleaved else (slice(0, P), slice(P, 2 * P))
    a, b, c, s = y[..., i].clone(), y[..., j].clone(), torch.cos(angle), torch.sin(angle)
    y[..., i], y[..., j] = a * c - b * s, b * c + a * s
    off = (a.abs() + b.abs()) * (10 * U32 + angle.abs() * 2.0 ** -51)
    tol[..., i], tol[..., j] = off, off
    turned = torch.zeros(d, dtype=torch.bool)
    turned[i] = turned[j] = True
    tol += torch.where(turned, U[x.dtype] * y.abs() + STEP[x.dtype], 0.0)  # channels behind the pairs are copied
    return y.reshape(x.shape), tol.reshape(x.shape)


def new_tokens(offsets, lengths, rows, most=None):
    """(sequence, first row, new tokens, older tokens) of each sequence that has new tokens"""
    for n in range(len(lengths)):
        a, b = (min(max(int(x), 0), rows) for x in offsets[n:n + 2])
        count = min(b - a, rows if most is None else most)
        if count > 0:
            yield n, a, count, max(int(lengths[n]), 0)


def append(x, pool, page_table, offsets, lengths):
    """Rows of x [T, kv * d] put into a copy of the pool, and which of its rows were written"""
    pool, written = pool.clone(), torch.zeros(pool.shape[:2], dtype=torch.bool)
    size = pool.shape[1]
    for n, a, count, length in new_tokens(offsets, lengths, x.shape[0]):
        for i in range(count):
            at = length + i
            page = int(page_table[n, at // size]) if at // size < page_table.shape[1] else -1
            if 0 <= page < pool.shape[0]:
                pool[page, at % size] = x[a + i].reshape(pool.shape[2:])
                written[page, at % size] = True
    return pool, written


def attention(q, k_pages, v_pages, page_table, offsets, lengths, heads, scale, causal=True, most=None):
    """dict of o and lse in 64 bits, _tol, and of the rows that are written"""
    dtype, (pages, size, kv, d) = q.dtype, k_pages.shape
    u, step, T, G = U[dtype], STEP[dtype], q.shape[0], heads // kv
    r = {"o": torch.zeros(q.shape, dtype=torch.float64), "lse": torch.full((T, heads), -math.inf, dtype=torch.float64)}
    r["o_tol"], r["lse_tol"] = torch.zeros_like(r["o"]), torch.zeros(T, heads, dtype=torch.float64)
    r["rows"] = torch.zeros(T, dtype=torch.bool)
    for n, a, count, length in new_tokens(offsets, lengths, T, most):
        r["rows"][a:a + count] = True
        total = min(length + count, page_table.shape[1] * size)
        at = page_table[n, : -(-total // size)].long()
        real = ((at >= 0) & (at < pages)).repeat_interleave(size)[:total]
        at = at.clamp(0, max(pages - 1, 0))
        K, V = (p[at].reshape(-1, kv, d)[:total].double() if pages else torch.zeros(total, kv, d).double() for p in (k_pages, v_pages))
        K, V = (torch.where(real[:, None, None], x, 0.0) for x in (K, V))
        seen = real[None].expand(count, total)
        if causal:
            seen = seen & (torch.arange(total)[None] <= torch.arange(length, length + count)[:, None])
        for h in range(heads):
            Q, k, v = q[a:a + count, h * d:(h + 1) * d].double(), K[:, h // G], V[:, h // G]
            s = (scale * (Q @ k.T)).masked_fill(~seen, -math.inf)
            mag = abs(scale) * (Q.abs() @ k.abs().T)
            top = s.amax(1, keepdim=True) if total else torch.full((count, 1), -math.inf, dtype=torch.float64)
            p = torch.where(top == -math.inf, 0.0, torch.exp(s - torch.where(top == -math.inf, 0.0, top)))
            l = p.sum(1, keepdim=True)
            some = (l > 0).squeeze(1)
            p = p / torch.where(l > 0, l, 1.0)
            rel = (d + 8) * U32 * mag + 16 * U32 * (1 + (s - top).abs().nan_to_num(nan=0.0, posinf=0.0).clamp(max=200.0))
            rel = rel + (p * rel).sum(1, keepdim=True) + 32 * U32
            o = p @ v
            o_tol = (p * (rel + (u if dtype != torch.float32 else 0.0))) @ v.abs() + step * (seen.double() @ v.abs()) + u * o.abs() + 64 * U32 * (p @ v.abs()) + step
            r["o"][a:a + count, h * d:(h + 1) * d] = o
            r["o_tol"][a:a + count, h * d:(h + 1) * d] = o_tol * some[:, None]
            r["lse"][a:a + count, h] = torch.where(some, (top + torch.log(torch.where(l > 0, l, 1.0))).squeeze(1), torch.tensor(-math.inf).double())
            r["lse_tol"][a:a + count, h] = (p * rel).sum(1) + 4 * U32 * top.abs().squeeze(1).nan_to_num(posinf=0.0) + 1e-6
    return r


def check_attention(got, stats, before, want, what):
    """Rows of the sequences within their bounds, the others as they were"""
    rows = want["rows"]
    check(got.cpu()[rows], want["o"][rows], want["o_tol"][rows], what)
    assert torch.equal(got.cpu()[~rows], before.cpu()[~rows]), (what, "rows of no sequence")
    if stats is not None:
        check((stats.double().sum(-1) * math.log(2.0)).cpu()[rows], want["lse"][rows], want["lse_tol"][rows], what + " lse")
