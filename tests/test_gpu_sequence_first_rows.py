"""dQ of rows that see few keys, one of which has nearly all the weight: dP - delta cancels there, so delta has to come from the products that dP comes
from and not from the rounded output, whose half a step would be many times dS.  The bound leaves that term out; what remains is the
rounding of dS in front of its product and of dQ, and fp32."""
import pytest
import torch

import sequence_reference as ref
from test_gpu_sequence import BF16, F16, F32, device, make

pytestmark = pytest.mark.gpu


def dq_and_bound(q, k, v, g, scale, causal):
    """dQ of one head in 64 bits, and what it may be off by with delta = sum P dP.  u of each dS and of dQ.  An exponent of e has an error of about e
    U32, a score (d + 8) U32 of its products' magnitudes, sums of n terms a few dozen U32 of the sum of magnitudes."""
    u, U32 = ref.U[q.dtype], ref.U32
    q, k, v, g = (t.double() for t in (q, k, v, g))
    d = q.shape[1]
    s, mag = scale * (q @ k.T), abs(scale) * (q.abs() @ k.abs().T)
    if causal:
        s = s.masked_fill(torch.arange(k.shape[0])[None] > torch.arange(q.shape[0])[:, None], -float("inf"))
    p = torch.softmax(s, 1)
    rel = (d + 8) * U32 * mag + 16 * U32 * (1 + (s - s.amax(1, keepdim=True)).abs().nan_to_num(posinf=0.0))
    rel = rel + (p * rel).sum(1, keepdim=True) + 32 * U32
    dp, dp_mag = g @ v.T, g.abs() @ v.abs().T
    delta = (p * dp).sum(1, keepdim=True)
    ds = p * (dp - delta)
    delta_tol = (p * dp_mag * (rel + 64 * U32)).sum(1, keepdim=True)
    ds_tol = rel * ds.abs() + (d + 8) * U32 * p * (dp_mag + delta.abs()) + p * delta_tol + ref.TINY * (dp.abs() + delta.abs())
    step = ref.STEP[torch.float16] if u == ref.U[F16] else ref.TINY
    tol = abs(scale) * ((ds_tol + (u if u != U32 else 0.0) * (ds.abs() + ds_tol) + (64 + len(k)) * U32 * ds.abs() + step * (p > 0)) @ k.abs())
    dq = scale * (ds @ k)
    return dq, tol + u * (dq.abs() + tol) + step


@pytest.mark.parametrize("dtype,d", [(BF16, 128), (F16, 128), (BF16, 64), (F16, 32), (F32, 64), (F32, 128)])
@pytest.mark.parametrize("N,H,KV", [(16, 8, 4), (1, 2, 1)])  # both forms: many heads, and waves that share out the keys
def test_first_causal_rows(dtype, d, N, H, KV):
    import paper_2501_06480_amd as fwa
    L = 300
    x, _, _ = make(dtype, N, L, L, H, KV, d, table=False)
    x["q"] = x["q"] * 3
    xd, scale = device(x), d ** -0.5
    o, stats = fwa.fwa_sequence_forward(xd["q"], xd["k"], xd["v"], H, scale, want_stats=True, causal=True)
    dq = fwa.fwa_sequence_backward(xd["q"], xd["k"], xd["v"], o, stats, xd["d_o"], H, scale, causal=True)[0]
    for n, h in ((0, 0), (N - 1, H - 1)):
        a, b = slice(h * d, (h + 1) * d), slice(h // (H // KV) * d, (h // (H // KV) + 1) * d)
        want, tol = dq_and_bound(x["q"][n, :128, a], x["k"][n, :128, b], x["v"][n, :128, b], x["d_o"][n, :128, a], scale, True)
        ref.check(dq[n, :128, a], want, tol, f"dq {n} {h}")


@pytest.mark.parametrize("dtype,d", [(BF16, 128), (F16, 64), (F16, 128), (F32, 128)])
@pytest.mark.parametrize("N", [70, 3])
@pytest.mark.parametrize("Lk", [2, 40, 97, 128])
def test_sequences_of_few_keys(dtype, d, N, Lk):
    """The same accuracy whatever form the number of sequences leads to."""
    import paper_2501_06480_amd as fwa
    H, Lq = 4, 90
    x, _, _ = make(dtype, N, Lq, Lk, H, H, d, table=False)
    x["q"] = x["q"] * 3
    xd, scale = device(x), d ** -0.5
    o, stats = fwa.fwa_sequence_forward(xd["q"], xd["k"], xd["v"], H, scale, want_stats=True)
    dq = fwa.fwa_sequence_backward(xd["q"], xd["k"], xd["v"], o, stats, xd["d_o"], H, scale)[0]
    for n, h in ((0, 0), (N - 1, H - 1)):
        a = slice(h * d, (h + 1) * d)
        want, tol = dq_and_bound(x["q"][n, :, a], x["k"][n, :, a], x["v"][n, :, a], x["d_o"][n, :, a], scale, False)
        ref.check(dq[n, :, a], want, tol, f"dq {n} {h}")
