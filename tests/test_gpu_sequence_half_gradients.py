"""Gradients of half sequences where d_o is in the thousands, as a scaled loss makes it, and rows have many keys of nearly one weight: every dS is
inside the range that half data are promised, the sum of a row's unnormalised weights is not.  Against 64 bits
(tests/sequence_reference.py)."""
import pytest
import torch

import sequence_reference as ref
from test_gpu_sequence import BF16, F16, device, make, run

pytestmark = pytest.mark.gpu


def largest_ds(x, t, heads, scale):
    """the largest |dS| of the call, in 64 bits"""
    d = x["q"].shape[2] // heads
    most = 0.0
    for n in range(x["q"].shape[0]):
        for h in range(heads):
            at = slice(h * d, (h + 1) * d)
            q, k, v, g = (x[i][n, :, at].double() for i in ("q", "k", "v", "d_o"))
            s = scale * (q @ k.T)
            if t.get("table") is not None:
                s = s + ref.bias(t["table"], t["buckets"], s.shape[0], s.shape[1])[h]
            p, dp = torch.softmax(s, 1), g @ v.T
            most = max(most, float((p * (dp - (p * dp).sum(1, keepdim=True))).abs().max()))
    return most


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("q_size,d_o_size,Lk,d,table", [
    (1.0, 1024.0, 2048, 64, False),   # ordinary scores
    (0.02, 8192.0, 2048, 64, True),   # a row of nearly equal ones
    (0.0, 4096.0, 3001, 32, False),   # equal ones
    (0.3, 2048.0, 1500, 128, True),
    (30.0, 16.0, 400, 64, False),     # scores whose reference is beyond a thousand
])
def test_gradients_of_large_d_o(dtype, q_size, d_o_size, Lk, d, table):
    H = 2
    x, t, _ = make(dtype, 1, 48, Lk, H, H, d, table=table)
    x["q"], x["d_o"] = x["q"] * q_size, x["d_o"] * d_o_size
    if q_size == 30.0:
        x["k"] = x["k"] * 30.0
    scale = d ** -0.5
    assert largest_ds(x, t, H, scale) < 1023.0
    want = ref.attention(x["q"], x["k"], x["v"], H, scale, d_o=x["d_o"], **t)
    got = run(x, t, H, scale)
    for n in ("o", "dq", "dk", "dv") + (("dtable",) if table else ()):
        ref.check(got[n], want[n], want[n + "_tol"], n)


@pytest.mark.parametrize("causal", [False, True])
def test_large_d_o_in_the_form_of_many_rows(causal):
    """More than a workgroup of 128 rows for each CU; two heads are compared."""
    import paper_2501_06480_amd as fwa
    H, L, d = 86, 1200, 64
    x, t, _ = make(F16, 1, L, L, H, H, d)
    x["q"], x["d_o"] = x["q"] * 0.05, x["d_o"] * 4096.0
    t["causal"] = causal
    t["table"] *= 0.1
    xd, td = device(x), device(t)
    o, stats = fwa.fwa_sequence_forward(xd["q"], xd["k"], xd["v"], H, 0.125, want_stats=True, **td)
    # the first rows of a causal call have few keys, whose dS may be beyond the range: small gradients there
    if causal:
        x["d_o"][:, :256] /= 256.0
        xd["d_o"] = x["d_o"].cuda()
    dq, dk, dv, dt = fwa.fwa_sequence_backward(xd["q"], xd["k"], xd["v"], o, stats, xd["d_o"], H, 0.125, want_dtable=True, **td)
    for h in (0, H - 1):
        at = slice(h * d, (h + 1) * d)
        part = {n: x[n][..., at] for n in x}
        want = ref.attention(part["q"], part["k"], part["v"], 1, 0.125, t["table"][h:h + 1], t["buckets"], causal=causal, d_o=part["d_o"])
        for got, n in ((o, "o"), (dq, "dq"), (dk, "dk"), (dv, "dv")):
            ref.check(got[..., at], want[n], want[n + "_tol"], f"{n} {h}")
        ref.check(dt[h:h + 1], want["dtable"], want["dtable_tol"], f"dtable {h}")
