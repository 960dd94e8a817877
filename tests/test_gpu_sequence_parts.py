"""Backward of calls with few blocks of keys, whose queries several workgroups share: parts of different number for each block, blocks that no query
sees, starts and lengths that only the device knows.  Against 64 bits (tests/sequence_reference.py), and the same bits whatever the
workspace held."""
import math

import pytest
import torch

import sequence_reference as ref

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32


@pytest.mark.parametrize("dtype,N,Lq,Lk,H,KV,d,causal,starts,q_lengths,k_lengths", [
    (BF16, 1, 900, 900, 4, 1, 128, True, None, None, None),
    (BF16, 2, 640, 640, 4, 2, 64, True, [0, 0], None, None),
    (F16, 2, 500, 700, 2, 1, 128, True, [200, -100], None, [700, 430]),
    (BF16, 1, 200, 900, 2, 1, 64, True, None, None, None),
    (F32, 2, 520, 520, 2, 1, 32, True, None, [520, 77], [520, 0]),
    (F32, 2, 300, 260, 4, 1, 128, False, None, [0, 290], [260, 33]),
    (F16, 1, 1500, 20, 3, 1, 32, False, None, None, None),
])
def test_queries_shared_among_workgroups(dtype, N, Lq, Lk, H, KV, d, causal, starts, q_lengths, k_lengths):
    import paper_2501_06480_amd as fwa
    from paper_2501_06480_amd import binding
    g = torch.Generator().manual_seed(Lq + 3 * Lk + d)
    x = {n: torch.randn(N, L, h * d, generator=g).to(dtype) for n, L, h in (("q", Lq, H), ("k", Lk, KV), ("v", Lk, KV), ("d_o", Lq, H))}
    t = {"table": torch.randn(H, 16, generator=g), "buckets": binding.log_buckets(16, 100), "causal": causal}
    for n, y in (("q_start", starts), ("q_lengths", q_lengths), ("k_lengths", k_lengths)):
        if y is not None:
            t[n] = torch.tensor(y, dtype=torch.int32)
    scale = d ** -0.5
    want = ref.attention(x["q"], x["k"], x["v"], H, scale, d_o=x["d_o"], **t)
    x = {n: y.cuda() for n, y in x.items()}
    t = {n: y.cuda() if torch.is_tensor(y) else y for n, y in t.items()}
    o, stats = fwa.fwa_sequence_forward(x["q"], x["k"], x["v"], H, scale, want_stats=True, **t)
    code = {F32: binding.FWA_F32, BF16: binding.FWA_BF16, F16: binding.FWA_F16}[dtype]
    need = fwa.fwa_sequence_backward_workspace_bytes(N, Lq, Lk, H, KV, d, 100, code, True)
    assert need > 0
    results = []
    for fill in (255, 0):  # NaN everywhere, zeros
        workspace = torch.full((need,), fill, dtype=torch.uint8, device="cuda")
        results.append(fwa.fwa_sequence_backward(x["q"], x["k"], x["v"], o, stats, x["d_o"], H, scale, want_dtable=True, workspace=workspace, **t))
    for name, y, z in zip(("dq", "dk", "dv", "dtable"), *results):
        ref.check(y, want[name], want[name + "_tol"], name)
        assert torch.equal(y, z), name
    assert math.isfinite(float(o.float().abs().max()))
    if causal and starts is None and Lk > Lq:
        assert float(results[0][1][:, Lq:].abs().max()) == 0.0 and float(results[0][2][:, Lq:].abs().max()) == 0.0
