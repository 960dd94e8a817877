"""Rows whose scores are all NaN: their gradients are NaN as their output is, those of other rows and heads have the bits that they have without
them, and padding stays zero."""
import pytest
import torch

from test_gpu_sequence import BF16, F16, F32, device, make

pytestmark = pytest.mark.gpu


def both(x, t, H, scale):
    import paper_2501_06480_amd as fwa
    xd, td = device(x), device(t)
    o, stats = fwa.fwa_sequence_forward(xd["q"], xd["k"], xd["v"], H, scale, want_stats=True, **td)
    return (o, stats) + fwa.fwa_sequence_backward(xd["q"], xd["k"], xd["v"], o, stats, xd["d_o"], H, scale, want_dtable=True, **td)


@pytest.mark.parametrize("dtype,H,L,d,causal", [(BF16, 2, 150, 64, False), (F16, 2, 300, 128, True), (F32, 2, 100, 32, False), (F32, 3, 70, 128, True),
                                                (BF16, 90, 300, 64, False), (F16, 90, 300, 32, True), (BF16, 90, 300, 128, False)])
def test_a_query_of_nan(dtype, H, L, d, causal):
    x, t, _ = make(dtype, 1, L, L, H, H, d)
    t["causal"] = causal
    t["k_lengths"] = torch.tensor([L - 20], dtype=torch.int32)
    i, klen = 33, L - 20
    clean = both(x, t, H, d ** -0.5)
    x["q"][0, i, 5] = float("nan")  # of the first head
    o, stats, dq, dk, dv, dt = both(x, t, H, d ** -0.5)
    others = torch.arange(L) != i
    seen = i + 1 if causal else klen
    assert torch.isnan(o[0, i, :d]).all() and torch.isnan(dq[0, i, :d]).all()
    assert torch.isnan(dk[0, :seen, :d]).all() and torch.isnan(dv[0, :seen, :d]).all()
    assert torch.isnan(dt[0, t["buckets"][40].item()])  # distance zero, which every row has
    assert float(dk[0, klen:].abs().max()) == 0.0 and float(dv[0, klen:].abs().max()) == 0.0
    for got, want in ((o, clean[0]), (dq, clean[2])):
        assert torch.equal(got[0, others, :d], want[0, others, :d])
    for got, want in ((o, clean[0]), (dq, clean[2]), (dk, clean[3]), (dv, clean[4])):
        assert torch.equal(got[..., d:], want[..., d:])
    assert torch.equal(dt[1:], clean[5][1:])


@pytest.mark.parametrize("dtype,H,L", [(BF16, 2, 200), (F16, 2, 90), (F32, 2, 130), (BF16, 90, 300)])
def test_a_table_of_nan(dtype, H, L):
    x, t, _ = make(dtype, 1, L, L, H, H, 64)
    clean = both(x, t, H, 0.125)
    t["table"][0] = float("nan")
    got = both(x, t, H, 0.125)
    for y, z in zip((got[0],) + got[2:5], (clean[0],) + clean[2:5]):
        assert torch.isnan(y[..., :64]).all()
        assert torch.equal(y[..., 64:], z[..., 64:])
    used = torch.zeros(16, dtype=torch.bool)
    used[t["buckets"].long()] = True
    assert torch.isnan(got[5][0].cpu()[used]).all() and torch.equal(got[5][1:], clean[5][1:])


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
def test_a_query_of_nan_and_one_key(dtype):
    x, t, _ = make(dtype, 2, 40, 1, 2, 2, 64)
    x["q"][1, 3, 70] = float("nan")
    o, _, dq, dk, dv, _ = both(x, t, 2, 0.125)
    assert torch.isnan(o[1, 3, 64:]).all() and torch.isnan(dq[1, 3, 64:]).all() and torch.isnan(dk[1, 0, 64:]).all() and torch.isnan(dv[1, 0, 64:]).all()
    dq[1, 3, 64:] = 0.0
    assert float(dq.abs().max()) == 0.0 and float(dk[0].abs().max()) == 0.0 and float(dk[1, :, :64].abs().max()) == 0.0
