"""A key of NaN: every row that sees it is NaN, the gradients of padding stay zero."""
import pytest
import torch

from test_gpu_sequence import BF16, F32, device, make

pytestmark = pytest.mark.gpu


def both(x, t, H, scale):
    import paper_2501_06480_amd as fwa
    xd, td = device(x), device(t)
    o, stats = fwa.fwa_sequence_forward(xd["q"], xd["k"], xd["v"], H, scale, want_stats=True, **td)
    return (o, stats) + fwa.fwa_sequence_backward(xd["q"], xd["k"], xd["v"], o, stats, xd["d_o"], H, scale, want_dtable=True, **td)


@pytest.mark.parametrize("dtype,L", [(BF16, 150), (F32, 70)])
def test_a_key_of_nan_leaves_padding_zero(dtype, L):
    """Every row that sees the key is NaN; the gradients of keys behind the length stay zero."""
    x, t, _ = make(dtype, 1, L, L, 2, 2, 64)
    t["k_lengths"] = torch.tensor([L - 9], dtype=torch.int32)
    x["k"][0, 12, 3] = float("nan")
    o, _, dq, dk, dv, _ = both(x, t, 2, 0.125)
    assert torch.isnan(o[..., :64]).all() and torch.isnan(dq[..., :64]).all() and torch.isnan(dv[0, :L - 9, :64]).all()
    assert float(dk[0, L - 9:].abs().max()) == 0.0 and float(dv[0, L - 9:].abs().max()) == 0.0
