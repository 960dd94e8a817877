"""Sequences whose queries see one key at most: its weight is one whatever the score, so all gradients but dV are zero, also where dP alone would
leave the range of half data."""
import pytest
import torch

import sequence_reference as ref
from test_gpu_sequence import BF16, F16, F32, device, make, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("N,Lq,Lk,H,d,terms", [
    (2, 104, 1, 2, 128, {}), (2, 40, 1, 2, 32, {}), (3, 20, 60, 2, 64, {"k_lengths": [1, 0, 1]}),
    (2, 1, 50, 2, 128, {"causal": True}), (2, 30, 50, 2, 64, {"causal": True, "q_start": [-29, -200]}), (2, 90, 70, 2, 128, {"causal": True, "q_lengths": [1, 1]}),
    (70, 90, 1, 4, 64, {}), (70, 90, 1, 4, 128, {}), (1, 2000, 1, 1, 32, {}),
])
def test_all_but_dv_is_zero(dtype, N, Lq, Lk, H, d, terms):
    x, t, _ = make(dtype, N, Lq, Lk, H, H, d)
    x["d_o"] = x["d_o"] * 500.0
    t.update({n: torch.tensor(y, dtype=torch.int32) if isinstance(y, list) else y for n, y in terms.items()})
    got = run(x, t, H, d ** -0.5)
    for n in ("dq", "dk", "dtable"):
        assert float(got[n].abs().max()) == 0.0, n
    want = ref.attention(x["q"][:3], x["k"][:3], x["v"][:3], H, d ** -0.5, d_o=x["d_o"][:3], **t)
    for n in ("o", "dv"):
        ref.check(got[n][:3], want[n], want[n + "_tol"], n)
