"""Sequences of a few keys: the rows of a tile that no load fills take part in its products with a weight of zero, so what memory holds there has to be
finite also after the first of two walks over the keys.  Against 64 bits (tests/sequence_reference.py); of one key all but dV is zero."""
import pytest
import torch

import sequence_reference as ref
from test_gpu_sequence import BF16, F16, F32, device, make, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("d", [32, 64])
@pytest.mark.parametrize("Lq", [17, 32, 100])
def test_one_to_nine_keys(dtype, d, Lq):
    N = 9
    x, t, _ = make(dtype, N, Lq, 9, 2, 2, d)
    # sums over the waves of every magnitude and sign, whose bits as two 16-bit numbers are of every kind
    x["d_o"] = (x["d_o"].float() * torch.logspace(-3, 1.5, Lq)[None, :, None]).to(dtype)
    t["k_lengths"] = torch.arange(1, N + 1, dtype=torch.int32)
    want = ref.attention(x["q"], x["k"], x["v"], 2, d ** -0.5, d_o=x["d_o"], **t)
    got = run(x, t, 2, d ** -0.5)
    for n in ("o", "dq", "dk", "dv", "dtable"):
        ref.check(got[n], want[n], want[n + "_tol"], n)
    assert float(got["dq"][0].abs().max()) == 0.0 and float(got["dk"][0].abs().max()) == 0.0
