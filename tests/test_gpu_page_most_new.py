"""A sequence with more new tokens than the call was told of: the first ones are computed as if they were all there are, seen by each other alone, the others left out."""
import pytest
import torch

import page_reference as ref
from test_gpu_page_forward import BF16, F16, F32, device, make, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype,H,KV,d,news,lengths,most", [(BF16, 4, 2, 64, [30, 1, 6], [20, 300, 0], 15), (F32, 2, 1, 32, [90, 90], [70, 0], 45), (F16, 2, 2, 128, [200, 3, 140], [33, 50, 400], 130),
                                                            (BF16, 4, 1, 128, [3, 2, 9], [900, 0, 40], 2)])
def test_tokens_beyond_are_not_there(dtype, H, KV, d, news, lengths, most, causal):
    x, _ = make(dtype, news, lengths, H, KV, d, 16)
    before = torch.full_like(x["q"], 7.0)
    o, stats = run(device(x), H, d ** -0.5, most_new=most, causal=causal, out=before.cuda())
    kept = [min(n, most) for n in news]
    rows = torch.cat([torch.arange(int(a), int(a) + n) for a, n in zip(x["offsets"], kept)])
    # the same call without the others: packed without their rows
    few = {**x, "q": x["q"][rows].contiguous(), "offsets": torch.tensor([sum(kept[:i]) for i in range(len(kept) + 1)], dtype=torch.int32)}
    want = ref.attention(few["q"], *(few[n] for n in ("k_pages", "v_pages", "page_table", "offsets", "lengths")), H, d ** -0.5, causal)
    assert bool(want["rows"].all())
    ref.check_attention(o[rows.cuda()], stats[rows.cuda()], few["q"], want, f"{dtype} {news} of {most}")
    rest = torch.ones(len(o), dtype=torch.bool)
    rest[rows] = False
    assert bool((o.cpu()[rest] == 7.0).all())
