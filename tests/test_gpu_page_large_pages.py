"""Large pages of many heads: attention that takes its workspace from the query, in a cache of one page and in one whose heads are outermost."""
import pytest
import torch

import page_reference as ref
from test_gpu_page_forward import BF16, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads_outermost", [False, True])
def test_pages_of_more_than_half_a_billion_elements(heads_outermost):
    if torch.cuda.mem_get_info()[0] < 16 << 30:
        pytest.skip("needs 16 GB of device memory")
    import paper_2501_06480_amd as fwa
    KV, d, size, pages, keys = 128, 128, 65536, 2 if heads_outermost else 1, 300
    assert fwa.fwa_page_forward_workspace_bytes(1, 1, KV, KV, d, size, 2, 1, 1) > 0
    g = torch.Generator().manual_seed(2)
    small = {n: torch.randn(1, 304, KV, d, generator=g).to(BF16) for n in ("k_pages", "v_pages")}  # the first rows, in a page of 304
    x = {"q": torch.randn(1, KV * d, generator=g).to(BF16), **small, "page_table": torch.zeros(1, 1, dtype=torch.int32),
         "offsets": torch.tensor([0, 1], dtype=torch.int32), "lengths": torch.tensor([keys - 1], dtype=torch.int32)}
    y = {n: t.cuda() for n, t in x.items()}
    for n in small:
        large = torch.empty((KV, pages, size, d), dtype=BF16, device="cuda").permute(1, 2, 0, 3) if heads_outermost else torch.empty((pages, size, KV, d), dtype=BF16, device="cuda")
        large[pages - 1, :304] = y[n][0]
        y[n] = large
    y["page_table"] = torch.tensor([[pages - 1, -1]], dtype=torch.int32, device="cuda")
    before = torch.full_like(x["q"], 7.0)
    o, stats = run(y, KV, d ** -0.5, most_new=1, out=before.cuda())
    want = ref.attention(x["q"], x["k_pages"], x["v_pages"], x["page_table"], x["offsets"], x["lengths"], KV, d ** -0.5)
    ref.check_attention(o, stats, before, want, "large pages")
