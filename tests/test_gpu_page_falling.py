"""Offsets that fall are against the contract, but no access leaves the tensors: blocks cut into parts of one length, more of them than the launch has workgroups."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,code,d", [(torch.bfloat16, 1, 64), (torch.float32, 0, 32)])
def test_falling_offsets_read_no_part_that_nobody_wrote(dtype, code, d):
    """64 sequences whose offsets rise and fall between none and all of 2560 rows, one with 256 tokens on a million: NaN in the workspace and behind it, so that a part
    from a place that no workgroup wrote, or from behind the workspace, is a NaN in the output; whatever else comes out is finite."""
    import paper_2501_06480_amd as fwa
    N, rows, size, width = 64, 2560, 16, 1 << 16
    g = torch.Generator().manual_seed(3)
    q = torch.randn(rows, d, generator=g).to(dtype).cuda()
    k_pages, v_pages = (torch.randn(50, size, 1, d, generator=g).to(dtype).cuda() for _ in range(2))
    table = torch.randint(0, 50, (N, width), generator=g, dtype=torch.int32).cuda()
    need = fwa.fwa_page_forward_workspace_bytes(rows, N, 1, 1, d, size, width, rows, code)
    assert need > 0
    for at in (0, 9, 40, 46, 57, 63):
        offsets = torch.tensor([2560 if n % 2 else 0 for n in range(N + 1)], dtype=torch.int32)
        offsets[at], offsets[at + 1] = 0, 256
        lengths = torch.zeros(N, dtype=torch.int32)
        lengths[at] = 1000000
        print(dtype, at, flush=True)
        whole = torch.full((need + (64 << 20),), 0xff, dtype=torch.uint8, device="cuda")
        o, _ = fwa.fwa_page_forward(q, k_pages, v_pages, table, offsets.cuda(), lengths.cuda(), 1, 0.1, want_stats=True, out=torch.zeros_like(q), workspace=whole[:need])
        torch.cuda.synchronize()
        assert bool(torch.isfinite(o).all()) and bool((whole[need:] == 0xff).all())
