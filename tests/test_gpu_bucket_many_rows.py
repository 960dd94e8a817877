"""A dense bias of more rows than one launch has workgroups."""
import pytest
import torch

import sequence_reference as ref

pytestmark = pytest.mark.gpu


def test_more_rows_than_workgroups():
    """2^24 rows of more than half a workgroup's elements, 137 GB: rows at the start, the end and in between are compared."""
    import paper_2501_06480_amd as fwa
    Lq, Lk, far, nb = 1 << 24, 4097, 128, 16
    if torch.cuda.mem_get_info()[0] < 150 << 30:
        pytest.skip("needs 150 GB of device memory")
    g = torch.Generator().manual_seed(1)
    table, buckets = torch.randn(1, nb, generator=g), torch.randint(0, nb, (2 * far + 1,), generator=g, dtype=torch.int32)
    q0 = -(1 << 23)
    got = fwa.fwa_bucket_gather(table.cuda(), buckets.cuda(), Lq, Lk, q0, torch.bfloat16)
    for i in (0, 1, 2, 3, (1 << 23) - 130, (1 << 23) + 1, (1 << 23) + 2000, (1 << 23) + 4100, Lq - 2, Lq - 1):
        want = ref.bias(table, buckets, 1, Lk, q0 + i).float().bfloat16()
        assert torch.equal(got[:, i:i + 1].cpu(), want), i
    del got
    torch.cuda.empty_cache()
