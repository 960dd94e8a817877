"""Sizes at the ends of what the calls of sequences take (no GPU needed)."""
import pytest

from paper_2501_06480_amd import binding as b
from test_sequence_abi import P, S, backward, forward, lib  # noqa: F401


@pytest.mark.parametrize("call", [forward, backward])
def test_heads_times_width_beyond_32_bits(lib, call):  # noqa: F811
    assert call(lib, H=1 << 16, KV=1, d=1 << 16) == b.FWA_ERR_UNSUPPORTED
    assert call(lib, H=1 << 30, KV=1 << 30, d=1 << 30, Lq=0) == b.FWA_ERR_UNSUPPORTED
    assert call(lib, H=1 << 15, KV=1, d=128, Lq=1) == b.FWA_ERR_UNSUPPORTED  # rows of more than 2^20 elements


# the last: blocks of 128 tokens of all heads of all sequences; with 8 more per block of a sequence, as they are dealt, they pass 2^32 threads
@pytest.mark.parametrize("N,L,H", [(1 << 24, 1, 1), (1 << 19, 100, 32), (29, 1 << 24, 4)])
def test_more_blocks_than_a_launch_has(lib, N, L, H):  # noqa: F811
    """Refused as such, with no workspace to ask for."""
    big = dict(N=N, Lq=L, Lk=L, H=H, KV=H)
    places = [(1 << 44) + i * (1 << 42) for i in range(9)]
    assert forward(lib, **big, **dict(zip(("q", "k", "v", "o"), places))) == b.FWA_ERR_UNSUPPORTED
    assert backward(lib, **big, **dict(zip(("q", "k", "v", "o", "g", "stats", "dq", "dk", "dv"), places)), ws=1 << 50, ws_bytes=1 << 42) == b.FWA_ERR_UNSUPPORTED
    assert lib.fwa_sequence_forward_workspace_bytes(N, L, L, H, H, 64, 1) == 0
    assert lib.fwa_sequence_backward_workspace_bytes(N, L, L, H, H, 64, 0, 1, 0) == 0
