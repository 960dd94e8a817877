"""Sizes at the ends of what the calls of sequences take (no GPU needed)."""
import pytest

from paper_2501_06480_amd import binding as b
from test_sequence_abi import P, S, backward, forward, lib  # noqa: F401


@pytest.mark.parametrize("call", [forward, backward])
def test_heads_times_width_beyond_32_bits(lib, call):  # noqa: F811
    assert call(lib, H=1 << 16, KV=1, d=1 << 16) == b.FWA_ERR_UNSUPPORTED
    assert call(lib, H=1 << 30, KV=1 << 30, d=1 << 30, Lq=0) == b.FWA_ERR_UNSUPPORTED
    assert call(lib, H=1 << 15, KV=1, d=128, Lq=1) == b.FWA_ERR_UNSUPPORTED  # rows of more than 2^20 elements
