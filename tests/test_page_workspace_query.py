"""The workspace of the attention over a paged cache goes by the sizes alone: large pages of many heads, whose distance would not fit if the heads lay inside them, are asked for like
any others (no GPU needed)."""
import pytest

from paper_2501_06480_amd import binding as b
from test_page_abi import forward
from test_sequence_abi import P, S, lib  # noqa: F401


@pytest.mark.parametrize("dtype", [0, 1, 2])
@pytest.mark.parametrize("rows,most", [(1, 1), (3, 1), (200, 200), (203, 150)])
@pytest.mark.parametrize("kv,size,d", [(128, 65536, 128), (64, 65536, 128), (256, 32768, 128), (512, 65536, 32), (1024, 65536, 64), (2, 64, 64)])
def test_the_query_has_what_the_call_demands(lib, kv, size, d, rows, most, dtype):  # noqa: F811
    N, width = (rows if most == 1 else 1 if rows == most else 4), 4
    need = lib.fwa_page_forward_workspace_bytes(rows, N, kv, kv, d, size, width, most, dtype)
    # the same places in smaller pages
    assert need == lib.fwa_page_forward_workspace_bytes(rows, N, kv, kv, d, 16, width * size // 16, most, dtype)
    # one page (its distance to the next is none), and four with the heads outermost: the call wants no more and no less
    apart = 1 << 36  # bytes
    for layout in (dict(pages=1, ps=0, ts=kv * d, hs=d), dict(pages=4, ps=size * d, ts=d, hs=4 * size * d)):
        at = dict(q=P, o=P + S * 16, kp=P + apart, vp=P + 2 * apart, size=size, width=width, table=P + 32 * S, offsets=P + 33 * S, lengths=P + 34 * S, **layout)
        call = dict(rows=rows, N=N, H=kv, KV=kv, d=d, most=most, dtype=dtype)
        if need > 0:
            assert forward(lib, ws=P + 64 * S, ws_bytes=need - 1, **call, **at) == b.FWA_ERR_WORKSPACE
            assert forward(lib, **call, **at) == b.FWA_ERR_WORKSPACE
    if size == 65536 and kv <= 128 and rows == 1:  # (256 keys are too few to be shared out)
        assert need > 0
