"""Refusals of the rotary positions and of the operators on a paged cache, and what the host side of them computes (no GPU needed)."""
import pytest
import torch

from paper_2501_06480_amd import binding as b
from test_sequence_abi import P, S, lib  # noqa: F401


def rotary(lib, x=P, y=P + S, rows=100, heads=4, d=64, ldx=None, ldy=None, positions=P + 2 * S, period=100, axes=2, frequencies=P + 3 * S, axis_of=P + 4 * S, pairs=32,
           dtype=1):
    C = heads * d
    return lib.fwa_rotary(x, y, rows, heads, d, C if ldx is None else ldx, C if ldy is None else ldy, positions, period, axes, frequencies, axis_of, pairs, 0, 0, dtype,
                          None)


CACHE = dict(pages=20, size=16, ps=16 * 128, ts=128, hs=64, table=P + 6 * S, width=8, offsets=P + 7 * S, lengths=P + 8 * S)


def append(lib, k=P, v=P + S, kp=P + 2 * S, vp=P + 3 * S, rows=100, N=3, KV=2, d=64, ldk=None, ldv=None, positions=None, axes=1, frequencies=P + 9 * S, axis_of=None,
           pairs=32, q=P + 4 * S, q_out=P + 5 * S, heads=4, ldq=None, ldo=None, dtype=1, **cache):
    c, pick = {**CACHE, **cache}, lambda x, y: y if x is None else x
    return lib.fwa_page_append(k, v, kp, vp, rows, N, KV, d, pick(ldk, KV * d), pick(ldv, KV * d), c["pages"], c["size"], c["ps"], c["ts"], c["hs"], c["table"], c["width"],
                               c["offsets"], c["lengths"], positions, axes, frequencies, axis_of, pairs, 0, q, q_out, heads, pick(ldq, heads * d), pick(ldo, heads * d), dtype,
                               None)


def forward(lib, q=P, kp=P + 2 * S, vp=P + 3 * S, o=P + S, stats=None, rows=100, N=3, H=4, KV=2, d=64, ldq=None, ldo=None, most=100, dtype=1, ws=None, ws_bytes=0, **cache):
    c, pick = {**CACHE, **cache}, lambda x, y: y if x is None else x
    return lib.fwa_page_forward(q, kp, vp, o, stats, rows, N, H, KV, d, 0.1, pick(ldq, H * d), pick(ldo, H * d), c["pages"], c["size"], c["ps"], c["ts"], c["hs"],
                                c["table"], c["width"], c["offsets"], c["lengths"], most, 1, dtype, ws, ws_bytes, None)


def test_rotary_refuses_bad_arguments(lib):  # noqa: F811
    assert rotary(lib, rows=-1) == b.FWA_ERR_SHAPE
    assert rotary(lib, heads=0) == b.FWA_ERR_SHAPE
    assert rotary(lib, d=0) == b.FWA_ERR_SHAPE
    assert rotary(lib, pairs=33) == b.FWA_ERR_SHAPE
    assert rotary(lib, pairs=-1) == b.FWA_ERR_SHAPE
    assert rotary(lib, axes=0) == b.FWA_ERR_SHAPE
    assert rotary(lib, period=0) == b.FWA_ERR_SHAPE
    assert rotary(lib, ldx=255) == b.FWA_ERR_SHAPE
    assert rotary(lib, dtype=3) == b.FWA_ERR_UNSUPPORTED
    assert rotary(lib, d=516, heads=1) == b.FWA_ERR_UNSUPPORTED
    assert rotary(lib, axes=17) == b.FWA_ERR_UNSUPPORTED
    assert rotary(lib, heads=1 << 16) == b.FWA_ERR_UNSUPPORTED
    assert rotary(lib, rows=1 << 31) == b.FWA_ERR_UNSUPPORTED
    assert rotary(lib, rows=1 << 29, period=1) == b.FWA_ERR_UNSUPPORTED  # more units than a launch has
    assert rotary(lib, ldy=260) == b.FWA_ERR_ALIGN
    assert rotary(lib, x=P + 8) == b.FWA_ERR_ALIGN
    assert rotary(lib, positions=P + 2 * S + 2) == b.FWA_ERR_ALIGN
    assert rotary(lib, frequencies=P + 3 * S + 1) == b.FWA_ERR_ALIGN
    assert rotary(lib, axis_of=P + 4 * S + 3) == b.FWA_ERR_ALIGN
    for name in ("x", "y", "positions", "frequencies"):
        assert rotary(lib, **{name: None}) == b.FWA_ERR_NULL
    assert rotary(lib, rows=0, x=None, y=None) == b.FWA_OK
    # on top of its inputs, but for x itself: in place (not launched here)
    assert rotary(lib, y=P + 64) == b.FWA_ERR_ALIAS
    assert rotary(lib, y=P, ldy=512) == b.FWA_ERR_ALIAS
    for at in (2, 3, 4):
        assert rotary(lib, y=P + at * S) == b.FWA_ERR_ALIAS


@pytest.mark.parametrize("call", [append, forward])
def test_paged_calls_refuse_bad_arguments(lib, call):  # noqa: F811
    heads = "heads" if call is append else "H"
    assert call(lib, rows=-1) == b.FWA_ERR_SHAPE
    assert call(lib, N=-1) == b.FWA_ERR_SHAPE
    assert call(lib, KV=3) == b.FWA_ERR_SHAPE
    assert call(lib, KV=0) == b.FWA_ERR_SHAPE
    assert call(lib, **{heads: 0}) == b.FWA_ERR_SHAPE
    assert call(lib, pages=-1) == b.FWA_ERR_SHAPE
    assert call(lib, width=-1) == b.FWA_ERR_SHAPE
    assert call(lib, size=0) == b.FWA_ERR_SHAPE
    assert call(lib, ldq=248) == b.FWA_ERR_SHAPE
    assert call(lib, d=48, hs=48) == b.FWA_ERR_UNSUPPORTED
    assert call(lib, dtype=7) == b.FWA_ERR_UNSUPPORTED
    assert call(lib, size=24) == b.FWA_ERR_UNSUPPORTED
    assert call(lib, size=1 << 17) == b.FWA_ERR_UNSUPPORTED
    assert call(lib, width=(1 << 25) + 1) == b.FWA_ERR_UNSUPPORTED
    assert call(lib, rows=(1 << 24) + 1) == b.FWA_ERR_UNSUPPORTED
    assert call(lib, N=(1 << 20) + 1) == b.FWA_ERR_UNSUPPORTED
    assert call(lib, ts=(1 << 20) + 8, ps=1 << 30) == b.FWA_ERR_UNSUPPORTED
    assert call(lib, ps=(1 << 29) + 8) == b.FWA_ERR_UNSUPPORTED
    # strides: multiples of 16 bytes that reach no element twice, in any order
    assert call(lib, ts=132) == b.FWA_ERR_ALIGN
    assert call(lib, ps=-16) == b.FWA_ERR_SHAPE
    assert call(lib, ts=64) == b.FWA_ERR_SHAPE
    assert call(lib, hs=0) == b.FWA_ERR_SHAPE
    assert call(lib, ps=0) == b.FWA_ERR_SHAPE
    assert call(lib, ps=16 * 128 - 16) == b.FWA_ERR_SHAPE
    for name in ("q", "kp", "vp", "table", "offsets", "lengths"):
        if not (name == "q" and call is append):
            assert call(lib, **{name: None}) == b.FWA_ERR_NULL, name
    assert call(lib, kp=P + 2 * S + 8) == b.FWA_ERR_ALIGN
    for name in ("table", "offsets", "lengths"):
        assert call(lib, **{name: CACHE[name] + 2}) == b.FWA_ERR_ALIGN
    assert call(lib, rows=0) == b.FWA_OK
    assert call(lib, N=0) == b.FWA_OK


def test_append_refuses_overlaps(lib):  # noqa: F811
    assert append(lib, q_out=None) == b.FWA_ERR_NULL
    assert append(lib, k=None) == b.FWA_ERR_NULL
    assert append(lib, pairs=33) == b.FWA_ERR_SHAPE
    assert append(lib, positions=P + 10 * S, axes=0) == b.FWA_ERR_SHAPE
    assert append(lib, positions=P + 10 * S, axes=17) == b.FWA_ERR_UNSUPPORTED
    assert append(lib, positions=P + 10 * S + 2) == b.FWA_ERR_ALIGN
    assert append(lib, frequencies=None) == b.FWA_ERR_NULL
    for at in (P, P + S, P + 4 * S, P + 9 * S, *(CACHE[n] for n in ("table", "offsets", "lengths"))):
        assert append(lib, kp=at) == b.FWA_ERR_ALIAS, at
        assert append(lib, vp=at) == b.FWA_ERR_ALIAS, at
    for at in (P, P + S, P + 2 * S, P + 3 * S, P + 4 * S + 64, P + 9 * S, CACHE["table"]):
        assert append(lib, q_out=at) == b.FWA_ERR_ALIAS, at
    assert append(lib, positions=P + 2 * S) == b.FWA_ERR_ALIAS
    # keys and values of one buffer: [pages, 2, page, kv, d], [pages, page, 2, kv, d], [pages, page, kv, 2, d], [2, ...]; a row nearer than that
    two = P + 2 * S
    for ps, ts, hs, apart in ((2 * 2048, 128, 64, 2048), (2 * 2048, 256, 64, 128), (2 * 2048, 256, 128, 64), (2048, 128, 64, 20 * 2048)):
        far = dict(kp=two, ps=ps, ts=ts, hs=hs, q_out=P + 40 * S)
        assert append(lib, vp=two + 2 * apart - 16, **far) == b.FWA_ERR_ALIAS
        assert append(lib, vp=two + 16, **far) == b.FWA_ERR_ALIAS
        assert append(lib, vp=two, **far) == b.FWA_ERR_ALIAS
        # apart: past the test of keys against values, stopped by that of the queries
        assert append(lib, vp=two + 2 * apart, **{**far, "q_out": P}) == b.FWA_ERR_ALIAS


def test_forward_refuses_overlaps_and_small_workspaces(lib):  # noqa: F811
    assert forward(lib, most=-1) == b.FWA_ERR_SHAPE
    assert forward(lib, most=0) == b.FWA_OK
    for at in (P, P + 64, P + 2 * S, P + 3 * S, *(CACHE[n] for n in ("table", "offsets", "lengths"))):
        assert forward(lib, o=at) == b.FWA_ERR_ALIAS, at
        assert forward(lib, stats=at) == b.FWA_ERR_ALIAS, at
    assert forward(lib, stats=P + S + 16) == b.FWA_ERR_ALIAS
    assert forward(lib, stats=P + 4 * S + 4) == b.FWA_ERR_ALIGN
    need = lib.fwa_page_forward_workspace_bytes(3, 3, 4, 2, 64, 16, 1000, 1, 1)
    assert need > 0
    assert forward(lib, rows=3, most=1, width=1000, ws=P + 40 * S, ws_bytes=need - 1) == b.FWA_ERR_WORKSPACE
    assert forward(lib, rows=3, most=1, width=1000) == b.FWA_ERR_WORKSPACE
    assert lib.fwa_page_forward_workspace_bytes(3, 3, 4, 2, 48, 16, 1000, 1, 1) == 0
    assert lib.fwa_page_forward_workspace_bytes(3, 3, 4, 2, 64, 8, 1000, 1, 1) == 0
    assert lib.fwa_page_forward_workspace_bytes(3, 3, 4, 2, 64, 16, 2, 1, 1) == 0  # too short to be shared out
    # an interleaved head layout: heads outermost of all
    assert forward(lib, hs=20 * 16 * 64, ps=16 * 64, ts=64, o=P) == b.FWA_ERR_ALIAS


def test_rotary_frequencies():
    f, axis = b.rotary_frequencies((2, 4))
    assert axis.tolist() == [0, 0, 1, 1, 1, 1] and axis.dtype == torch.int32
    assert torch.allclose(f, torch.tensor([1, 0.01, 1, 0.1, 0.01, 0.001]), rtol=1e-6)
    f, axis = b.rotary_frequencies((1, 0, 3), joint=True)
    assert axis.tolist() == [0, 2, 2, 2] and torch.allclose(f, torch.tensor([1, 0.1, 0.01, 0.001]), rtol=1e-6)
    for bad in ((), (-1, 2)):
        with pytest.raises(ValueError):
            b.rotary_frequencies(bad)
    with pytest.raises(ValueError):
        b.rotary_frequencies((4,), theta=0.0)


def test_bindings_refuse_cpu_tensors():
    import paper_2501_06480_amd as fwa
    x, i = torch.zeros(4, 128), torch.zeros(4, 1, dtype=torch.int32)
    with pytest.raises(TypeError):
        fwa.fwa_rotary(x, 2, i, torch.ones(32))
    pool, one = torch.zeros(2, 16, 2, 64), torch.zeros(1, dtype=torch.int32)
    tables = (pool, pool.clone(), torch.zeros(1, 2, dtype=torch.int32), torch.zeros(2, dtype=torch.int32), one)
    with pytest.raises(TypeError):
        fwa.fwa_page_append(x, x, *tables)
    with pytest.raises(TypeError):
        fwa.fwa_page_forward(x, *tables, 2, 0.1)
