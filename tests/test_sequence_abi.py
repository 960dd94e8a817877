"""Refusals of the bias by buckets and of the attention of whole sequences, and what the host side of them computes (no GPU needed)."""
import pytest
import torch

from paper_2501_06480_amd import binding as b

P = 0x10000000  # stands for a device pointer; never dereferenced on error paths
S = 0x1000000


@pytest.fixture(scope="module")
def lib():
    import os
    if not os.path.exists(b.library_path()):
        from paper_2501_06480_amd import build
        build.build(verbose=False)
    return b.load_library()


def test_bucket_calls_refuse_bad_arguments(lib):
    def gather(table=P, buckets=P + S, bias=P + 2 * S, heads=4, columns=32, far=128, Lq=10, Lk=10, dtype=0):
        return lib.fwa_bucket_gather(table, buckets, bias, heads, columns, far, Lq, Lk, 0, dtype, None)

    def scatter(dbias=P, buckets=P + S, dtable=P + 2 * S, heads=4, columns=32, far=128, Lq=10, Lk=10, ws=P + 3 * S, ws_bytes=1 << 24):
        return lib.fwa_bucket_scatter(dbias, buckets, dtable, heads, columns, far, Lq, Lk, 0, ws, ws_bytes, None)
    for call in (gather, scatter):
        assert call(heads=0) == b.FWA_ERR_SHAPE
        assert call(columns=0) == b.FWA_ERR_SHAPE
        assert call(far=-1) == b.FWA_ERR_SHAPE
        assert call(Lq=-1) == b.FWA_ERR_SHAPE
        assert call(far=b.FWA_BUCKET_MAX_FAR + 1) == b.FWA_ERR_UNSUPPORTED
        assert call(columns=(1 << 16) + 1) == b.FWA_ERR_UNSUPPORTED
        assert call(Lk=(1 << 24) + 1) == b.FWA_ERR_UNSUPPORTED
        assert call(heads=1 << 15, Lq=1 << 14) == b.FWA_ERR_UNSUPPORTED
        assert call(buckets=None) == b.FWA_ERR_NULL
        assert call(buckets=P + S + 2) == b.FWA_ERR_ALIGN
    assert gather(dtype=2) == b.FWA_ERR_UNSUPPORTED
    assert gather(table=None) == b.FWA_ERR_NULL
    assert gather(bias=P + 4) == b.FWA_ERR_ALIGN
    assert gather(bias=P) == b.FWA_ERR_ALIAS
    assert gather(Lq=0, table=None) == b.FWA_OK
    assert scatter(dtable=None) == b.FWA_ERR_NULL
    assert scatter(dbias=P + 8) == b.FWA_ERR_ALIGN
    assert scatter(dtable=P) == b.FWA_ERR_ALIAS
    need = lib.fwa_bucket_scatter_workspace_bytes(4, 32, 128, 10, 10)
    assert need > 0 and scatter(ws_bytes=need - 1) == b.FWA_ERR_WORKSPACE and scatter(ws=None) == b.FWA_ERR_WORKSPACE
    assert lib.fwa_bucket_scatter_workspace_bytes(4, 32, -1, 10, 10) == 0


def forward(lib, q=P, k=P + S, v=P + 2 * S, o=P + 3 * S, stats=None, N=2, Lq=100, Lk=100, H=4, KV=2, d=64, ldq=None, ldkv=None, ldo=None, table=None,
            buckets=None, columns=0, far=0, ql=None, kl=None, start=None, dtype=1, ws=None, ws_bytes=0):
    C, CK = H * d, KV * d
    return lib.fwa_sequence_forward(q, k, v, o, stats, N, Lq, Lk, H, KV, d, 0.125, C if ldq is None else ldq, CK if ldkv is None else ldkv,
                                    C if ldo is None else ldo, table, buckets, columns, far, ql, kl, start, 0, dtype, ws, ws_bytes, None)


def backward(lib, q=P, k=P + S, v=P + 2 * S, o=P + 3 * S, g=P + 4 * S, stats=P + 5 * S, dq=P + 6 * S, dk=P + 7 * S, dv=P + 8 * S, dtable=None, N=2, Lq=100,
             Lk=100, H=4, KV=2, d=64, lds=None, table=None, buckets=None, columns=0, far=0, dtype=1, ws=P + 9 * S, ws_bytes=1 << 30):
    C, CK = H * d, KV * d
    return lib.fwa_sequence_backward(q, k, v, o, g, stats, dq, dk, dv, dtable, N, Lq, Lk, H, KV, d, 0.125, *(lds or (C, CK, C, C, C, CK)), table, buckets, columns,
                                     far, None, None, None, 0, dtype, ws, ws_bytes, None)


@pytest.mark.parametrize("call", [forward, backward])
def test_sequence_calls_refuse_bad_arguments(lib, call):
    assert call(lib, N=-1) == b.FWA_ERR_SHAPE
    assert call(lib, Lq=-1) == b.FWA_ERR_SHAPE
    assert call(lib, KV=3) == b.FWA_ERR_SHAPE
    assert call(lib, KV=0) == b.FWA_ERR_SHAPE
    assert call(lib, d=48) == b.FWA_ERR_UNSUPPORTED
    assert call(lib, d=256) == b.FWA_ERR_UNSUPPORTED
    assert call(lib, dtype=3) == b.FWA_ERR_UNSUPPORTED
    assert call(lib, Lk=(1 << 24) + 1) == b.FWA_ERR_UNSUPPORTED
    assert call(lib, N=1 << 40) == b.FWA_ERR_UNSUPPORTED
    assert call(lib, q=None) == b.FWA_ERR_NULL
    assert call(lib, v=None) == b.FWA_ERR_NULL
    assert call(lib, k=P + S + 8) == b.FWA_ERR_ALIGN
    assert call(lib, table=P + 20 * S, columns=32, far=4) == b.FWA_ERR_NULL                      # no map
    assert call(lib, table=P + 20 * S, buckets=P + 21 * S, columns=0, far=4) == b.FWA_ERR_SHAPE
    assert call(lib, table=P + 20 * S, buckets=P + 21 * S, columns=8, far=9000) == b.FWA_ERR_UNSUPPORTED
    assert call(lib, table=P + 20 * S + 2, buckets=P + 21 * S, columns=8, far=4) == b.FWA_ERR_ALIGN


def test_sequence_strides_and_overlaps(lib):
    assert forward(lib, ldq=255) == b.FWA_ERR_SHAPE
    assert forward(lib, ldkv=130) == b.FWA_ERR_ALIGN
    assert forward(lib, ldo=1 << 21) == b.FWA_ERR_UNSUPPORTED
    assert forward(lib, o=P + 64) == b.FWA_ERR_ALIAS
    assert forward(lib, o=P + S) == b.FWA_ERR_ALIAS
    assert forward(lib, stats=P + 3 * S + 16) == b.FWA_ERR_ALIAS
    assert forward(lib, N=0, q=None) == b.FWA_OK
    assert forward(lib, Lq=0, q=None) == b.FWA_OK
    assert backward(lib, dq=P) == b.FWA_ERR_ALIAS
    assert backward(lib, dk=P + 8 * S) == b.FWA_ERR_ALIAS
    assert backward(lib, dtable=P + 30 * S) == b.FWA_ERR_NULL                                        # no table
    assert backward(lib, table=P + 20 * S, buckets=P + 21 * S, columns=8, far=4, dtable=P + 20 * S) == b.FWA_ERR_ALIAS
    assert backward(lib, lds=(256, 128, 256, 256, 256, 64)) == b.FWA_ERR_SHAPE
    # parts of unequal width of one buffer [N, L, (4 + 2 + 2) 64]: past the overlap test, stopped by the workspace
    G, C = P + 40 * S, 512
    assert backward(lib, dq=G, dk=G + 512, dv=G + 768, lds=(256, 128, 256, 256, C, C), ws=None) == b.FWA_ERR_WORKSPACE
    assert backward(lib, dq=G, dk=G + 496, dv=G + 768, lds=(256, 128, 256, 256, C, C), ws=None) == b.FWA_ERR_ALIAS
    assert backward(lib, dq=G, dk=G + 512, dv=G + 784, lds=(256, 128, 256, 256, C, C), ws=None) == b.FWA_ERR_ALIAS  # into the next row of dq
    need = lib.fwa_sequence_backward_workspace_bytes(2, 100, 100, 4, 2, 64, 0, 1, 0)
    assert need >= 2 * 100 * 4 * 4 and backward(lib, ws_bytes=need - 1) == b.FWA_ERR_WORKSPACE


def test_split_form_asks_for_its_workspace(lib):
    need = lib.fwa_sequence_forward_workspace_bytes(1, 1, 8192, 8, 8, 64, 1)
    assert need > 0
    assert forward(lib, N=1, Lq=1, Lk=8192, H=8, KV=8, o=P + 30 * S, ws=P + 40 * S, ws_bytes=need - 1) == b.FWA_ERR_WORKSPACE
    assert lib.fwa_sequence_forward_workspace_bytes(4, 2048, 2048, 16, 16, 64, 1) == 0
    assert lib.fwa_sequence_forward_workspace_bytes(1, 1, 8192, 8, 8, 48, 1) == 0


def test_log_buckets():
    m = b.log_buckets(32, 128)
    assert m.dtype == torch.int32 and m.numel() == 257
    at = lambda d: int(m[128 + d])  # noqa: E731
    assert [at(-d) for d in (0, 1, 7, 8, 11, 12, 16, 32, 64, 128)] == [0, 1, 7, 8, 8, 9, 10, 12, 14, 15]  # 8 * 16^(t/8): borders 8, 11.3, 16, ...
    assert [at(d) - 16 for d in (1, 7, 8, 64, 128)] == [1, 7, 8, 14, 15]
    one_way = b.log_buckets(8, 16, bidirectional=False)
    assert one_way[16:].tolist() == [0] * 17 and one_way[:17].tolist()[::-1] == [0, 1, 2, 3, 4, 4, 5, 5, 6, 6, 6, 6, 7, 7, 7, 7, 7]  # 4 * 4^(t/4)
    for bad in ((1, 128), (32, 0), (32, 1 << 14), (64, 8)):
        with pytest.raises(ValueError):
            b.log_buckets(*bad)


def test_bindings_refuse_cpu_tensors():
    import paper_2501_06480_amd as fwa
    q = torch.zeros(2, 10, 64)
    with pytest.raises(TypeError):
        fwa.fwa_sequence_forward(q, q, q, 2, 0.1)
    with pytest.raises(TypeError):
        fwa.fwa_bucket_gather(torch.zeros(2, 8), torch.zeros(3, dtype=torch.int32), 4)
    with pytest.raises(TypeError):
        fwa.fwa_bucket_scatter(torch.zeros(2, 4, 4), torch.zeros(3, dtype=torch.int32), 8)
    with pytest.raises(TypeError):
        fwa.fwa_bucket_gather(torch.zeros(2, 8), torch.zeros(3, dtype=torch.int32), 4, dtype=torch.float16)
