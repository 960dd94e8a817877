"""Outputs of the sequence calls that share memory with any input or with each other are refused before anything is launched (no GPU needed)."""
import pytest

from paper_2501_06480_amd import binding as b
from test_sequence_abi import P, S, lib  # noqa: F401

TERMS = {"table": P + 20 * S, "buckets": P + 21 * S, "ql": P + 22 * S, "kl": P + 23 * S, "start": P + 24 * S}
N, L, H, KV, d, COLUMNS, FAR = 2, 100, 4, 2, 64, 32, 40
SIZES = {"table": 4 * H * COLUMNS, "buckets": 4 * (2 * FAR + 1), "ql": 4 * N, "kl": 4 * N, "start": 4 * N}


def forward(lib, q=P, k=P + S, v=P + 2 * S, o=P + 3 * S, stats=P + 4 * S, table=TERMS["table"], buckets=TERMS["buckets"], ql=TERMS["ql"], kl=TERMS["kl"],
            start=TERMS["start"]):
    return lib.fwa_sequence_forward(q, k, v, o, stats, N, L, L, H, KV, d, 0.125, H * d, KV * d, H * d, table, buckets, COLUMNS, FAR, ql, kl, start, 0, 1,
                                    P + 40 * S, 1 << 30, None)


def backward(lib, dq=P + 6 * S, dk=P + 7 * S, dv=P + 8 * S, dtable=P + 9 * S, table=TERMS["table"], buckets=TERMS["buckets"], ql=TERMS["ql"], kl=TERMS["kl"],
             start=TERMS["start"], n=N, ws=0):
    return lib.fwa_sequence_backward(P, P + S, P + 2 * S, P + 3 * S, P + 4 * S, P + 5 * S, dq, dk, dv, dtable, n, L, L, H, KV, d, 0.125, H * d, KV * d, H * d,
                                     H * d, H * d, KV * d, table, buckets, COLUMNS, FAR, ql, kl, start, 0, 1, P + 40 * S, ws, None)


@pytest.mark.parametrize("term", TERMS)
def test_outputs_on_top_of_the_terms(lib, term):  # noqa: F811
    at = TERMS[term]
    last = (at + SIZES[term] - 1) & ~15  # the last aligned place that still has one of its bytes
    for place in (at, last):
        for out in ("o", "stats"):
            assert forward(lib, **{out: place}) == b.FWA_ERR_ALIAS, (term, out)
        for out in ("dq", "dk", "dv", "dtable"):
            assert backward(lib, **{out: place}) == b.FWA_ERR_ALIAS, (term, out)
    # an output that ends inside the term
    assert forward(lib, o=at - N * L * H * d * 2 + 16) == b.FWA_ERR_ALIAS
    assert forward(lib, stats=at - N * L * H * 8 + 16) == b.FWA_ERR_ALIAS
    assert backward(lib, dk=at - N * L * KV * d * 2 + 16) == b.FWA_ERR_ALIAS
    assert backward(lib, dtable=at - 4 * H * COLUMNS + 16) == b.FWA_ERR_ALIAS


def test_outputs_next_to_the_terms_pass(lib):  # noqa: F811
    """Past the overlap test, stopped by the workspace."""
    after = {n: (TERMS[n] + SIZES[n] + 15) & ~15 for n in TERMS}
    for place in after.values():
        for out in ("dq", "dk", "dv", "dtable"):
            assert backward(lib, **{out: place}) == b.FWA_ERR_WORKSPACE
    assert backward(lib, ql=TERMS["kl"]) == b.FWA_ERR_WORKSPACE  # inputs may be one


def test_gradient_of_the_table_of_no_sequences(lib):  # noqa: F811
    """N == 0 writes dtable too."""
    assert backward(lib, n=0, dtable=TERMS["table"]) == b.FWA_ERR_ALIAS
    assert backward(lib, n=0, dtable=TERMS["buckets"]) == b.FWA_ERR_ALIAS


def test_outputs_on_top_of_each_other(lib):  # noqa: F811
    assert forward(lib, stats=P + 3 * S + 64) == b.FWA_ERR_ALIAS
    for x, y in (("dq", 7), ("dk", 8), ("dv", 9), ("dtable", 6)):
        assert backward(lib, **{x: P + y * S}) == b.FWA_ERR_ALIAS
