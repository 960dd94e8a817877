"""Pairs whose axis lies outside the axes stay as they are, whatever they hold: infinities and NaN of one channel do not reach the other, zeros keep their signs."""
import pytest
import torch

import page_reference as ref
import test_gpu_page_append as append
from test_gpu_rotary import BF16, F16, F32, make

pytestmark = pytest.mark.gpu

INTS = {F32: torch.int32, BF16: torch.int16, F16: torch.int16}


def channels(pairs, stay, interleaved):
    """(first, second) channel of the pairs that stay"""
    p = torch.arange(pairs)[stay]
    return (2 * p, 2 * p + 1) if interleaved else (p, p + pairs)


def fill(x, first, second, dtype):
    """x [rows, d]: values of all kinds in pairs that stay, each beside a plain one and beside each other"""
    odd = torch.tensor([float("inf"), -float("inf"), float("nan"), -0.0, 0.0, torch.finfo(dtype).max, torch.finfo(dtype).tiny, -1.5]).to(dtype)
    for r in range(x.shape[0]):
        x[r, first] = odd[(torch.arange(len(first)) + r) % 8]
        x[r, second] = odd[(torch.arange(len(second)) * 3 + r // 8) % 8]


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,pairs", [(64, 32), (64, 24), (72, 36), (24, 5)])  # vectors of 16 and of 8 bytes, single elements
def test_pairs_without_an_axis_stay(dtype, interleaved, d, pairs):
    import paper_2501_06480_amd as fwa
    N, L, H = 2, 65, 8
    x, positions, f, _, g = make(dtype, N, L, H, d, (pairs - 2, 2))
    axis = torch.randint(0, 2, (pairs,), generator=g, dtype=torch.int32)
    axis[::3], axis[1::5] = -1, 2
    stay = (axis < 0) | (axis > 1)
    first, second = channels(pairs, stay, interleaved)
    for at in x.view(N * L, H, d).unbind(1):
        fill(at, first, second, dtype)
    for inverse in (False, True):
        got = fwa.fwa_rotary(x.cuda(), H, positions.cuda(), f.cuda(), axis.cuda(), interleaved, inverse).cpu().view(N, L, H, d)
        for at in (first, second):
            have, want = got[..., at].contiguous(), x.view(N, L, H, d)[..., at].contiguous()
            same = have.view(INTS[dtype]) == want.view(INTS[dtype])
            assert bool((same | (torch.isnan(have) & torch.isnan(want))).all())
        # the others as ever
        plain = x.clone().view(N, L, H, d)
        plain[..., torch.cat((first, second))] = 0.0
        want, tol = (t.view(N, L, H, d) for t in ref.rotate(plain.view(x.shape), H, positions, f, axis, interleaved, inverse))
        rest = torch.ones(d, dtype=torch.bool)
        rest[torch.cat((first, second))] = False
        ref.check(got[..., rest], want[..., rest], tol[..., rest], f"{dtype} {d} {pairs}")


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_keys_and_queries_of_an_append_stay(dtype):
    H, KV, d, size, news = 4, 2, 64, 16, [1, 30]
    x, _ = append.make(dtype, news, [3, 20], H, KV, d, size, sections=(20, 12))
    x["axis_of"][::4] = 9
    first, second = channels(32, x["axis_of"] == 9, False)
    for at in x["fused"].view(31, H + 2 * KV, d)[:, :H + KV].unbind(1):
        fill(at, first, second, dtype)
    y = append.device(x)
    q = append.call(y, H, KV, d).cpu().view(31, H, d)
    here = torch.cat((first, second))
    rows = x["fused"].view(31, H + 2 * KV, d)
    assert torch.equal(q[..., here].nan_to_num(7.0, 8.0, 9.0), rows[:, :H, here].nan_to_num(7.0, 8.0, 9.0))
    for n, t in enumerate([0] + [1] * 30):
        place = 3 if n == 0 else 20 + n - 1
        key = y["k_pages"][int(x["page_table"][t, place // size]), place % size].cpu()
        assert torch.equal(key[:, here].nan_to_num(7.0, 8.0, 9.0), rows[n, H:H + KV, here].nan_to_num(7.0, 8.0, 9.0))
