"""Rotary positions against 64 bits (tests/page_reference.py, whose bounds follow from the arithmetic): types, head widths whole and in part, axes, both kinds of
pairs, odd rows, strides, places, gradients, streams and graphs."""
import pytest
import torch

import page_reference as ref

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32


def make(dtype, N, L, heads, d, sections, shared=True, far=0, seed=0, joint=False):
    from paper_2501_06480_amd import binding
    g = torch.Generator().manual_seed(seed + 31 * L + d + len(sections))
    x = torch.randn(N, L, heads * d, generator=g).to(dtype)
    positions = torch.randint(far, far + 5000, (*(() if shared else (N,)), L, len(sections)), generator=g, dtype=torch.int32)
    return x, positions, *binding.rotary_frequencies(sections, joint=joint), g


CASES = [  # dtype, N, L, heads, d, sections, interleaved, shared
    (F16, 64, 49, 3, 32, (8, 8), False, True),
    (BF16, 2, 100, 16, 128, (16, 24, 24), False, True),
    (BF16, 3, 77, 5, 64, (32,), True, False),
    (F32, 1, 333, 12, 64, (24,), True, True),
    (F32, 2, 19, 3, 128, (40, 24), False, False),
    (BF16, 1, 1, 1, 32, (16,), False, True),
    (BF16, 2, 65, 4, 72, (18, 18), False, True),       # 8-byte vectors
    (F16, 2, 65, 4, 72, (12, 12, 4), True, False),
    (BF16, 1, 53, 2, 64, (13, 8), False, True),        # single elements
    (F16, 1, 53, 8, 40, (7,), True, True),
    (F32, 1, 53, 8, 24, (5, 6), False, False),
    (BF16, 1, 37, 8, 24, (8,), False, True),           # eight channels behind the pairs: half a unit
    (F16, 2, 30, 2, 256, (64, 64), False, True),
    (F32, 1, 9, 1, 512, (100, 100, 56), True, True),
    (BF16, 1, 2000, 1, 16, (8,), False, True),
    (BF16, 1, 11, 8, 1, (), False, True),              # no pair
    (F32, 1, 7, 4, 5, (1,), True, True),
    (BF16, 2, 33, 2, 64, (0, 32, 0), False, True),
]


@pytest.mark.parametrize("dtype,N,L,heads,d,sections,interleaved,shared", CASES)
@pytest.mark.parametrize("inverse", [False, True])
def test_rotation(dtype, N, L, heads, d, sections, interleaved, shared, inverse):
    import paper_2501_06480_amd as fwa
    x, positions, f, axis, _ = make(dtype, N, L, heads, d, sections or (0,), shared)
    got = fwa.fwa_rotary(x.cuda(), heads, positions.cuda(), f.cuda(), axis.cuda(), interleaved, inverse)
    want, tol = ref.rotate(x, heads, positions, f, axis, interleaved, inverse)
    ref.check(got, want, tol, f"{dtype} {d} {sections}")
    assert got.dtype == dtype


@pytest.mark.parametrize("far", [-(1 << 31), -7, 1 << 20, (1 << 31) - 5000])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_far_positions(dtype, far):
    import paper_2501_06480_amd as fwa
    x, positions, f, axis, _ = make(dtype, 1, 200, 2, 64, (32,), far=far)
    ref.check(fwa.fwa_rotary(x.cuda(), 2, positions.cuda(), f.cuda()), *ref.rotate(x, 2, positions, f), f"from {far}")


def test_axes_outside_leave_their_pairs():
    import paper_2501_06480_amd as fwa
    x, positions, f, axis, _ = make(BF16, 2, 40, 2, 64, (16, 16))
    axis[::3] = -1
    axis[1::5] = 2
    axis[7] = 1 << 30
    got = fwa.fwa_rotary(x.cuda(), 2, positions.cuda(), f.cuda(), axis.cuda())
    ref.check(got, *ref.rotate(x, 2, positions, f, axis), "axes outside")


@pytest.mark.parametrize("dtype", [F32, F16])
def test_views_places_and_packed_rows(dtype):
    import paper_2501_06480_amd as fwa
    N, L, H, d = 2, 45, 3, 64
    x, positions, f, axis, g = make(dtype, N, L, H, d, (20, 8))
    fused = torch.randn(N, L, 3 * H * d, generator=g).to(dtype).cuda()
    before = fused.clone()
    part = fused[..., H * d:2 * H * d]
    want, tol = ref.rotate(part.cpu(), H, positions, f, axis)
    args = (H, positions.cuda(), f.cuda(), axis.cuda())
    got = fwa.fwa_rotary(part, *args)
    ref.check(got, want, tol, "view")
    out = torch.full_like(fused, 7.0)
    fwa.fwa_rotary(part, *args, out=out[..., :H * d])
    assert torch.equal(out[..., :H * d], got) and bool((out[..., H * d:] == 7.0).all())
    assert fwa.fwa_rotary(part, *args, out=part) is part  # in place
    assert torch.equal(part, got) and torch.equal(fused[..., :H * d], before[..., :H * d]) and torch.equal(fused[..., 2 * H * d:], before[..., 2 * H * d:])
    packed = before[0, :, H * d:2 * H * d]
    assert torch.equal(fwa.fwa_rotary(packed, *args), got[0])
    for empty in (x[:0], x[:, :0]):
        assert fwa.fwa_rotary(empty.cuda(), H, positions[:empty.shape[1]].cuda(), f.cuda(), axis.cuda()).shape == empty.shape


@pytest.mark.parametrize("native", [True, False])
@pytest.mark.parametrize("dtype,interleaved", [(F32, False), (BF16, True)])
def test_gradient(native, dtype, interleaved):
    """The gradient is the rotation back: against the formula, and (fp32) against differences of the output."""
    from paper_2501_06480_amd import autograd
    N, L, H, d = 2, 21, 2, 32
    x, positions, f, axis, g = make(dtype, N, L, H, d, (6, 8), shared=False)
    dy = torch.randn(N, L, H * d, generator=g).to(dtype)
    xd = x.cuda().requires_grad_(True)
    args = (positions.cuda(), f.cuda(), axis.cuda())
    call = (lambda t: autograd.rotary(t, H, *args, interleaved)) if native else (lambda t: autograd._Rotary.apply(t, *args, H, interleaved, False))
    y = call(xd)
    y.backward(dy.cuda())
    ref.check(xd.grad, *ref.rotate(dy, H, positions, f, axis, interleaved, True), "gradient")
    if dtype == F32:
        # y is linear in x: a difference of two outputs along a direction, 2^-24 of values around 4 in each of them
        v = torch.randn(N, L, H * d, generator=g)
        by_difference = ((call((x + v).cuda()).double() - call((x - v).cuda()).double()) / 2 * dy.cuda().double()).sum()
        along = (xd.grad.double() * v.cuda().double()).sum()
        assert abs(float(by_difference - along)) <= 32 * ref.U32 * float((dy.abs().double() * (x.abs() + v.abs() + 8)).sum())
    # an expanded gradient, and one that starts at an odd element of a larger one
    one, = torch.autograd.grad(call(xd).sum(), xd)
    ref.check(one, *ref.rotate(torch.ones_like(dy), H, positions, f, axis, interleaved, True), "of a sum")
    wide = torch.randn(N * L * H * d + 1, generator=g).to(dtype).cuda()
    odd, = torch.autograd.grad(call(xd), xd, wide[1:].view(N, L, H * d))
    ref.check(odd, *ref.rotate(wide[1:].cpu().view(N, L, H * d), H, positions, f, axis, interleaved, True), "odd place")


@pytest.mark.parametrize("native", [True, False])
def test_gradient_of_a_gradient(native):
    """f = |g|^2 / 2 with g = dx of sum(w y): of turns alone g has the length of w, so df/dw = w, up to the errors of two turns."""
    from paper_2501_06480_amd import autograd
    x, positions, f, axis, g = make(F32, 2, 9, 2, 32, (8, 8))
    args = (positions.cuda(), f.cuda(), axis.cuda())
    xd, w = x.cuda().requires_grad_(True), torch.randn(x.shape, generator=g).cuda().requires_grad_(True)
    y = autograd.rotary(xd, 2, *args, True) if native else autograd._Rotary.apply(xd, *args, 2, True, False)
    dx, = torch.autograd.grad((w * y).sum(), xd, create_graph=True)
    assert dx.requires_grad
    dw, = torch.autograd.grad((dx * dx).sum() / 2, w)
    # a turn is off by 10 U32 of |a| + |b| at most; the first's error through the second, and the second's of a turned pair: sqrt 2 of that each
    pair = w.detach().abs().view(2, 9, 2, 16, 2).sum(-1, keepdim=True).expand(2, 9, 2, 16, 2).reshape(w.shape)
    assert bool(((dw - w.detach()).abs() <= 32 * ref.U32 * pair).all())


def test_forward_mode_and_transforms_go_the_python_way():
    from paper_2501_06480_amd import autograd
    x, positions, f, axis, _ = make(F32, 2, 5, 1, 32, (16,))
    args = (1, positions.cuda(), f.cuda())
    with pytest.raises(Exception):
        torch.func.jvp(lambda t: autograd.rotary(t, *args), (x.cuda(),), (x.cuda(),))


def test_streams_and_graphs():
    import paper_2501_06480_amd as fwa
    x, positions, f, axis, g = make(BF16, 2, 300, 4, 64, (16, 16))
    xd, pd, fd, ad = x.cuda(), positions.cuda(), f.cuda(), axis.cuda()
    want = fwa.fwa_rotary(xd, 4, pd, fd, ad)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = fwa.fwa_rotary(xd, 4, pd, fd, ad, stream=side)
    side.synchronize()
    assert torch.equal(got, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        y = fwa.fwa_rotary(xd, 4, pd, fd, ad, stream=torch.cuda.current_stream())
        z = fwa.fwa_rotary(y, 4, pd, fd, ad, inverse=True, stream=torch.cuda.current_stream())
    for _ in range(3):
        xd.copy_(torch.randn(x.shape, generator=g).to(BF16))
        pd.copy_(torch.randint(0, 9000, positions.shape, generator=g, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        a, b = y.clone(), z.clone()
        y.fill_(7.0)
        z.fill_(7.0)
        assert torch.equal(a, fwa.fwa_rotary(xd, 4, pd, fd, ad)) and torch.equal(b, fwa.fwa_rotary(a, 4, pd, fd, ad, inverse=True))


def test_refusals():
    import paper_2501_06480_amd as fwa
    x, positions, f, axis, _ = make(BF16, 2, 40, 2, 64, (32,))
    x, p, f, a = x.cuda(), positions.cuda(), f.cuda(), axis.cuda()
    for bad in (lambda: fwa.fwa_rotary(x, 3, p, f), lambda: fwa.fwa_rotary(x, 2, p[:39], f), lambda: fwa.fwa_rotary(x, 2, p.long(), f),
                lambda: fwa.fwa_rotary(x, 2, p, f.double()), lambda: fwa.fwa_rotary(x, 2, p, f, a[:5]), lambda: fwa.fwa_rotary(x, 2, p, f, a.long()),
                lambda: fwa.fwa_rotary(x[0, 0], 2, p, f), lambda: fwa.fwa_rotary(x, 2, p[None].expand(3, 40, 1).contiguous(), f),
                lambda: fwa.fwa_rotary(x.transpose(0, 1), 2, p[:2], f), lambda: fwa.fwa_rotary(x, 2, p, f, out=torch.empty_like(x[:1])),
                lambda: fwa.fwa_rotary(x[0], 2, p[None], f), lambda: fwa.fwa_rotary(x, 2, p.cpu(), f), lambda: fwa.fwa_rotary(x.double(), 2, p, f)):
        with pytest.raises((TypeError, ValueError)):
            bad()
    with pytest.raises(fwa.FwaError):  # more pairs than the head has
        fwa.fwa_rotary(x, 2, p, torch.ones(33, device="cuda"))
    with pytest.raises(fwa.FwaError):  # an output on top of a part of the input
        fwa.fwa_rotary(x[:1], 2, p, f, out=x.view(-1)[8:8 + x[:1].numel()].view(1, 40, 128))
    with pytest.raises(fwa.FwaError):
        fwa.fwa_rotary(x.view(-1)[4:4 + 128].view(1, 1, 128), 2, p[:1].contiguous(), f)
