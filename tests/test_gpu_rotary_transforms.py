"""What of the rotation cannot go through the native autograd node goes through the Python function, which says what it does not do: forward mode, functorch's transforms, subclasses
in any place, traced calls."""
import pytest
import torch
import torch.autograd.forward_ad as fwd

from test_gpu_rotary import BF16, F32, make

pytestmark = pytest.mark.gpu


@pytest.fixture
def no_native_node(monkeypatch):
    from paper_2501_06480_amd import binding

    def refuse(*args):
        raise AssertionError("the native node was called")
    monkeypatch.setattr(binding._native(), "rotary_node", refuse)


def inputs(dtype=F32):
    x, positions, f, axis, _ = make(dtype, 2, 5, 2, 32, (8, 8))
    return x.cuda(), positions.cuda(), f.cuda(), axis.cuda()


def test_the_native_node_is_what_a_plain_call_takes(no_native_node):
    from paper_2501_06480_amd import autograd
    x, positions, f, axis = inputs()
    with pytest.raises(AssertionError, match="native node"):
        autograd.rotary(x, 2, positions, f, axis)


def test_forward_mode(no_native_node):
    from paper_2501_06480_amd import autograd
    x, positions, f, axis = inputs()
    with fwd.dual_level():
        dual = fwd.make_dual(x, torch.ones_like(x))
        with pytest.raises(NotImplementedError, match="jvp"):
            autograd.rotary(dual, 2, positions, f, axis)


@pytest.mark.parametrize("transform", ["jvp", "vjp", "grad", "vmap"])
def test_transforms(no_native_node, transform):
    from paper_2501_06480_amd import autograd
    x, positions, f, axis = inputs()
    call = lambda t: autograd.rotary(t, 2, positions, f, axis)  # noqa: E731
    with pytest.raises(RuntimeError, match="setup_context"):
        if transform == "jvp":
            torch.func.jvp(call, (x,), (x,))
        elif transform == "vjp":
            torch.func.vjp(call, x)
        elif transform == "grad":
            torch.func.grad(lambda t: call(t).sum())(x)
        else:
            torch.func.vmap(call)(x[None])


class Tagged(torch.Tensor):
    pass


@pytest.mark.parametrize("which", range(4))
def test_subclasses(no_native_node, which):
    from paper_2501_06480_amd import autograd, binding
    args = list(inputs())
    want = binding.fwa_rotary(args[0], 2, *args[1:])
    args[0].requires_grad_()
    args[which] = args[which].as_subclass(Tagged)
    y = autograd.rotary(args[0], 2, *args[1:])
    assert "autograd" in type(y.grad_fn).__module__  # the Python function's
    assert torch.equal(y.detach().as_subclass(torch.Tensor), want)


@pytest.mark.parametrize("grad", [False, True])
def test_traced(no_native_node, grad):
    """A traced call computes: its replay on other inputs is the call on those inputs."""
    from paper_2501_06480_amd import autograd, binding
    x, positions, f, axis = inputs(BF16)
    traced = torch.jit.trace(lambda t: autograd.rotary(t, 2, positions, f, axis), (x.clone().requires_grad_(grad),), check_trace=False)
    other = torch.randn_like(x).requires_grad_(grad)
    assert torch.equal(traced(other), binding.fwa_rotary(other.detach(), 2, positions, f, axis))
