"""Forward-mode derivatives: what has none says so, before anything is launched (needs no GPU); a result without a tangent would pass for a constant."""
import pytest
import torch
import torch.autograd.forward_ad as fwd

import paper_2202_13808_b200 as dropit
from paper_2202_13808_b200 import build as build_mod


@pytest.fixture(scope="module", autouse=True)
def _built():
    build_mod.build()


def _refuses(call):
    with pytest.raises(NotImplementedError, match="forward-mode"):
        call()


@pytest.mark.parametrize("which", [0, 1, 2])
@pytest.mark.parametrize("grad", [False, True])
def test_gated_linear(which, grad):
    x, w, b = (torch.randn(s) for s in ((4, 16), (16, 16), (16,)))
    layer = dropit.DropITGatedLinear(16, 8).train()
    with fwd.dual_level(), torch.set_grad_enabled(grad):
        args = [x, w, b]
        args[which] = fwd.make_dual(args[which], torch.ones_like(args[which]))
        _refuses(lambda: dropit.dropit_gated_linear(*args))
        if grad:
            layer.weight.requires_grad_(False)
            _refuses(lambda: torch.func.functional_call(layer, {"weight": args[1], "bias": args[2]}, (args[0],)))
        layer.eval()            # outside of training the derivative is that of the stock operations
        h = torch.func.functional_call(layer, {"weight": args[1], "bias": args[2]}, (args[0],))
        a, u = torch.nn.functional.linear(*args).chunk(2, -1)
        want = torch.nn.functional.silu(a) * u
        got, ref = fwd.unpack_dual(h), fwd.unpack_dual(want)
        assert torch.equal(got.primal, ref.primal) and torch.equal(got.tangent, ref.tangent)


def test_gated_linear_gradients():
    dh, gu, w = torch.randn(4, 8), torch.randn(4, 16), torch.randn(16, 16)
    with fwd.dual_level():
        dual = lambda t: fwd.make_dual(t, torch.ones_like(t))
        _refuses(lambda: dropit.dropit_gated_linear_backward(dual(dh), gu))
        _refuses(lambda: dropit.dropit_gated_linear_backward(dh, dual(gu)))
        _refuses(lambda: dropit.dropit_gated_input_grad(dual(gu), w))
        _refuses(lambda: dropit.dropit_gated_input_grad(gu, dual(w)))


@pytest.mark.parametrize("which", [0, 1, 2])
def test_rotation(which):
    args = [torch.randn(1, 4, 2, 16), torch.randn(1, 4, 2, 16), torch.randn(4, 1)]
    rot = dropit.DropITRotary(16, (16,))
    with fwd.dual_level():
        args[which] = fwd.make_dual(args[which], torch.ones_like(args[which]))
        _refuses(lambda: rot(*args))
        _refuses(lambda: dropit.dropit_rotary(*args, rot._plan))
        with torch.no_grad():
            _refuses(lambda: rot(*args))


@pytest.mark.gpu
def test_on_the_gpu(cuda_device):
    """With gradients recorded, through the layers; and a gradient whose own input has a tangent."""
    layer = dropit.DropITGatedLinear(16, 8, device=cuda_device).train()
    rot = dropit.DropITRotary(8, (8,))
    x = torch.randn(4, 16, device=cuda_device, requires_grad=True)
    at = torch.arange(4, device=cuda_device).unsqueeze(1)
    h = layer(x)
    turned, _ = rot(h.view(4, 1, 8), None, at)
    with fwd.dual_level():
        moved = fwd.make_dual(x, torch.ones_like(x))
        _refuses(lambda: layer(moved))
        _refuses(lambda: rot(moved.view(4, 2, 8), None, at))
        _refuses(lambda: torch.autograd.grad(h, x, fwd.make_dual(torch.ones_like(h), torch.ones_like(h)), retain_graph=True))
        _refuses(lambda: torch.autograd.grad(turned, x, fwd.make_dual(torch.ones_like(turned), torch.ones_like(turned)), retain_graph=True))
    grad, = torch.autograd.grad(turned.sum(), x)
    assert bool(torch.isfinite(grad).all())
