"""The gated linear's gate functions in the tails, its attributes, and dx where rows of their own share a summed axis."""
import ctypes

import pytest
import torch

import paper_2202_13808_b200 as dropit

pytestmark = pytest.mark.gpu

U = 2.0 ** -8


def _gelu64(a):
    """a Phi(a), the lower tail from erfc: relative accuracy in 64 bits."""
    return a * 0.5 * torch.special.erfc(-a.double() / 2 ** 0.5)


@pytest.mark.parametrize("training", [True, False])
def test_attributes_are_read_at_the_call(cuda_device, training):
    """As those of DropITLinear are: the gate and the cache's format may change between two calls."""
    torch.manual_seed(1)
    layer = dropit.DropITGatedLinear(64, 32, gate="silu", gamma=0.5, device=cuda_device).train(training)
    x = torch.randn(50, 64, device=cuda_device)
    for gate in ("relu", "gelu", "silu"):
        layer.gate = gate
        want = dropit.dropit_gated_linear(x, layer.weight.detach(), layer.bias.detach(), gate)
        assert torch.allclose(layer(x), want, rtol=1e-5, atol=1e-5)
        with torch.no_grad():
            assert torch.equal(layer(x), want)
    layer.gate = "tanh"
    with pytest.raises(ValueError):
        layer(x)
    layer.gate, grads = "silu", {}
    layer.train()
    for fmt in ("bitmask", "index32"):
        layer.fmt, layer.weight.grad = fmt, None
        layer(x).sum().backward()
        grads[fmt] = layer.weight.grad
    assert torch.allclose(grads["bitmask"], grads["index32"], rtol=1e-4, atol=1e-4)
    layer.fmt = "dense"
    with pytest.raises((KeyError, ValueError)):
        layer(x)
