"""DropITGatedLinear outside of training: as with the other layers, the stock operations where the kernels have no form (needs no GPU)."""
import pytest
import torch
import torch.nn.functional as F

import paper_2202_13808_b200 as dropit
from paper_2202_13808_b200 import build as build_mod

GATES = {"silu": F.silu, "gelu": F.gelu, "relu": F.relu}


@pytest.fixture(scope="module", autouse=True)
def _built():
    build_mod.build()


def _check(device, dtype, gate, bias):
    layer = dropit.DropITGatedLinear(24, 10, bias=bias, gate=gate, device=device, dtype=dtype).eval()
    x = torch.randn(3, 5, 24, device=device, dtype=dtype)
    a, u = F.linear(x, layer.weight, layer.bias).chunk(2, -1)
    with torch.no_grad():
        assert torch.equal(layer(x), (GATES[gate](a) * u).detach())
        assert torch.equal(layer.train()(x), (GATES[gate](a) * u).detach())
    with pytest.raises((TypeError, ValueError)):        # in training there is no other path
        layer(x)


@pytest.mark.parametrize("dtype", [torch.float32, torch.float64, torch.bfloat16])
@pytest.mark.parametrize("gate", sorted(GATES))
def test_on_the_host(dtype, gate):
    _check("cpu", dtype, gate, gate != "relu")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float16, torch.float64])
def test_other_types(cuda_device, dtype):
    _check(cuda_device, dtype, "silu", True)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_no_rows(cuda_device, dtype):
    layer = dropit.DropITGatedLinear(64, 16, gamma=0.5, device=cuda_device, dtype=dtype).train()
    x = torch.randn(2, 0, 64, device=cuda_device, dtype=dtype, requires_grad=True)
    h = layer(x)
    h.sum().backward()
    assert h.shape == (2, 0, 16) and x.grad.shape == x.shape
    assert not bool(layer.weight.grad.any()) and not bool(layer.bias.grad.any())
    with torch.no_grad():
        assert layer.eval()(x).shape == (2, 0, 16)


@pytest.mark.gpu
def test_more_values_than_a_call_takes(cuda_device):
    """2^31 projections and one row more: the library's call is refused, the layer takes the stock operations."""
    if torch.cuda.mem_get_info(cuda_device)[0] < 20 * 2 ** 30:
        pytest.skip("needs 20 GB")
    M = 2 ** 20 + 1
    layer = dropit.DropITGatedLinear(8, 1024, device=cuda_device, dtype=torch.bfloat16).eval()
    x = torch.randn(M, 8, device=cuda_device, dtype=torch.bfloat16)
    with torch.no_grad():
        with pytest.raises(dropit.DropITError):
            dropit.dropit_gated_linear(x, layer.weight, layer.bias)
        h = layer(x)
        a, u = F.linear(x[-3:], layer.weight, layer.bias).float().chunk(2, -1)
    # a, u, f(a) and the product each rounded to bf16
    assert h.shape == (M, 1024) and bool(((h[-3:].float() - F.silu(a) * u).abs() <= 5 * 2.0 ** -8 * (a * u).abs() + 1e-6).all())
