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


@pytest.mark.parametrize("M", [8, 300])
@pytest.mark.parametrize("span", [(-12.5, -3.0), (-3.0, 3.0), (3.0, 200.0)])
def test_gelu_is_accurate_relative_to_its_value(cuda_device, M, span):
    """Every bf16 of the span, as a with u = 1: one rounding of a value that is off by 2^-12 of itself at most, in the tail too."""
    H = 64
    bits = torch.arange(2 ** 16, dtype=torch.int32).to(torch.int16).view(torch.bfloat16).float()
    a = bits[(bits >= span[0]) & (bits <= span[1])].to(cuda_device)
    a = a[a.abs() >= 2.0 ** -100]
    for start in range(0, a.numel(), M * H):
        part = torch.ones(M * H, device=cuda_device)
        part[:min(M * H, a.numel() - start)] = a[start:start + M * H]
        part = part.view(M, H)
        x = torch.cat([part, torch.ones_like(part)], 1).bfloat16()
        w = torch.eye(2 * H, device=cuda_device).bfloat16()
        h, gu = dropit.dropit_gated_linear(x, w, None, "gelu", keep=True)
        want = _gelu64(part.double())
        assert bool(((h.double() - want).abs() <= (U + 2.0 ** -12) * want.abs()).all())
        # du = dh f(a) with dh = 1
        dgu = dropit.dropit_gated_linear_backward(torch.ones_like(h), gu, "gelu")
        assert bool(((dgu[:, H:].double() - want).abs() <= (U + 2.0 ** -12) * want.abs()).all())
        # f' = Phi + a phi passes through zero at -0.7518; elsewhere its terms do not cancel beyond a digit or two
        slope = 0.5 * torch.special.erfc(-part.double() / 2 ** 0.5) + part.double() * torch.exp(-part.double() ** 2 / 2) / (2 * torch.pi) ** 0.5
        terms = 0.5 * torch.special.erfc(-part.double() / 2 ** 0.5) + part.double().abs() * torch.exp(-part.double() ** 2 / 2) / (2 * torch.pi) ** 0.5
        assert bool(((dgu[:, :H].double() - slope).abs() <= U * slope.abs() + 2.0 ** -12 * terms).all())


def _kernel_nodes(graph):
    runtime = ctypes.CDLL("libcudart.so.12")
    count = ctypes.c_size_t(0)
    assert runtime.cudaGraphGetNodes(ctypes.c_void_p(graph.raw_cuda_graph()), None, ctypes.byref(count)) == 0
    return count.value


def test_rows_behind_the_full_waves_whose_tiles_share_a_long_axis(cuda_device):
    """Where the last wave is nearly empty its rows are a launch of their own; their summed axis of 4096 is long enough for the clusters of two and
    four pairs that a few tiles get, which then begin at another row."""
    C, H = 256, 2048
    g = torch.Generator(device=cuda_device).manual_seed(1)
    w = (torch.randn(2 * H, C, generator=g, device=cuda_device) * C ** -0.5).bfloat16()
    pairs, split = torch.cuda.get_device_properties(cuda_device).multi_processor_count // 2, 0
    for tiles_over in (1, 2, 4):
        for less in range(0, 5):                # some SMs may have no partner
            M = 256 * (pairs - less + tiles_over) - 37
            dgu = torch.randn(M, 2 * H, generator=g, device=cuda_device).bfloat16()
            dx = dropit.dropit_gated_input_grad(dgu, w)
            want, size = dgu.double() @ w.double(), dgu.double().abs() @ w.double().abs()
            bound = 2 * H * 2.0 ** -24 * size
            assert bool(((dx.double() - want).abs() <= bound + U * (want.abs() + bound)).all())
            graph = torch.cuda.CUDAGraph(keep_graph=True)
            with torch.cuda.graph(graph):
                again = dropit.dropit_gated_input_grad(dgu, w)
            split += _kernel_nodes(graph) == 2
            graph.replay()
            assert torch.equal(again, dx)
    dropit.check_device_status(cuda_device)
    assert split
