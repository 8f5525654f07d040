"""Rotary positions of every type, in both types of values and through the layer."""
import pytest
import torch

import paper_2202_13808_b200 as dropit
from test_gpu_rotary import _check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", [torch.int32, torch.int64, torch.float32])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("each", [False, True])
@pytest.mark.parametrize("interleaved", [False, True])
def test_positions_through_the_layer(cuda_device, kind, dtype, each, interleaved):
    B, L, sections = 3, 53, (16, 24)
    g = torch.Generator(device=cuda_device).manual_seed(5)
    rot = dropit.DropITRotary(48, sections, theta=500.0, interleaved=interleaved, shared=each)
    q = torch.randn(B, L, 4, 48, generator=g, device=cuda_device).to(dtype).requires_grad_(True)
    k = torch.randn(B, L, 2, 48, generator=g, device=cuda_device).to(dtype).requires_grad_(True)
    positions = torch.randn((B, L, 2) if each else (L, 2), generator=g, device=cuda_device) * 300
    if kind != torch.float32:
        positions = positions.round().to(kind)
    dq, dk = torch.randn(q.shape, generator=g, device=cuda_device).to(dtype), torch.randn(k.shape, generator=g, device=cuda_device).to(dtype)
    q2, k2 = rot(q, k, positions)
    gq, gk = torch.autograd.grad((q2, k2), (q, k), (dq, dk))
    at = positions if each else positions.unsqueeze(0)
    for got, x, sign in ((q2, q, 1.0), (k2, k, 1.0), (gq, dq, -1.0), (gk, dk, -1.0)):
        _check(got.detach(), x.detach(), at, sections, 500.0, interleaved, each, sign)
