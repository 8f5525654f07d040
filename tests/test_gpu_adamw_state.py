"""The state of DropITAdamW: where it lies, what may change under it, what a captured step and a checkpoint may rely on."""
import copy

import pytest
import torch

import paper_2202_13808_b200 as dropit

pytestmark = pytest.mark.gpu


def _model(device, dtype=torch.float32, seed=0):
    torch.manual_seed(seed)
    return torch.nn.Linear(40, 20, device=device, dtype=dtype)


def _fill_grads(model, seed):
    g = torch.Generator(device=model.weight.device).manual_seed(seed)
    for p in model.parameters():
        p.grad = torch.randn(p.shape, generator=g, device=p.device).to(p.dtype)


def _values(opt, params):
    return [[v.clone() for v in opt.state[p].values()] for p in params]


def _equal(a, b):
    return all(x.dtype == y.dtype and torch.equal(x.float(), y.float()) for s, t in zip(a, b) for x, y in zip(s, t))


@pytest.mark.parametrize("bits", [8, 32])
def test_a_copy_in_fp32_belongs_to_the_type_it_was_made_for(cuda_device, bits):
    """fp32 parameters have no copy: as bf16 ones they would be stepped from what lies in its place."""
    model = _model(cuda_device)
    opt = dropit.DropITAdamW(model.parameters(), lr=1e-3, state_bits=bits, master=True)
    _fill_grads(model, 1)
    opt.step()
    model.bfloat16()
    _fill_grads(model, 2)
    kept = [p.detach().clone() for p in model.parameters()]
    with pytest.raises(ValueError, match="type"):
        opt.step()
    assert all(torch.equal(p, k) for p, k in zip(model.parameters(), kept))
