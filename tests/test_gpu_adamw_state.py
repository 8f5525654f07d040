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


@pytest.mark.parametrize("first, then", [(torch.float32, torch.bfloat16), (torch.bfloat16, torch.float32)])
def test_a_state_laid_out_again_has_the_copies_of_the_types_there_are(cuda_device, first, then):
    model = _model(cuda_device, first)
    opt = dropit.DropITAdamW(model.parameters(), lr=1e-3, weight_decay=0.0, master=True)
    _fill_grads(model, 1)
    opt.step()
    moments = [opt.state[p]["exp_avg"].clone() for p in model.parameters()]
    model.to(then)
    opt.add_param_group(dict(params=[torch.nn.Parameter(torch.ones(3, device=cuda_device))]))
    opt.init_state()
    for p, m in zip(model.parameters(), moments):
        assert torch.equal(opt.state[p]["exp_avg"], m) and ("master" in opt.state[p]) == (then == torch.bfloat16)
        if then == torch.bfloat16:
            assert torch.equal(opt.state[p]["master"], p.detach().float())
    kept = [p.detach().clone() for p in model.parameters()]
    _fill_grads(model, 2)
    opt.step()
    # a step is at most lr (1 - b1^t)^-1 sqrt(1 - b2^t) m / sqrt(v) < 5 lr here, and a bf16 value rounds to within 2^-8 of itself
    for p, k in zip(model.parameters(), kept):
        assert float((p.detach().float() - k.float()).abs().max()) <= 5e-3 + 2.0 ** -8 * float(k.float().abs().max())


@pytest.mark.parametrize("again", [False, True])
def test_a_state_is_not_laid_out_while_a_step_is_captured(cuda_device, again):
    """Its zeros would be part of the graph, and every replay would begin anew."""
    model = _model(cuda_device)
    opt = dropit.DropITAdamW(model.parameters(), lr=1e-2)
    _fill_grads(model, 1)
    late = torch.nn.Parameter(torch.ones(5, device=cuda_device))
    late.grad = torch.ones_like(late)
    if again:
        opt.step()
        opt.add_param_group(dict(params=[late]))
    with pytest.raises(RuntimeError, match="init_state"):
        with torch.cuda.graph(torch.cuda.CUDAGraph()):
            opt.step()
    opt.init_state()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        opt.step()
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert int(opt.state[model.weight]["step"]) == 3 + again
    assert not again or int(opt.state[late]["step"]) == 3


def test_a_group_that_comes_after_a_capture_is_refused(cuda_device):
    """The state would move from under the captured step, whose replays would go on in memory that is somebody else's."""
    model = _model(cuda_device)
    opt = dropit.DropITAdamW(model.parameters(), lr=1e-2)
    _fill_grads(model, 1)
    opt.step()
    opt.add_param_group(dict(params=[torch.nn.Parameter(torch.ones(3, device=cuda_device))]))        # nothing is captured yet
    opt.step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        opt.step()
    with pytest.raises(RuntimeError, match="captured"):
        opt.add_param_group(dict(params=[torch.nn.Parameter(torch.ones(5, device=cuda_device))]))
    assert len(opt.param_groups) == 2
    graph.replay()
    opt.step()
    torch.cuda.synchronize()
    assert int(opt.state[model.weight]["step"]) == 4
