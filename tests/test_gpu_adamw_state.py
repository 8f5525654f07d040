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


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_checkpoint_is_copied_into_the_state_there_is(cuda_device, bits, dtype):
    model = _model(cuda_device, dtype)
    opt = dropit.DropITAdamW(model.parameters(), lr=1e-2, state_bits=bits, master=True, seed=1)
    _fill_grads(model, 1)
    opt.step()
    saved, params = copy.deepcopy(opt.state_dict()), [p.detach().clone() for p in model.parameters()]
    places = [[v.data_ptr() for v in opt.state[p].values()] for p in model.parameters()]
    arena = opt.whole_state("exp_avg").data_ptr()
    opt.step()
    want = [p.detach().clone() for p in model.parameters()], _values(opt, model.parameters())
    opt.step()
    opt.load_state_dict(saved)
    assert [[v.data_ptr() for v in opt.state[p].values()] for p in model.parameters()] == places
    assert opt.whole_state("exp_avg").data_ptr() == arena
    with torch.no_grad():
        for p, k in zip(model.parameters(), params):
            p.copy_(k)
    opt.step()
    assert all(torch.equal(p, w) for p, w in zip(model.parameters(), want[0])) and _equal(_values(opt, model.parameters()), want[1])


@pytest.mark.parametrize("bits", [8, 32])
def test_a_captured_step_goes_on_from_a_checkpoint(cuda_device, bits):
    model = _model(cuda_device)
    lr = torch.tensor(1e-2, device=cuda_device)
    opt = dropit.DropITAdamW(model.parameters(), lr=lr, state_bits=bits)
    _fill_grads(model, 1)
    opt.step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        opt.step()
    saved, params = copy.deepcopy(opt.state_dict()), [p.detach().clone() for p in model.parameters()]
    for _ in range(2):
        graph.replay()
    want = [p.detach().clone() for p in model.parameters()], _values(opt, model.parameters())
    lr.fill_(0.5)
    opt.load_state_dict(saved)
    assert opt.param_groups[0]["lr"] is lr and float(lr) == float(torch.tensor(1e-2))       # what the graph reads
    with torch.no_grad():
        for p, k in zip(model.parameters(), params):
            p.copy_(k)
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    assert int(opt.state[model.weight]["step"]) == 3
    assert all(torch.equal(p, w) for p, w in zip(model.parameters(), want[0])) and _equal(_values(opt, model.parameters()), want[1])


def test_a_checkpoint_without_a_state_begins_anew(cuda_device):
    model = _model(cuda_device, torch.bfloat16)
    fresh = dropit.DropITAdamW(model.parameters(), lr=3e-2, master=True).state_dict()
    assert not fresh["state"]
    opt = dropit.DropITAdamW(model.parameters(), lr=1e-2, master=True)
    _fill_grads(model, 1)
    opt.step()
    opt.load_state_dict(fresh)
    assert opt.param_groups[0]["lr"] == 3e-2
    for p in model.parameters():
        s = opt.state[p]
        assert int(s["step"]) == 0 and not bool(s["exp_avg"].any()) and not bool(s["exp_avg_sq"].any())
        assert torch.equal(s["master"], p.detach().float())


def test_learning_rates_that_are_tensors_keep_their_places(cuda_device):
    a, b, c = (torch.nn.Parameter(torch.ones(n, device=cuda_device)) for n in (3, 4, 5))
    shared, own = torch.tensor(1e-2, device=cuda_device), torch.tensor([1e-3], device=cuda_device)
    opt = dropit.DropITAdamW([dict(params=[a], lr=shared), dict(params=[b], lr=shared), dict(params=[c], lr=own)])
    saved = opt.state_dict()
    for lr, other, third in ((0.3, 0.3, torch.tensor(0.7)), (0.1, 0.2, 0.9)):
        for g, v in zip(saved["param_groups"], (lr, other, third)):
            g["lr"] = v
        opt.load_state_dict(saved)
        got = [g["lr"] for g in opt.param_groups]
        assert [float(v) for v in got] == [float(torch.tensor(float(v))) for v in (lr, other, third)]
        assert got[2] is own and (got[0] is shared) == (got[1] is shared) == (lr == other)
        assert all(v.device == a.device for v in got)


def test_a_learning_rate_that_a_captured_step_reads_is_not_torn_in_two(cuda_device):
    params = [torch.nn.Parameter(torch.ones(n, device=cuda_device)) for n in (3, 4)]
    lr = torch.tensor(1e-2, device=cuda_device)
    opt = dropit.DropITAdamW([dict(params=[p], lr=lr) for p in params])
    for p in params:
        p.grad = torch.ones_like(p)
    opt.step()
    with torch.cuda.graph(torch.cuda.CUDAGraph()):
        opt.step()
    saved = opt.state_dict()
    saved["param_groups"][0]["lr"] = 0.5
    with pytest.raises(ValueError, match="captured"):
        opt.load_state_dict(saved)
    assert all(g["lr"] is lr for g in opt.param_groups) and float(lr) == float(torch.tensor(1e-2))


@pytest.mark.parametrize("how", ["shape", "type", "name", "count"])
def test_a_checkpoint_that_is_refused_changes_nothing(cuda_device, how):
    model = _model(cuda_device)
    opt = dropit.DropITAdamW(model.parameters(), lr=1e-2)
    _fill_grads(model, 1)
    opt.step()
    saved = copy.deepcopy(opt.state_dict())
    saved["param_groups"][0]["lr"] = 7.0
    last = saved["state"][1]
    if how == "shape":
        last["exp_avg_sq"] = last["exp_avg_sq"][:-1]
    elif how == "type":
        last["exp_avg_sq"] = last["exp_avg_sq"].double()
    elif how == "name":
        last["other"] = last.pop("exp_avg_sq")
    else:
        saved["param_groups"][0]["params"] = [0]
    before = _values(opt, model.parameters())
    with pytest.raises(ValueError):
        opt.load_state_dict(saved)
    assert opt.param_groups[0]["lr"] == 1e-2 and _equal(_values(opt, model.parameters()), before)
    opt.step()
    assert int(opt.state[model.weight]["step"]) == 2


def test_hooks_around_a_checkpoint_see_its_state(cuda_device):
    model = _model(cuda_device)
    opt = dropit.DropITAdamW(model.parameters(), lr=1e-2)
    _fill_grads(model, 1)
    opt.step()
    saved = copy.deepcopy(opt.state_dict())
    opt.step()
    seen = []

    def before(o, state_dict):
        seen.append(sorted(state_dict["state"]))
        state_dict["state"][0]["step"] = state_dict["state"][0]["step"] + 4
        return state_dict
    opt.register_load_state_dict_pre_hook(before)
    opt.register_load_state_dict_post_hook(lambda o: seen.append(int(o.state[model.weight]["step"])))
    opt.load_state_dict(saved)
    assert seen == [[0, 1], 5]


@pytest.mark.parametrize("bits", [8, 32])
def test_a_state_that_is_emptied_begins_anew(cuda_device, bits):
    model, other = _model(cuda_device), _model(cuda_device)
    opt = dropit.DropITAdamW(model.parameters(), lr=1e-2, state_bits=bits)
    _fill_grads(model, 1)
    opt.step()
    with torch.no_grad():
        for p, q in zip(model.parameters(), other.parameters()):
            q.copy_(p)
    opt.state.clear()
    _fill_grads(model, 2)
    _fill_grads(other, 2)
    opt.step()
    fresh = dropit.DropITAdamW(other.parameters(), lr=1e-2, state_bits=bits)
    fresh.step()
    assert all(torch.equal(p, q) for p, q in zip(model.parameters(), other.parameters()))
    assert _equal(_values(opt, model.parameters()), _values(fresh, other.parameters())) and len(opt.state_dict()["state"]) == 2
    opt.state.clear()
    assert int(opt.init_state(model.weight)["step"]) == 0
    with torch.cuda.graph(torch.cuda.CUDAGraph()):
        opt.step()
    opt.state.clear()
    with pytest.raises(RuntimeError, match="captured"):
        opt.step()
