"""The AdamW step against the formula in 64 bits: types, moments in 32 and in 8 bits, ragged tensors, groups, capture, checkpoints."""
import copy
import math

import numpy as np
import pytest
import torch

import paper_2202_13808_b200 as dropit

pytestmark = pytest.mark.gpu

BLOCK = 256


def _mix(x):
    with np.errstate(over="ignore"):
        x = (x ^ (x >> np.uint32(16))) * np.uint32(0x7FEB352D)
        x = (x ^ (x >> np.uint32(15))) * np.uint32(0x846CA68B)
        return x ^ (x >> np.uint32(16))


def _words(seed, step, ordinal, n):
    with np.errstate(over="ignore"):
        key = _mix(np.array([seed], dtype=np.uint32))
        key = _mix(key + np.uint32(step))
        key = _mix(key + np.uint32(ordinal))
        w = _mix(np.arange(n, dtype=np.uint32) ^ key)
        return w, w * np.uint32(0x9E3779B1)


def _code_values():
    return np.array([m / 512 for m in range(8)] + [(8 + m) / 8 * 2.0 ** e for e in range(-6, 9) for m in range(8)][:-1])


def _step64(p, g, m, v, t, lr, wd, b1, b2, eps):
    """The step, and how far fp32 may be from its parameter.  m is off by half a unit (2^-24) for each of its two products, the sum and the constants,
    of the terms' size: where the terms cancel that is more than the move's own error, and it is divided by the root as m is.  Root
    and quotients are off by a few units each, below 3e-6 of the move in all; decay, product and difference by a half each."""
    size = b1 * m.abs() + (1 - b1) * g.abs()
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g * g
    unit = lr / (1 - b1 ** t) / ((v / (1 - b2 ** t)).sqrt() + eps)
    move = unit * m
    bound = 4 * 2.0 ** -24 * (p.abs() + move.abs()) + 3e-6 * move.abs() + 6 * 2.0 ** -24 * unit * size + 1e-40
    return p * (1 - lr * wd) - move, m, v, bound


def _grads(params, seed, dtype, scale=0.02):
    g = torch.Generator(device="cuda").manual_seed(seed)
    for p in params:
        p.grad_dtype = None
        grad = torch.empty_like(p, dtype=dtype)
        grad.copy_(torch.randn(p.shape, generator=g, device="cuda") * scale)
        p.grad = grad


SHAPES = [(1,), (3,), (255,), (256,), (257,), (16, 64), (1000, 37), (5, 0), (7, 3, 3, 3)]


def _params(dtype, shapes=SHAPES, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return [torch.nn.Parameter((torch.randn(s, generator=g, device="cuda") * 0.1).to(dtype)) for s in shapes]


@pytest.mark.parametrize("p_type", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("g_type", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("master", [False, True])
def test_steps_with_moments_in_32_bits(cuda_device, p_type, g_type, master):
    params = _params(p_type)
    hyper = dict(lr=3e-3, betas=(0.9, 0.99), eps=1e-8, weight_decay=0.1)
    opt = dropit.DropITAdamW(params, master=master, **hyper)
    held = [dict(p=p.detach().double().clone(), m=torch.zeros(p.shape, dtype=torch.float64, device="cuda"),
                 v=torch.zeros(p.shape, dtype=torch.float64, device="cuda")) for p in params]
    for t in range(1, 4):
        _grads(params, t, g_type)
        opt.step()
        for p, h in zip(params, held):
            want, m, v, bound = _step64(h["p"], p.grad.double(), h["m"], h["v"], t, 3e-3, 0.1, 0.9, 0.99, 1e-8)
            s = opt.state[p]
            # moments: two products, a sum and the constants' roundings, half a unit (2^-24) each
            for got, ref, size in ((s["exp_avg"], m, 0.9 * h["m"].abs() + 0.1 * p.grad.double().abs()), (s["exp_avg_sq"], v, v)):
                assert bool(((got.double() - ref).abs() <= 6 * 2.0 ** -24 * size + 1e-40).all())
            mine = s["master"] if "master" in s else p
            if "master" in s:
                assert torch.equal(p.detach(), s["master"].to(torch.bfloat16))
            elif p_type == torch.bfloat16:
                bound = bound * 2 + 2.0 ** -8 * want.abs()
            assert bool(((mine.double() - want).abs() <= bound).all())
            # the next step starts from what is held
            h.update(p=mine.detach().double().clone(), m=s["exp_avg"].double().clone(), v=s["exp_avg_sq"].double().clone())
        assert all(int(opt.state[p]["step"]) == (t if p.numel() else 0) for p in params)


@pytest.mark.parametrize("p_type, g_type, dither", [(torch.float32, torch.float32, False), (torch.bfloat16, torch.bfloat16, True),
                                                    (torch.bfloat16, torch.float32, False), (torch.float32, torch.bfloat16, False)])
def test_steps_with_moments_in_8_bits(cuda_device, p_type, g_type, dither):
    params = _params(p_type)
    opt = dropit.DropITAdamW(params, lr=3e-3, betas=(0.9, 0.99), weight_decay=0.1, state_bits=8, dither=dither, seed=77)
    values = _code_values()
    with torch.no_grad():
        opt.init_state()
    for t in range(1, 5):
        _grads(params, t, g_type)
        before = [(p.detach().double().clone(), {k: v.clone() for k, v in opt.state[p].items()}) for p in params]
        opt.step()
        for ordinal, (p, (p0, s0)) in enumerate(zip(params, before)):
            n, s = p.numel(), opt.state[p]
            block = torch.arange(n, device="cuda") // BLOCK
            m0 = s0["exp_avg"].double().reshape(-1) * s0["exp_avg_scale"].double()[block]
            r0 = s0["exp_avg_root"].double().reshape(-1) * s0["exp_avg_root_scale"].double()[block]
            want, m, v, bound = _step64(p0.reshape(-1), p.grad.double().reshape(-1), m0, r0 ** 2, t, 3e-3, 0.1, 0.9, 0.99, 1e-8)
            words, other = _words(77, t, ordinal, n)
            differ = 0
            for x, codes, scale, bits in ((m, s["exp_avg"], s["exp_avg_scale"], words >> 16), (v.sqrt(), s["exp_avg_root"], s["exp_avg_root_scale"], words & 0xFFFF)):
                if not n:
                    continue
                pad = torch.nn.functional.pad(x, (0, -n % BLOCK)).view(-1, BLOCK).abs().amax(1)
                assert bool(((scale.double() - pad / 448).abs() <= 1e-6 * pad / 448).all())
                y = (x / scale.double()[block]).abs().cpu().numpy()
                got = codes.double().reshape(-1).abs().cpu().numpy()
                low = np.clip(np.searchsorted(values, y, side="right") - 1, 0, len(values) - 2)
                place = (y - values[low]) / (values[low + 1] - values[low]) + bits.astype(np.float64) / 65536
                code = values[np.where(place >= 1, low + 1, low)]
                if x is not m:
                    code = np.where(y > 0, np.maximum(code, values[1]), code)
                # one of the two neighbours always, and the right one but where the sum is within fp32's reach of one
                edge = (np.abs(place - 1) < 1e-4) | (y < 1e-12) | (y > 447.9)
                assert (np.isclose(got, values[low]) | np.isclose(got, values[low + 1])).all()
                assert (got == code)[~edge].all()
                assert bool((torch.sign(codes.double().reshape(-1)) * torch.sign(x) >= 0).all())
            if not n:
                continue
            if p_type == torch.bfloat16:
                bound = bound * 2 + (2.0 ** -7 if dither else 2.0 ** -8) * want.abs()
            assert bool(((p.detach().double().reshape(-1) - want).abs() <= bound).all())
            if dither:
                w = want.cpu().numpy()
                unit = np.exp2(np.floor(np.log2(np.maximum(np.abs(w), 1e-38))) - 7)
                sum_ = np.abs(w) / unit + (other >> np.uint32(16)).astype(np.float64) / 65536
                edge = np.abs(sum_ - np.round(sum_)) < 2e-3
                assert (np.isclose(p.detach().double().reshape(-1).abs().cpu().numpy(), np.floor(sum_) * unit, rtol=1e-12) | edge).all()


def test_8_bit_moments_move_with_a_slow_average(cuda_device):
    """Gradients of a smaller size than those that the second moment comes from: v falls by a part in a thousand a step, far less than the distance of
    two codes, and follows the exact average all the same (each block's mean of 256 values; the dither's deviation of one value is at most a
    code's spacing, an eighth, every step that it moves)."""
    n, steps = 64 * BLOCK, 300
    p = torch.nn.Parameter(torch.zeros(n, device="cuda"))
    opt = dropit.DropITAdamW([p], lr=0.0, betas=(0.9, 0.999), weight_decay=0.0, state_bits=8, seed=5)
    p.grad = torch.ones(n, device="cuda")
    v = 0.0
    for t in range(steps):
        opt.step()
        v = 0.999 * v + 0.001
    p.grad = torch.full((n,), 0.5, device="cuda")
    for t in range(steps):
        opt.step()
        v = 0.999 * v + 0.001 * 0.25
    s = opt.state[p]
    held = (s["exp_avg_root"].double().view(-1, BLOCK) * s["exp_avg_root_scale"].double()[:, None]) ** 2
    # E[r^2] is above r^2 by the roundings' variance: every step adds up to (spacing / 2)^2 * 2 p (1 - p) < 1e-4 v, which the decay holds below
    # a tenth; the mean over 16384 values scatters by less than a hundredth
    assert abs(float(held.mean()) / v - 1) < 0.1
    assert abs(float((s["exp_avg"].double().view(-1, BLOCK) * s["exp_avg_scale"].double()[:, None]).mean()) - 0.5) < 0.01


def test_groups_missing_gradients_and_lr_on_the_device(cuda_device):
    a, b, c = _params(torch.float32, [(300,), (70, 5), (11,)])
    lr = torch.tensor(1e-2, device="cuda")
    opt = dropit.DropITAdamW([dict(params=[a], lr=lr, weight_decay=0.5), dict(params=[b, c], betas=(0.5, 0.6), eps=1e-4)], lr=1e-3)
    _grads([a, b], 1, torch.float32)
    kept, start = c.detach().clone(), {p: p.detach().double().clone() for p in (a, b)}
    factor = torch.tensor([0.25], device="cuda")
    opt.step(grad_factor=factor)
    assert torch.equal(c, kept) and int(opt.state[c]["step"]) == 0 and int(opt.state[b]["step"]) == 1
    zero = torch.zeros((), dtype=torch.float64, device="cuda")
    for p, (l, wd, b1, b2, eps) in ((a, (1e-2, 0.5, 0.9, 0.999, 1e-8)), (b, (1e-3, 1e-2, 0.5, 0.6, 1e-4))):
        l32 = float(torch.tensor(l))
        want, m, v, bound = _step64(start[p], 0.25 * p.grad.double(), zero, zero, 1, l32, wd, b1, b2, eps)
        assert bool(((p.detach().double() - want).abs() <= bound).all())
    # a group that comes later grows the arenas and keeps what there is
    m = opt.state[a]["exp_avg"].clone()
    d = torch.nn.Parameter(torch.ones(400, device="cuda"))
    opt.add_param_group(dict(params=[d]))
    d.grad = torch.ones_like(d)
    a.grad = b.grad = None
    opt.step()
    assert torch.equal(opt.state[a]["exp_avg"], m) and int(opt.state[a]["step"]) == 1 and int(opt.state[d]["step"]) == 1


@pytest.mark.parametrize("bits", [8, 32])
def test_captured_steps_count_on(cuda_device, bits):
    shapes = [(513,), (40, 40)]
    eager, captured = _params(torch.float32, shapes), _params(torch.float32, shapes)
    opts = [dropit.DropITAdamW(ps, lr=torch.tensor(1e-2, device="cuda"), state_bits=bits) for ps in (eager, captured)]
    for ps in (eager, captured):
        _grads(ps, 1, torch.float32)
    for o in opts:
        o.step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        opts[1].step()
    for i in range(4):
        for o in opts:
            o.param_groups[0]["lr"].fill_(1e-2 / (i + 1))
        opts[0].step()
        graph.replay()
    torch.cuda.synchronize()
    for p, q in zip(eager, captured):
        assert torch.equal(p, q) and int(opts[1].state[q]["step"]) == 5
        assert all(torch.equal(x.view(torch.uint8) if x.dtype == torch.float8_e4m3fn else x, y.view(torch.uint8) if y.dtype == torch.float8_e4m3fn else y)
                   for x, y in zip(opts[0].state[p].values(), opts[1].state[q].values()))


@pytest.mark.parametrize("bits", [8, 32])
def test_a_checkpoint_goes_on_where_it_stopped(cuda_device, bits):
    make = lambda ps: dropit.DropITAdamW(ps, lr=1e-2, state_bits=bits, master=True, seed=3)
    ps = _params(torch.bfloat16)
    opt = make(ps)
    for t in range(2):
        _grads(ps, t, torch.bfloat16)
        opt.step()
    saved = copy.deepcopy(opt.state_dict())
    others = [torch.nn.Parameter(p.detach().clone()) for p in ps]
    second = make(others)
    second.load_state_dict(saved)
    for p, q in zip(ps, others):
        q.grad = p.grad.clone()
    opt.step()
    second.step()
    for p, q in zip(ps, others):
        assert torch.equal(p, q)
        for x, y in zip(opt.state[p].values(), second.state[q].values()):
            assert x.dtype == y.dtype and torch.equal(x.float(), y.float())
    with pytest.raises(ValueError):
        dropit.DropITAdamW([torch.nn.Parameter(p.detach().clone()) for p in ps], state_bits=40 - bits).load_state_dict(saved)
    twin = copy.deepcopy(opt)
    assert all(torch.equal(x.float(), y.float()) for x, y in zip(opt.state[ps[1]].values(), list(twin.state.values())[1].values()))


def test_layouts(cuda_device):
    """Channels-last parameters, gradients of other strides, tensors that start anywhere, more tensors than one launch takes."""
    g = torch.Generator(device="cuda").manual_seed(4)
    draw = lambda *s: torch.randn(*s, generator=g, device="cuda")
    last = torch.nn.Parameter(draw(6, 5, 3, 3).contiguous(memory_format=torch.channels_last))
    flat = draw(2001)
    odd = torch.nn.Parameter(flat[1:1000])
    many = [torch.nn.Parameter(draw(1 + i % 7)) for i in range(1100)]
    params = [last, odd] + many
    before = [p.detach().double().clone() for p in params]
    last.grad = draw(6, 5, 3, 3)                        # contiguous
    odd.grad = draw(2000)[::2][:999]                    # gaps
    for p in many:
        p.grad = draw(*p.shape)
    opt = dropit.DropITAdamW(params, lr=1e-2)
    opt.step()
    zero = torch.zeros((), dtype=torch.float64, device="cuda")
    for p, b in zip(params, before):
        want, m, v, bound = _step64(b, p.grad.double(), zero, zero, 1, 1e-2, 1e-2, 0.9, 0.999, 1e-8)
        assert bool(((p.detach().double() - want).abs() <= bound).all())
        assert bool(((opt.state[p]["exp_avg"].double() - m).abs() <= 4 * 2.0 ** -24 * m.abs()).all())
    assert float(flat[0]) == float(flat[0]) and int(opt.state[many[-1]]["step"]) == 1


def test_not_finite_gradients_spoil_what_they_touch(cuda_device):
    for bits in (8, 32):
        p = torch.nn.Parameter(torch.ones(3 * BLOCK, device="cuda"))
        opt = dropit.DropITAdamW([p], lr=1e-2, state_bits=bits)
        p.grad = torch.ones_like(p)
        p.grad[5], p.grad[BLOCK + 7] = float("nan"), float("inf")
        opt.step()
        assert (~torch.isfinite(p)).nonzero().flatten().tolist() == [5, BLOCK + 7]
        p.grad = torch.ones_like(p)
        opt.step()
        bad = (~torch.isfinite(p)).view(3, BLOCK).sum(1).tolist()
        assert bad == ([BLOCK, BLOCK, 0] if bits == 8 else [1, 1, 0])


def test_refusals(cuda_device):
    p = torch.nn.Parameter(torch.ones(8, device="cuda"))
    make = lambda *a, **k: dropit.DropITAdamW([p], *a, **k)
    for kw in (dict(lr=-1.0), dict(betas=(1.0, 0.9)), dict(eps=-1.0), dict(weight_decay=-0.1), dict(state_bits=4)):
        with pytest.raises(ValueError):
            make(**kw)
    with pytest.raises(TypeError):
        dropit.DropITAdamW([torch.nn.Parameter(torch.ones(8, device="cuda").half())])
    with pytest.raises(ValueError):
        dropit.DropITAdamW([torch.nn.Parameter(torch.ones(8, 2, device="cuda")[:, 0])])
    with pytest.raises(ValueError):
        cpu = torch.nn.Parameter(torch.ones(3))
        cpu.grad = torch.ones(3)
        dropit.DropITAdamW([cpu]).step()
    with pytest.raises(ValueError):
        dropit.DropITAdamW([p, p])
    both = torch.ones(12, device="cuda")
    with pytest.raises(ValueError, match="share memory"):
        dropit.DropITAdamW([torch.nn.Parameter(both[:8]), torch.nn.Parameter(both[4:])]).init_state()
    opt = make()
    p.grad = torch.ones_like(p)
    for bad in (1.0, torch.ones(1), torch.ones(1, device="cuda").half(), torch.ones(2, device="cuda")):
        with pytest.raises(ValueError):
            opt.step(grad_factor=bad)
    p.grad = torch.ones_like(p).to_sparse()
    with pytest.raises(TypeError):
        opt.step()
    p.grad = None
    opt.init_state()
    p.data = torch.ones(9, device="cuda")
    p.grad = torch.ones_like(p)
    with pytest.raises(ValueError):
        opt.step()


def test_hooks_and_closures(cuda_device):
    p = torch.nn.Parameter(torch.ones(8, device="cuda"))
    opt = dropit.DropITAdamW([p], lr=1e-2)
    calls = []
    pre = opt.register_step_pre_hook(lambda o, args, kwargs: calls.append("pre"))
    post = opt.register_step_post_hook(lambda o, args, kwargs: calls.append("post"))

    def closure():
        calls.append("closure")
        opt.zero_grad()
        loss = (p * p).sum()
        loss.backward()
        return loss
    assert float(opt.step(closure)) == 8.0 and calls == ["pre", "closure", "post"]
    pre.remove()
    post.remove()
    with torch.no_grad():
        assert float(opt.step(closure)) < 8.0 and calls == ["pre", "closure", "post", "closure"]
    schedule = torch.optim.lr_scheduler.StepLR(opt, 1, 0.5)
    opt.step()
    schedule.step()
    assert opt.param_groups[0]["lr"] == 5e-3
    version = p._version
    opt.step()
    assert p._version == version + 1        # autograd sees that p has changed


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_tensors_of_many_runs(cuda_device, dtype):
    """Enough values that warps take whole runs of blocks, with a ragged end and small tensors around; a second step on the first one's state."""
    g = torch.Generator(device="cuda").manual_seed(6)
    sizes = [300, 27_000_037, 5, 4096 * 3 + 1]
    params = [torch.nn.Parameter((torch.randn(n, generator=g, device="cuda") * 0.1).to(dtype)) for n in sizes]
    opt = dropit.DropITAdamW(params, lr=1e-2, weight_decay=0.1, state_bits=8, seed=9)
    for t in (1, 2):
        before = []
        for p in params:
            p.grad = (torch.randn(p.shape, generator=g, device="cuda") * 0.02).to(dtype)
            s = opt.init_state(p)
            block = torch.arange(p.numel(), device="cuda") // BLOCK
            before.append((p.detach().double().clone(), s["exp_avg"].double() * s["exp_avg_scale"].double()[block],
                           (s["exp_avg_root"].double() * s["exp_avg_root_scale"].double()[block]) ** 2, block))
        opt.step()
        for p, (p0, m0, v0, block) in zip(params, before):
            s = opt.state[p]
            want, m, v, bound = _step64(p0, p.grad.double(), m0, v0, t, 1e-2, 0.1, 0.9, 0.999, 1e-8)
            if dtype == torch.bfloat16:
                bound = 2 * bound + 2.0 ** -8 * want.abs()
            assert bool(((p.detach().double() - want).abs() <= bound).all()) and int(s["step"]) == t
            # m in fp32 is off by e = 6 units (2^-24) of its terms' size (see _step64), a root by a part in 1e5 at most
            e = 6 * 2.0 ** -24 * (0.9 * m0.abs() + 0.1 * p.grad.double().abs())
            for x, off, codes, scale in ((m, e, s["exp_avg"], s["exp_avg_scale"]), (v.sqrt(), 0 * e, s["exp_avg_root"], s["exp_avg_root_scale"])):
                top = torch.nn.functional.pad(x, (0, -x.numel() % BLOCK)).view(-1, BLOCK).abs().amax(1)
                assert bool(((scale.double() - top / 448).abs() <= 1e-6 * top / 448).all())
                # Within a code's spacing: an eighth of the value, 2^-9 of the scale at least.  What is coded is x' with |x' - x| <= e, and
                # |held - x| <= spacing(x') + e <= spacing(x) + e / 8 + e: where bf16 gradients cancel 0.9 m exactly, x and x' lie on both sides of zero.
                held, unit = codes.double() * scale.double()[block], scale.double()[block]
                assert bool(((held - x).abs() <= torch.maximum(x.abs() / 8, unit * 2.0 ** -9) * (1 + 1e-5) + off * 9 / 8).all())
