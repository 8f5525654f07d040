"""AdamW at the ends of fp32's range, and the forms of the step one by one: 8-bit moments against the same operations in fp32, bit by bit."""
import numpy as np
import pytest
import torch

import paper_2202_13808_b200 as dropit
from test_gpu_adamw import BLOCK, _code_values, _step64, _words

pytestmark = pytest.mark.gpu

f32 = np.float32


def _codes(values, scale, amax, words16, keep_above_zero):
    """Codes of a block's values as include/dropit.h states them, every operation rounded to fp32: a product with the scale's reciprocal, and the
    place between two codes plus the random fraction."""
    with np.errstate(divide="ignore", over="ignore", invalid="ignore"):
        y = (np.abs(values) * np.where(scale > 0, f32(1) / scale, f32(0)).astype(f32)).astype(f32)
    table = _code_values().astype(np.float64)
    y = y.astype(np.float64)
    low = np.clip(np.searchsorted(table, y, side="right") - 1, 0, len(table) - 1)
    high = np.minimum(low + 1, len(table) - 1)
    gap = np.where(high > low, table[high] - table[low], 1.0)
    # the place is held in 20 bits of the normal codes, and rounded to them below
    place = np.clip((y - table[low]) / gap, 0, 1)
    held = np.rint(place * 2 ** 20) / 2 ** 20
    code = table[np.where(held + words16.astype(np.float64) / 65536 >= 1, high, low)]
    if keep_above_zero:
        code = np.where((values > 0) & (code == 0), table[1], code)
    sure = (held == place) | (np.abs(held + words16 / 65536.0 - 1) > 2.0 ** -19)
    return code * np.sign(np.where(values == 0, 0, values)), sure


def _emulate(g, m0, r0, b1, b2, factor):
    """m and the root in fp32, each operation rounded by itself."""
    with np.errstate(over="ignore", under="ignore"):
        one1, one2 = f32(1.0 - b1), f32(1.0 - b2)
        if factor is not None:
            g = (g * f32(factor)).astype(f32)
        m = ((f32(b1) * m0).astype(f32) + (one1 * g).astype(f32)).astype(f32)
        v = ((f32(b2) * (r0 * r0).astype(f32)).astype(f32) + ((one2 * g).astype(f32) * g).astype(f32)).astype(f32)
        return m, np.sqrt(v)


@pytest.mark.parametrize("span", [(-3, 3), (-62, -30), (-75, -60), (0, 60)])
@pytest.mark.parametrize("factor", [None, 0.37])
def test_8_bit_moments_are_those_of_fp32_operations(cuda_device, span, factor):
    """Scales bit by bit and codes wherever the 20 bits of a place decide, for gradients of 2^-75 to 2^60: every block has a size of its own.  Roots are
    exact roots of fp32 rounded once, of v below 2^-126 too."""
    blocks, b1, b2 = 4000, 0.9, 0.99
    n = blocks * BLOCK
    rng = np.random.RandomState(span[0] + 100)
    p = torch.nn.Parameter(torch.zeros(n, device=cuda_device))
    opt = dropit.DropITAdamW([p], lr=0.0, betas=(b1, b2), weight_decay=0.0, state_bits=8, seed=11)
    s = opt.init_state(p)
    scale_by = None if factor is None else torch.tensor(factor, device=cuda_device)
    for t in range(1, 4):
        size = np.exp2(rng.uniform(span[0], span[1], (blocks, 1)))
        g = (rng.randn(blocks, BLOCK) * size).astype(f32)
        block = lambda k, scale: (s[k].float().cpu().numpy().reshape(blocks, BLOCK) * s[scale].cpu().numpy()[:, None]).astype(f32)
        m, r = _emulate(g, block("exp_avg", "exp_avg_scale"), block("exp_avg_root", "exp_avg_root_scale"), b1, b2, factor)
        p.grad = torch.from_numpy(g.reshape(-1)).to(cuda_device)
        opt.step(grad_factor=scale_by)
        words, _ = _words(11, t, 0, n)
        for x, k, bits in ((m, "exp_avg", words >> 16), (r, "exp_avg_root", words & 0xFFFF)):
            top = np.abs(x).max(1)
            want = np.where(top < 1e-30, f32(0), (top * f32(1 / 448)).astype(f32))
            got = s[k + "_scale"].cpu().numpy()
            assert (got == want).all(), (k, int((got != want).sum()))
            code, sure = _codes(x, want[:, None], top[:, None], bits.reshape(blocks, BLOCK), k != "exp_avg")
            held = s[k].double().cpu().numpy().reshape(blocks, BLOCK)
            assert (held == code)[sure & (want[:, None] > 0)].all()
            assert sure.mean() > 0.99
            assert not held[want == 0].any()


@pytest.mark.parametrize("low, high", [(-126, -90), (-102, 0), (-2, 2), (0, 127)])
def test_roots_and_reciprocals_over_their_range(cuda_device, low, high):
    """One value in each of half a million blocks, b1 = b2 = 0: the scales are the values' and their roots' of fp32, and the value's own code is 448.  Roots of squares'
    neighbours, where a second moment is nearest to one whose root lies between two floats, among them."""
    n = 1 << 19
    rng = np.random.RandomState(high + 200)
    g = np.exp2(rng.uniform(low / 2, min(high / 2, 63.4), n)).astype(f32) * rng.choice([-1, 1], n).astype(f32)
    g[::4] = (np.round(np.exp2(rng.uniform(11, 12, n // 4))) * np.exp2(np.floor(np.log2(np.abs(g[::4]))) - 11)).astype(f32)
    p = torch.nn.Parameter(torch.zeros(n * BLOCK, device=cuda_device))
    opt = dropit.DropITAdamW([p], lr=0.0, betas=(0.0, 0.0), weight_decay=0.0, state_bits=8, seed=1)
    p.grad = torch.zeros_like(p)
    p.grad.view(n, BLOCK)[:, 7] = torch.from_numpy(g).to(cuda_device)
    opt.step()
    s = opt.state[p]
    with np.errstate(under="ignore"):
        root = np.sqrt((g * g).astype(f32))
        want = [(x * f32(1 / 448)).astype(f32) for x in (np.abs(g), root)]
    for k, w in zip(("exp_avg", "exp_avg_root"), want):
        assert (s[k + "_scale"].cpu().numpy() == w).all()
        # value times reciprocal is 448 but for three halves of a unit; the code below takes a fraction of 2^-16 and less
        codes = s[k].view(n, BLOCK)[:, 7].float().abs().cpu().numpy()
        assert ((codes == 448) | (codes == 416)).all() and (codes == 448).mean() > 0.999


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("size", [1e-17, 3e-19, 1e-20, 1e-21])
def test_gradients_whose_squares_are_tiny(cuda_device, bits, size):
    """v falls below 2^-126, where fp32 has fewer digits but still a root.  eps = 0: the first step moves every value by lr, whatever the gradients' size."""
    p = torch.nn.Parameter(torch.zeros(2 * BLOCK, device=cuda_device))
    opt = dropit.DropITAdamW([p], lr=1.0, betas=(0.9, 0.99), eps=0.0, weight_decay=0.0, state_bits=bits)
    p.grad = torch.full_like(p, size)
    opt.step()
    # v = 0.01 size^2 is off by half of 2^-149, 7.0e-46: for 1e-21 (1e-44) a part in 14, half of that for the root
    assert bool(((p.detach() + 1).abs() <= 1e-5 + 0.6 * 7.1e-46 / (0.01 * size * size) + 7.1e-46 / (size * size) * (bits == 32)).all())
    s = opt.state[p]
    root = s["exp_avg_root"].double() * s["exp_avg_root_scale"].double()[0] if bits == 8 else s["exp_avg_sq"].double().sqrt()
    assert bool((root / (0.1 * size) - 1).abs().max() <= 0.12)          # half of 7 % of v, and the next code below the largest


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("size, factor", [(1e20, 1e-20), (1e-3, 1e3), (3e30, 1e-31), (1e-18, 1e18)])
def test_a_factor_holds_for_the_gradients_and_not_for_their_squares(cuda_device, bits, size, factor):
    """Gradients of a loss that is scaled or far off: their squares leave fp32's range, what they are after the factor does not."""
    g = torch.randn(3 * BLOCK, generator=torch.Generator(device=cuda_device).manual_seed(1), device=cuda_device)
    p, q = (torch.nn.Parameter(torch.zeros(3 * BLOCK, device=cuda_device)) for _ in range(2))
    make = lambda t: dropit.DropITAdamW([t], lr=1e-2, weight_decay=0.0, state_bits=bits, seed=3)
    a, b = make(p), make(q)
    p.grad = g * size
    factor = torch.tensor(factor, device=cuda_device)
    q.grad = p.grad * factor
    a.step(grad_factor=factor)
    b.step()
    assert torch.equal(p, q)
    assert all(torch.equal(x.float(), y.float()) for x, y in zip(a.state[p].values(), b.state[q].values()))


FORMS = [(bits, master, dither) for bits in (8, 32) for master in (False, True) for dither in (False, True)]


@pytest.mark.parametrize("bits, master, dither", FORMS)
@pytest.mark.parametrize("g_type", [torch.float32, torch.bfloat16])
def test_every_form_of_a_bf16_step(cuda_device, bits, master, dither, g_type):
    """Parameters rounded to nearest or with a dither, stepped as they are or in an fp32 copy; from held moments, against 64 bits."""
    shapes = [(5,), (300,), (64, 33), (2, 3, 5, 7)]
    gen = torch.Generator(device=cuda_device).manual_seed(2)
    draw = lambda s: torch.randn(s, generator=gen, device=cuda_device)
    params = [torch.nn.Parameter((draw(s) * 0.1).bfloat16()) for s in shapes]
    opt = dropit.DropITAdamW(params, lr=3e-3, betas=(0.9, 0.99), weight_decay=0.1, state_bits=bits, master=master, dither=dither, seed=21)
    opt.init_state()
    factor = torch.tensor(0.7, device=cuda_device)
    for t in range(1, 4):
        held = []
        for p in params:
            p.grad_dtype = None
            p.grad = (draw(p.shape) * 0.02).to(g_type)
            s = opt.state[p]
            block = torch.arange(p.numel(), device=cuda_device) // BLOCK
            if bits == 8:
                m0 = s["exp_avg"].double().reshape(-1) * s["exp_avg_scale"].double()[block]
                v0 = (s["exp_avg_root"].double().reshape(-1) * s["exp_avg_root_scale"].double()[block]) ** 2
            else:
                m0, v0 = s["exp_avg"].double().reshape(-1), s["exp_avg_sq"].double().reshape(-1)
            held.append(((s["master"] if master else p.detach()).double().reshape(-1).clone(), m0.clone(), v0.clone()))
        opt.step(grad_factor=factor)
        for ordinal, (p, (p0, m0, v0)) in enumerate(zip(params, held)):
            g = (p.grad.float() * factor).double().reshape(-1)
            want, m, v, bound = _step64(p0, g, m0, v0, t, 3e-3, 0.1, 0.9, 0.99, 1e-8)
            s, n = opt.state[p], p.numel()
            _, other = _words(21, t, ordinal, n)
            fraction = (other >> np.uint32(16)).astype(np.uint32)
            now = p.detach().reshape(-1)
            if master:
                copy = s["master"].reshape(-1)
                assert bool(((copy.double() - want).abs() <= bound).all())
                if dither:              # the copy's pattern plus the fraction, cut to its high half
                    sums = copy.cpu().numpy().view(np.uint32) + fraction
                    assert (now.view(torch.int16).cpu().numpy().view(np.uint16) == (sums >> np.uint32(16)).astype(np.uint16)).all()
                else:
                    assert torch.equal(now, copy.bfloat16())
            elif dither:
                w = want.cpu().numpy()
                unit = np.exp2(np.floor(np.log2(np.maximum(np.abs(w), 1e-38))) - 7)
                total = np.abs(w) / unit + fraction / 65536.0
                # the fp32 value is off by `bound`, and its last 2^-16 of a unit count
                sure = np.abs(total - np.round(total)) > bound.cpu().numpy() / unit + 2.0 ** -15
                assert sure.mean() > 0.9 or n < 100
                assert (now.double().abs().cpu().numpy() == np.floor(total) * unit)[sure].all()
            else:
                assert bool(((now.double() - want).abs() <= 2 * bound + 2.0 ** -8 * want.abs()).all())
            if bits == 32:
                assert bool(((s["exp_avg"].double().reshape(-1) - m).abs() <= 6 * 2.0 ** -24 * (0.9 * m0.abs() + 0.1 * g.abs()) + 1e-40).all())
                assert bool(((s["exp_avg_sq"].double().reshape(-1) - v).abs() <= 6 * 2.0 ** -24 * v + 1e-40).all())
            else:
                block = torch.arange(n, device=cuda_device) // BLOCK
                for x, k in ((m, "exp_avg"), (v.sqrt(), "exp_avg_root")):
                    scale = s[k + "_scale"].double()[block]
                    off = 6 * 2.0 ** -24 * (0.9 * m0.abs() + 0.1 * g.abs())
                    assert bool(((s[k].double().reshape(-1) * scale - x).abs() <= torch.maximum(x.abs() / 8, scale * 2.0 ** -9) * (1 + 1e-5) + 9 / 8 * off).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("bits", [8, 32])
def test_what_lies_beside_a_parameter_stays(cuda_device, dtype, bits):
    flat = torch.randn(4003, device=cuda_device).to(dtype)
    spans = [(1, 1000), (1003, 1004), (1024, 1024 + 256), (2001, 4000)]
    kept = flat.clone()
    params = [torch.nn.Parameter(flat[a:b]) for a, b in spans]
    opt = dropit.DropITAdamW(params, lr=1e-1, state_bits=bits)
    for p in params:
        p.grad = torch.ones_like(p)
    opt.step()
    inside = torch.zeros(4003, dtype=torch.bool, device=cuda_device)
    for a, b in spans:
        inside[a:b] = True
    assert torch.equal(flat[~inside], kept[~inside]) and not bool((flat[inside] == kept[inside]).any())
