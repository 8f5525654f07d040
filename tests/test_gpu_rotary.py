"""Rotary positions with several axes against the rotation in 64 bits, and their gradient."""
import math

import pytest
import torch

import paper_2202_13808_b200 as dropit

pytestmark = pytest.mark.gpu


def _reference(x, positions, sections, theta, interleaved, shared, sign=1.0):
    """x [batch, length, heads, dim] in 64 bits, one pair after the other."""
    x, rotated = x.double(), sum(sections)
    y, at = x.clone(), 0
    for axis, d in enumerate(sections):
        p = positions[..., axis].double().unsqueeze(-1)
        for i in range(d // 2):
            j = at + i
            angle = p * theta ** (-(2 * j / rotated) if shared else -(2 * i / d))
            c, s = torch.cos(angle), sign * torch.sin(angle)
            a, b = (2 * j, 2 * j + 1) if interleaved else (j, j + rotated // 2)
            y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., a] * s + x[..., b] * c
        at += d // 2
    return y


def _partner_size(x, sections, interleaved):
    """|a| + |b| of the pair that each channel belongs to (the channel's own size where it is not rotated)."""
    x, rotated = x.double().abs(), sum(sections)
    size = x.clone()
    if interleaved:
        size[..., 0:rotated:2] = size[..., 1:rotated:2] = x[..., 0:rotated:2] + x[..., 1:rotated:2]
    else:
        h = rotated // 2
        size[..., :h] = size[..., h:rotated] = x[..., :h] + x[..., h:rotated]
    return size


def _check(got, x, positions, sections, theta, interleaved, shared, sign=1.0):
    """The angle is off by half a unit of fp32 in half turns (2^-25 pi) and 2^-31 of a turn, sine and cosine by two units (2^-23), two
    products and a sum by three halves of a unit: below 5e-7 (|a| + |b|) in all.  bf16 results are rounded once (2^-8)."""
    want = _reference(x, positions, sections, theta, interleaved, shared, sign)
    bound = 1e-6 * _partner_size(x, sections, interleaved) + 1e-37
    if got.dtype == torch.bfloat16:
        bound = bound * (1 + 2.0 ** -8) + 2.0 ** -8 * want.abs()
    assert got.dtype == x.dtype and got.shape == x.shape
    assert bool(((got.double() - want).abs() <= bound).all())


# batch, length, query and key heads, head_dim, sections: whole vectors of 8 and of 4, odd numbers of pairs, heads that are rotated in part, one axis,
# an axis without channels, one token and many; more heads than are looked up at once, more units in a head than threads in a block, tiny heads.
SHAPES = [(2, 197, 12, 12, 64, (32, 32)), (1, 1, 16, 4, 128, (48, 40, 40)), (3, 37, 3, 1, 40, (20, 20)), (2, 19, 2, 2, 34, (10, 12, 6)),
          (1, 1000, 5, 3, 96, (32, 0, 32)), (5, 7, 1, 1, 2, (2,)), (1, 3, 2, 1, 512, (256, 256)), (4, 50, 6, 2, 72, (24, 24, 16, 8)),
          (1, 3, 1100, 7, 16, (16,)), (2, 2, 2, 1, 4096, (256, 256)), (3, 90, 1, 1, 16, (8, 8))]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("shape", SHAPES)
def test_rotation(cuda_device, shape, interleaved, dtype):
    B, L, hq, hk, D, sections = shape
    shared = L % 2 == 0
    g = torch.Generator(device=cuda_device).manual_seed(L)
    q = torch.randn(B, L, hq, D, generator=g, device=cuda_device).to(dtype)
    k = torch.randn(B, L, hk, D, generator=g, device=cuda_device).to(dtype)
    positions = torch.randint(-50, 5000, (B, L, len(sections)), generator=g, device=cuda_device, dtype=torch.int32)
    plan = dropit.dropit_rotary_plan(D, sections, 100.0, interleaved, shared)
    q2, k2 = dropit.dropit_rotary(q, k, positions, plan)
    _check(q2, q, positions, sections, 100.0, interleaved, shared)
    _check(k2, k, positions, sections, 100.0, interleaved, shared)
    back, none = dropit.dropit_rotary(q2, None, positions, plan, inverse=True)
    assert none is None
    _check(back, q2, positions, sections, 100.0, interleaved, shared, -1.0)
    # one set of positions for all sequences, as a matrix and with a batch of one; a single sequence without a batch
    one = positions[0]
    q3, _ = dropit.dropit_rotary(q, None, one, plan)
    q4, _ = dropit.dropit_rotary(q, None, one.unsqueeze(0), plan)
    q5, k5 = dropit.dropit_rotary(q[0], k[0], one, plan)
    _check(q3, q, one.unsqueeze(0), sections, 100.0, interleaved, shared)
    assert torch.equal(q3, q4) and torch.equal(q3[0], q5) and k5.shape == k[0].shape


@pytest.mark.parametrize("kind", ["int32", "int64", "fp32"])
def test_far_positions(cuda_device, kind):
    """At two billion an fp32 angle would be known to a hundred radians; fractions and large values of fp32 positions."""
    sections, L = (32, 32), 64
    g = torch.Generator(device=cuda_device).manual_seed(1)
    x = torch.randn(1, L, 2, 64, generator=g, device=cuda_device)
    if kind == "fp32":
        positions = (torch.randn(L, 2, generator=g, device=cuda_device) * 1e4).contiguous()
        positions[0] = 2.0 ** 22 + 0.5
    else:
        positions = torch.randint(-2 ** 31, 2 ** 31 - 1, (L, 2), generator=g, device=cuda_device, dtype=torch.int64)
        positions[0], positions[1] = 2 ** 31 - 1, -2 ** 31
        positions = positions.to(torch.int32 if kind == "int32" else torch.int64)
    plan = dropit.dropit_rotary_plan(64, sections, 10000.0)
    got, _ = dropit.dropit_rotary(x, None, positions, plan)
    # the reference's own angle, p * speed in 64 bits, is off by 2^31 * 2^-53 radians
    _check(got, x, positions.unsqueeze(0), sections, 10000.0, False, False)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_strides_and_places(cuda_device, dtype):
    """Queries and keys inside one projection, heads in front of the tokens, odd starts, channels with gaps, results in place."""
    B, L, H, D = 2, 21, 3, 48
    sections, plan = (24, 24), dropit.dropit_rotary_plan(48, (24, 24), 100.0, True)
    g = torch.Generator(device=cuda_device).manual_seed(2)
    positions = torch.stack([torch.arange(L, device=cuda_device) // 5, torch.arange(L, device=cuda_device) % 5], 1).int()
    want = dict(positions=positions.unsqueeze(0), sections=sections, theta=100.0, interleaved=True, shared=False)
    qkv = torch.randn(B, L, 3, H, D, generator=g, device=cuda_device).to(dtype)
    heads_first = torch.randn(B, H, L, D, generator=g, device=cuda_device).to(dtype).transpose(1, 2)
    flat = torch.randn(B * L * H * D + 1, generator=g, device=cuda_device).to(dtype)
    odd_start = flat[1:].view(B, L, H, D)
    gaps = torch.randn(B, L, H, 2 * D, generator=g, device=cuda_device).to(dtype)[..., ::2]
    expanded = torch.randn(B, L, 1, D, generator=g, device=cuda_device).to(dtype).expand(B, L, H, D)
    turned = positions.t().contiguous().t()             # axes far apart
    for x in (qkv[:, :, 1], heads_first, odd_start, gaps, expanded):
        got, other = dropit.dropit_rotary(x, qkv[:, :, 0], turned, plan)
        _check(got, x, **want)
        _check(other, qkv[:, :, 0], **want)
        assert got.is_contiguous()
    before = qkv.clone()
    a, b = dropit.dropit_rotary(qkv[:, :, 0], qkv[:, :, 1], positions, plan, in_place=True)
    assert a.data_ptr() == qkv.data_ptr()
    _check(qkv[:, :, 0], before[:, :, 0], **want)
    _check(qkv[:, :, 1], before[:, :, 1], **want)
    assert torch.equal(qkv[:, :, 2], before[:, :, 2])
    for x in (gaps, expanded):
        with pytest.raises(ValueError):
            dropit.dropit_rotary(x, None, positions, plan, in_place=True)


def test_gradient_is_the_inverse_rotation(cuda_device):
    rot = dropit.DropITRotary(32, (16, 8), theta=100.0)
    g = torch.Generator(device=cuda_device).manual_seed(3)
    q = torch.randn(2, 9, 4, 32, generator=g, device=cuda_device).requires_grad_(True)
    k = torch.randn(2, 9, 2, 32, generator=g, device=cuda_device).requires_grad_(True)
    positions = torch.randint(0, 40, (9, 2), generator=g, device=cuda_device)
    dq, dk = torch.randn(q.shape, generator=g, device=cuda_device), torch.randn(k.shape, generator=g, device=cuda_device)
    q2, k2 = rot(q, k, positions)
    gq, gk = torch.autograd.grad((q2, k2), (q, k), (dq, dk), create_graph=True)
    for got, d in ((gq, dq), (gk, dk)):
        _check(got.detach(), d, positions.unsqueeze(0), (16, 8), 100.0, False, False, -1.0)
    # against differences: the map is linear, so a step of any size will do
    with torch.no_grad():
        step = torch.randn(q.shape, generator=g, device=cuda_device)
        moved = ((rot(q + step, None, positions)[0].double() - rot(q - step, None, positions)[0].double()) / 2 * dq.double()).sum()
        size = (step.abs().double().sum() + q.abs().double().sum()) * dq.abs().max().double()
    assert abs(float(moved - (gq.double() * step.double()).sum())) <= 4e-6 * float(size)
    # only one of the two outputs is used
    only, = torch.autograd.grad(rot(q, k, positions)[1].sum(), k)
    assert bool(torch.isfinite(only).all())
    # and the gradient can be differentiated again
    dq2 = dq.clone().requires_grad_(True)
    first, = torch.autograd.grad(rot(q, None, positions)[0], q, dq2, create_graph=True)
    second, = torch.autograd.grad(first, dq2, step)
    _check(second, step, positions.unsqueeze(0), (16, 8), 100.0, False, False)


def test_infinities_and_nans_stay_in_their_pair(cuda_device):
    plan = dropit.dropit_rotary_plan(16, (16,), 100.0)
    x = torch.ones(1, 3, 2, 16, device=cuda_device)
    x[0, 1, 0, 2], x[0, 2, 1, 9] = float("nan"), float("inf")
    y, _ = dropit.dropit_rotary(x, None, torch.tensor([[1], [2], [3]], device=cuda_device), plan)
    bad = ~torch.isfinite(y)
    assert bad.nonzero().tolist() == [[0, 1, 0, 2], [0, 1, 0, 10], [0, 2, 1, 1], [0, 2, 1, 9]]


def test_empty_tensors(cuda_device):
    plan = dropit.dropit_rotary_plan(16, (16,))
    for shape in ((0, 5, 2, 16), (2, 0, 2, 16), (2, 5, 0, 16)):
        x = torch.empty(shape, device=cuda_device)
        y, _ = dropit.dropit_rotary(x, None, torch.zeros(shape[1], 1, dtype=torch.int32, device=cuda_device), plan)
        assert y.shape == x.shape


def test_captured_and_on_a_stream_of_its_own(cuda_device):
    plan = dropit.dropit_rotary_plan(64, (64,), 10000.0)
    q = torch.randn(4, 1, 8, 64, device=cuda_device)
    positions = torch.full((4, 1, 1), 7, dtype=torch.int64, device=cuda_device)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        first, _ = dropit.dropit_rotary(q, None, positions, plan)
    torch.cuda.current_stream().wait_stream(stream)
    _check(first, q, positions, (64,), 10000.0, False, False)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, _ = dropit.dropit_rotary(q, None, positions, plan)
    for _ in range(3):
        positions += 1
        graph.replay()
        _check(out, q, positions, (64,), 10000.0, False, False)


def test_refusals(cuda_device):
    plan = dropit.dropit_rotary_plan(16, (8, 8))
    x, p = torch.zeros(1, 4, 2, 16, device=cuda_device), torch.zeros(4, 2, dtype=torch.int32, device=cuda_device)
    cases = [(x[..., :8], x, p, ValueError), (x, x[:, :3], p, ValueError), (x, x, p[:3], ValueError), (x, x, p[:, :1], ValueError),
             (x.half(), x, p, TypeError), (x, x.bfloat16(), p, TypeError), (x, x, p.half(), TypeError), (x.cpu(), x, p, ValueError),
             (x, x, p.cpu(), ValueError), (x[0, 0], None, p, ValueError), (x, x, p.expand(3, 4, 2), ValueError)]
    for q, k, positions, error in cases:
        with pytest.raises(error):
            dropit.dropit_rotary(q, k, positions, plan)
    with pytest.raises(ValueError):
        dropit.dropit_rotary(x, x, p, plan[:-1])
    both = torch.zeros(1, 4, 4, 16, device=cuda_device)
    for q, k in ((x, x), (both[:, :, :3], both[:, :, 2:])):
        with pytest.raises(ValueError, match="share"):
            dropit.dropit_rotary(q, k, p, plan, in_place=True)
    dropit.dropit_rotary(both[:, :, :2], both[:, :, 2:], p, plan, in_place=True)
    dropit.dropit_rotary(both[:, :, :1], both[:, :, 1:], p, plan, in_place=True)
    dropit.dropit_rotary(both[:, :, 3:], both[:, :, :3], p, plan, in_place=True)


def test_a_token_far_into_a_batch_of_more_than_two_to_the_31_values(cuda_device):
    """Offsets that pass 32 bits: 2.2 billion bf16 values, of which the last token is looked at."""
    if torch.cuda.mem_get_info(cuda_device)[0] < 12 * 2 ** 30:
        pytest.skip("needs 12 GB")
    D, H, L = 128, 16, 2 ** 20 + 2 ** 16
    x = torch.zeros(1, L, H, D, dtype=torch.bfloat16, device=cuda_device)
    assert x.numel() > 2 ** 31
    x[0, -1] = torch.randn(H, D, device=cuda_device).bfloat16()
    positions = torch.arange(L, dtype=torch.int32, device=cuda_device).unsqueeze(1)
    y, _ = dropit.dropit_rotary(x, None, positions, dropit.dropit_rotary_plan(D, (D,)))
    _check(y[:, -1:], x[:, -1:], positions[None, -1:], (D,), 10000.0, False, False)
    assert not bool(y[0, :-1].any())
