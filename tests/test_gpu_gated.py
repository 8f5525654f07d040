"""The gated linear against 64-bit arithmetic: both products, gates, kept projections, the three gradients, the layer around them."""
import math

import pytest
import torch

import paper_2202_13808_b200 as dropit

pytestmark = pytest.mark.gpu

U = 2.0 ** -8           # half a unit of bf16, relative
GATES = ["silu", "gelu", "relu"]


def _gate64(a, gate):
    if gate == "silu":
        s = torch.sigmoid(a)
        return a * s, s + a * s * torch.sigmoid(-a)
    if gate == "gelu":
        phi = torch.special.ndtr(a)
        return a * phi, phi + a * torch.exp(-a * a / 2) / math.sqrt(2 * math.pi)
    return a.clamp_min(0), (a > 0).double()


def _inputs(M, C, H, dtype, device, bias=True, scale=1.0):
    g = torch.Generator(device=device).manual_seed(M * 7 + C * 3 + H)
    draw = lambda *s: torch.randn(*s, generator=g, device=device)
    x = (draw(M, C) * scale).to(dtype)
    w = (draw(2 * H, C) * C ** -0.5).to(dtype)
    b = (draw(2 * H) * 0.1).to(dtype) if bias else None
    return x, w, b, draw(M, H).to(dtype)


def _unit(dtype):
    return U if dtype == torch.bfloat16 else 2.0 ** -24


def _check_forward(x, w, b, gate, h, gu=None):
    """a and u: fp32 sums of C exact products, C half units of the sum of magnitudes; f is off by a few units and moves by its slope (at most 1.13)
    times a's error; one rounding."""
    C, H = w.shape[1], w.shape[0] // 2
    xd, wd = x.double().reshape(-1, C), w.double()
    both, size = xd @ wd.t(), xd.abs() @ wd.abs().t()
    if b is not None:
        both, size = both + b.double(), size + b.double().abs()
    off = (C + 1) * 2.0 ** -24 * size
    unit = _unit(x.dtype)
    if gu is not None:
        assert bool(((gu.double().reshape(-1, 2 * H) - both).abs() <= off + unit * (both.abs() + off) + 1e-37).all())
    a, u, da, du = both[:, :H], both[:, H:], off[:, :H], off[:, H:]
    f, _ = _gate64(a, gate)
    df = 1.13 * da + 2e-6 * a.abs()
    bound = f.abs() * du + u.abs() * df + df * du
    bound = bound + unit * ((f * u).abs() + bound) + 1e-37
    assert h.dtype == x.dtype and bool(((h.double().reshape(-1, H) - f * u).abs() <= bound).all())


def _check_backward(dh, gu, gate, dgu, db):
    H = dh.shape[-1]
    d, a, u = dh.double().reshape(-1, H), gu.double().reshape(-1, 2 * H)[:, :H], gu.double().reshape(-1, 2 * H)[:, H:]
    f, slope = _gate64(a, gate)
    want = torch.cat([d * u * slope, d * f], 1)
    # value and slope are off by a few units of fp32 of terms of up to 1 + |a|, below 2e-6; products of three factors
    off = torch.cat([(d * u).abs(), d.abs()], 1) * 2e-6 * torch.cat([1 + a.abs(), 1 + a.abs()], 1)
    unit = _unit(dh.dtype)
    assert bool(((dgu.double().reshape(-1, 2 * H) - want).abs() <= unit * (want.abs() + off) + off + 1e-37).all())
    if db is not None:
        M = d.shape[0]
        bound = M * 2.0 ** -24 * want.abs().sum(0) + off.sum(0)
        assert bool(((db.double() - want.sum(0)).abs() <= bound + unit * (want.sum(0).abs() + bound) + 1e-37).all())


def _check_input_grad(dgu, w, dx):
    K = w.shape[0]
    want, size = dgu.double().reshape(-1, K) @ w.double(), dgu.double().abs().reshape(-1, K) @ w.double().abs()
    bound = K * 2.0 ** -24 * size
    assert bool(((dx.double().reshape(-1, w.shape[1]) - want).abs() <= bound + _unit(dx.dtype) * (want.abs() + bound) + 1e-37).all())


# rows x channels x hidden: one token and few, rows around the tiles' edges, widths that are multiples of 8 around 64, 128 and 256 and some that
# are not, hidden widths where the gate's last tile would run into the other half, long sums
SHAPES = [(1, 64, 8), (1, 768, 2048), (2, 200, 136), (7, 136, 264), (8, 768, 2048), (9, 520, 72), (17, 64, 128), (33, 1024, 512), (100, 8, 8),
          (127, 72, 120), (128, 128, 128), (129, 192, 200), (255, 256, 384), (257, 264, 136), (591, 768, 2048), (1000, 328, 1000), (3000, 192, 512),
          (1, 3, 5), (13, 37, 101), (65, 65, 65), (130, 100, 36)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("shape", SHAPES)
def test_products_and_gradients(cuda_device, shape, dtype):
    M, C, H = shape
    gate = GATES[(M + C + H) % 3]
    bias = (M + H) % 2 == 0
    x, w, b, dh = _inputs(M, C, H, dtype, cuda_device, bias)
    h, gu = dropit.dropit_gated_linear(x, w, b, gate, keep=True)
    _check_forward(x, w, b, gate, h, gu)
    alone = dropit.dropit_gated_linear(x, w, b, gate)
    _check_forward(x, w, b, gate, alone)
    dgu, db = dropit.dropit_gated_linear_backward(dh, gu, gate, bias_grad=True)
    _check_backward(dh, gu, gate, dgu, db)
    assert torch.equal(dropit.dropit_gated_linear_backward(dh, gu, gate), dgu)
    dx = dropit.dropit_gated_input_grad(dgu, w)
    _check_input_grad(dgu, w, dx)
    dropit.check_device_status(cuda_device)
    # the same again: every sum has an order of its own
    again = dropit.dropit_gated_linear(x, w, b, gate, keep=True)
    assert torch.equal(again[0], h) and torch.equal(again[1], gu)
    assert torch.equal(dropit.dropit_gated_input_grad(dgu, w), dx)
    assert torch.equal(dropit.dropit_gated_linear_backward(dh, gu, gate, bias_grad=True)[1], db)


@pytest.mark.parametrize("gate", GATES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("M", [3, 300])
def test_gates_over_their_range(cuda_device, gate, dtype, M):
    """Projections from 2^-20 to 200 of both signs: tails, saturation, the middle.  x holds them and W is the identity."""
    H = 64
    g = torch.Generator(device=cuda_device).manual_seed(9)
    a = torch.exp2(torch.rand(M, H, generator=g, device=cuda_device) * 27.6 - 20) * torch.sign(torch.randn(M, H, generator=g, device=cuda_device))
    a[0, :6] = torch.tensor([0.0, -0.0, 88.0, -88.0, -150.0, 150.0], device=cuda_device)
    u = torch.randn(M, H, generator=g, device=cuda_device)
    x = torch.cat([a, u], 1).to(dtype)
    w = torch.eye(2 * H, device=cuda_device).to(dtype)
    h, gu = dropit.dropit_gated_linear(x, w, None, gate, keep=True)
    assert torch.equal(gu, x + 0.0)
    _check_forward(x, w, None, gate, h, gu)
    dgu, db = dropit.dropit_gated_linear_backward(u.to(dtype), gu, gate, bias_grad=True)
    _check_backward(u.to(dtype), gu, gate, dgu, db)


@pytest.mark.parametrize("M, C, H", [(5, 64, 40), (300, 72, 264), (40, 33, 20)])
def test_infinities_and_nans_reach_their_rows_only(cuda_device, M, C, H):
    x, w, b, dh = _inputs(M, C, H, torch.bfloat16, cuda_device)
    clean = dropit.dropit_gated_linear(x, w, b)
    x[1, 3], x[M - 1, 0] = float("nan"), float("inf")
    h, gu = dropit.dropit_gated_linear(x, w, b, keep=True)
    rows = torch.ones(M, dtype=torch.bool, device=cuda_device)
    rows[1] = rows[M - 1] = False
    assert torch.equal(h[rows], clean[rows])
    assert bool(torch.isnan(h[1]).all()) and not bool(torch.isfinite(gu[M - 1]).any())
    dgu = dropit.dropit_gated_linear_backward(dh, gu)
    dx = dropit.dropit_gated_input_grad(dgu, w)
    assert bool(torch.isfinite(dx[rows]).all()) and bool(torch.isnan(dx[1]).all())


def test_a_pass_with_nothing_in_it(cuda_device):
    x, w, b, _ = _inputs(1, 64, 16, torch.bfloat16, cuda_device)
    h, gu = dropit.dropit_gated_linear(x[:0], w, b, keep=True)
    assert h.shape == (0, 16) and gu.shape == (0, 32)
    dgu, db = dropit.dropit_gated_linear_backward(h, gu, bias_grad=True)
    assert dgu.shape == (0, 32) and not bool(db.any())
    assert dropit.dropit_gated_input_grad(dgu, w).shape == (0, 64)


def _layer(C, H, dtype, device, gamma, gate="silu", bias=True):
    torch.manual_seed(C + H)
    return dropit.DropITGatedLinear(C, H, bias=bias, gate=gate, gamma=gamma, device=device, dtype=dtype).train()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("shape, gamma, bias", [((2, 61, 72), 0.9, True), ((500, 256), 0.5, False), ((33, 37), 0.8, True), ((4, 200, 64), 0.0, True)])
def test_the_layer_is_its_parts(cuda_device, shape, gamma, bias, dtype):
    C, H = shape[-1], 88
    layer = _layer(C, H, dtype, cuda_device, gamma, bias=bias)
    g = torch.Generator(device=cuda_device).manual_seed(1)
    x = torch.randn(shape, generator=g, device=cuda_device).to(dtype).requires_grad_(True)
    dh = torch.randn(*shape[:-1], H, generator=g, device=cuda_device).to(dtype)
    h = layer(x)
    h.backward(dh)
    with torch.no_grad():
        x2 = x.detach().reshape(-1, C)
        want, gu = dropit.dropit_gated_linear(x2, layer.weight, layer.bias, "silu", keep=True)
        dgu, db = dropit.dropit_gated_linear_backward(dh.reshape(-1, H), gu, "silu", bias_grad=True)
        kept = dropit.dropit_decompress(dropit.dropit_compress(x2, gamma)).double()
    assert torch.equal(h.reshape(-1, H), want) and h.shape == dh.shape
    assert torch.equal(x.grad.reshape(-1, C), dropit.dropit_gated_input_grad(dgu, layer.weight.detach()))
    if bias:
        assert torch.equal(layer.bias.grad, db)
    dw, size = dgu.double().t() @ kept, dgu.double().abs().t() @ kept.abs()
    bound = x2.shape[0] * 2.0 ** -24 * size
    assert bool(((layer.weight.grad.double() - dw).abs() <= bound + _unit(dtype) * (dw.abs() + bound) + 1e-37).all())
    layer.eval()
    with torch.no_grad():
        _check_forward(x2, layer.weight, layer.bias, "silu", layer(x))
    assert torch.allclose(layer(x).float(), h.float(), rtol=0.05, atol=0.05)      # gradients at inference: stock operations


@pytest.mark.parametrize("gate", GATES)
def test_gradients_against_differences(cuda_device, gate):
    """fp32, nothing dropped: the change of sum(h dh) along a direction against the gradients' share of it."""
    M, C, H = 50, 24, 20
    layer = _layer(C, H, torch.float32, cuda_device, 0.0, gate)
    g = torch.Generator(device=cuda_device).manual_seed(2)
    x = torch.randn(M, C, generator=g, device=cuda_device).requires_grad_(True)
    dh = torch.randn(M, H, generator=g, device=cuda_device)
    layer(x).backward(dh)
    leaves = [x, layer.weight, layer.bias]
    steps = [torch.randn(t.shape, generator=g, device=cuda_device) for t in leaves]
    eps = 2.0 ** -7 if gate != "relu" else 2.0 ** -12
    start = [t.detach().clone() for t in leaves]
    sums = []
    with torch.no_grad():
        for sign in (1, -1):
            moved = [t + sign * eps * s for t, s in zip(start, steps)]
            sums.append((dropit.dropit_gated_linear(moved[0], moved[1], moved[2], gate).double() * dh.double()).sum())
    want = sum((t.grad.double() * s.double()).sum() for t, s in zip(leaves, steps))
    got = (sums[0] - sums[1]) / (2 * eps)
    # third-order terms: eps^2 times a few of the gradient's size; fp32 noise of the sums: 1e-6 sqrt(M H) / eps; a ReLU's corners: the few a
    # within eps of zero
    scale = sum((t.grad.double().abs() * s.double().abs()).sum() for t, s in zip(leaves, steps))
    assert abs(float(got - want)) <= 0.02 * float(scale)


def test_needs_of_the_caller(cuda_device):
    layer = _layer(64, 32, torch.bfloat16, cuda_device, 0.5)
    x = torch.randn(40, 64, device=cuda_device, dtype=torch.bfloat16)
    layer(x).sum().backward()                                   # x needs no gradient
    assert layer.weight.grad is not None and x.grad is None
    layer.weight.requires_grad_(False)
    layer.weight.grad = None
    x.requires_grad_(True)
    layer(x).sum().backward()
    assert layer.weight.grad is None and x.grad is not None
    layer.weight.requires_grad_(True)
    dx, = torch.autograd.grad(layer(x).float().sum(), x, create_graph=True)
    with pytest.raises(RuntimeError, match="cannot be differentiated again"):
        dx.float().sum().backward()
    # gradients that are expanded or start anywhere, inputs with gaps
    ones = torch.ones(1, device=cuda_device, dtype=torch.bfloat16).expand(40, 32)
    wide = torch.randn(40, 129, device=cuda_device, dtype=torch.bfloat16)[:, 1:65].detach().requires_grad_(True)
    layer(wide).backward(ones)
    y = wide.detach().contiguous().requires_grad_(True)
    layer(y).backward(ones.contiguous())
    assert torch.equal(wide.grad, y.grad)
    with torch.autocast("cuda", dtype=torch.bfloat16):
        full = _layer(64, 32, torch.float32, cuda_device, 0.5)
        h = full(torch.randn(8, 64, device=cuda_device))
        assert h.dtype == torch.bfloat16
        h.float().sum().backward()
    assert full.weight.grad.dtype == torch.float32


def test_captured_passes(cuda_device):
    """Forward and backward pass in one graph, replayed on other inputs."""
    layer = _layer(72, 136, torch.bfloat16, cuda_device, 0.5)
    x = torch.randn(300, 72, device=cuda_device, dtype=torch.bfloat16).requires_grad_(True)
    dh = torch.randn(300, 136, device=cuda_device, dtype=torch.bfloat16)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        for _ in range(2):
            torch.autograd.grad(layer(x), (x, layer.weight, layer.bias), dh)
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        h = layer(x)
        grads = torch.autograd.grad(h, (x, layer.weight, layer.bias), dh)
    for _ in range(2):
        with torch.no_grad():
            x.copy_(torch.randn_like(x))
        graph.replay()
        want = layer(x)
        for got, ref in zip((h, *grads), (want, *torch.autograd.grad(want, (x, layer.weight, layer.bias), dh))):
            assert torch.equal(got, ref)
    dropit.check_device_status(cuda_device)


def test_refusals(cuda_device):
    x, w, b, dh = _inputs(4, 16, 8, torch.bfloat16, cuda_device)
    cases = [((x.half(), w, b), TypeError), ((x.float(), w, b), TypeError), ((x, w, b.float()), TypeError), ((x[:, :8], w, b), ValueError),
             ((x, w[:15], b), ValueError), ((x, w, b[:8]), ValueError), ((x.cpu(), w, b), ValueError), ((x, w.cpu(), b), ValueError),
             ((x, w[0], b), ValueError)]
    for args, error in cases:
        with pytest.raises(error):
            dropit.dropit_gated_linear(*args)
    with pytest.raises(ValueError):
        dropit.dropit_gated_linear(x, w, b, gate="tanh")
    _, gu = dropit.dropit_gated_linear(x, w, b, keep=True)
    for args, error in [((dh[:, :4], gu), ValueError), ((dh[:3], gu), ValueError), ((dh.float(), gu), TypeError)]:
        with pytest.raises(error):
            dropit.dropit_gated_linear_backward(*args)
    for args, error in [((gu[:, :8], w), ValueError), ((gu, w.float()), TypeError), ((gu.cpu(), w), ValueError)]:
        with pytest.raises(error):
            dropit.dropit_gated_input_grad(*args)


@pytest.mark.parametrize("M, C, H", [(4100, 1024, 1152), (200, 768, 2048)])      # many tiles a pair; pairs that share dx's summed axis
def test_waits_that_run_out_are_reported(cuda_device, monkeypatch, M, C, H):
    x, w, b, dh = _inputs(M, C, H, torch.bfloat16, cuda_device)

    def both():
        h, gu = dropit.dropit_gated_linear(x, w, b, keep=True)
        return h, gu, dropit.dropit_gated_input_grad(kept, w)
    kept = dropit.dropit_gated_linear(x, w, b, keep=True)[1]
    good = both()
    dropit.check_device_status(cuda_device)
    monkeypatch.setenv("DROPIT_TEST_SPIN_LIMIT", "1")
    timed_out = 0
    for _ in range(3):
        out = both()                                             # must return
        try:
            dropit.check_device_status(cuda_device)
            assert all(torch.equal(p, q) for p, q in zip(out, good))
        except dropit.DropITError as e:
            assert e.code == 5
            timed_out += 1
    monkeypatch.delenv("DROPIT_TEST_SPIN_LIMIT")
    assert all(torch.equal(p, q) for p, q in zip(both(), good))
    dropit.check_device_status(cuda_device)
    assert timed_out >= 1


def test_the_graph_is_freed_and_saved_tensors_can_be_hooked(cuda_device):
    layer = _layer(64, 32, torch.bfloat16, cuda_device, 0.9)
    x = torch.randn(512, 64, device=cuda_device, dtype=torch.bfloat16).requires_grad_(True)
    h = layer(x)
    h.sum().backward()
    with pytest.raises(RuntimeError, match="second time"):
        h.sum().backward()
    h = layer(x)
    h.sum().backward(retain_graph=True)
    h.sum().backward()
    packed = []
    with torch.autograd.graph.saved_tensors_hooks(lambda t: packed.append(t.numel() * t.element_size()) or t.cpu(), lambda t: t.to(cuda_device)):
        h = layer(x)
    grad = x.grad.clone()
    x.grad = None
    h.sum().backward()
    assert len(packed) == 5 and x.grad is not None and grad.shape == x.grad.shape
    # what the layer holds: the gate's two projections and the cache of a tenth of x, its mask and its table, beside the weights
    assert sum(packed) < layer.weight.numel() * 2 + 512 * 64 * 2 + 0.2 * 512 * 64 * 2 + 64
    # a weight that changes between the passes is noticed
    h = layer(x)
    with torch.no_grad():
        layer.weight.add_(1)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        h.sum().backward()
