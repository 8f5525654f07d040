"""Gated blocks, rotary positions and AdamW together, as `python -m paper_2202_13808_b200.vit` uses them."""
import copy
import json
import sys

import pytest
import torch
import torch.nn as nn
import torch.nn.functional as F

import paper_2202_13808_b200 as dropit
from paper_2202_13808_b200 import vit
from paper_2202_13808_b200.nn import DropITGatedLinear, DropITLinear, convert_linear_layers

pytestmark = pytest.mark.gpu


class _Turn(nn.Module):
    """The rotation of a Block in stock operations of any type."""

    def __init__(self, of):
        super().__init__()
        self.of = of

    def forward(self, q, k, positions):
        angle = torch.cat([positions[:, a, None].double() * self.of.theta ** -(torch.arange(d // 2, device=q.device).double() * 2 / d)
                           for a, d in enumerate(self.of.sections)], -1)[:, None]
        c, s = torch.cos(angle).to(q.dtype), torch.sin(angle).to(q.dtype)

        def turn(x):
            n = sum(self.of.sections) // 2
            a, b = x[..., :n], x[..., n:2 * n]
            return torch.cat([a * c - b * s, a * s + b * c, x[..., 2 * n:]], -1)
        return turn(q), turn(k)


def test_gradients_of_a_block_against_64_bits(cuda_device):
    """fp32, nothing dropped: every gradient of attention with rotary positions and a gated block.  Sums of up to 200 products of fp32, a softmax and
    two normalisations behind one another: 1e-4 of the largest value is a hundred times what they lose."""
    torch.manual_seed(3)
    block = vit.Block(60, 3, 96, "gated", True).to(cuda_device)
    want = copy.deepcopy(block).double()
    want.rotary = _Turn(block.rotary)
    old = block.fc1.both
    block.fc1 = DropITGatedLinear(60, 64, gamma=0.0, device=cuda_device)
    block.fc1.weight, block.fc1.bias = old.weight, old.bias
    convert_linear_layers(block, 0.0)
    assert isinstance(block.fc2, DropITLinear) and isinstance(block.fc1, DropITGatedLinear)
    x = torch.randn(2, 10, 60, device=cuda_device, requires_grad=True)
    grid = torch.stack([torch.arange(10) // 4, torch.arange(10) % 4], 1).int().to(cuda_device)
    y = x.detach().double().requires_grad_(True)
    g = torch.randn(2, 10, 60, device=cuda_device)
    out, ref = block(x, grid), want(y, grid)
    out.backward(g)
    ref.backward(g.double())
    theirs = {n.replace("fc1.both.", "fc1."): p.grad for n, p in want.named_parameters()}
    pairs = [(out, ref), (x.grad, y.grad)] + [(p.grad, theirs[n]) for n, p in block.named_parameters()]
    assert len(pairs) == 2 + 12
    for a, b in pairs:
        assert float((a.double() - b).abs().max()) <= 1e-4 * float(b.abs().max())


@pytest.mark.parametrize("optimizer", ["adamw", "adamw8"])
@pytest.mark.parametrize("gamma", [None, 0.9])
def test_training_steps(cuda_device, gamma, optimizer):
    model = vit.build_vit_b16(gamma, device=cuda_device, depth=2, ffn="gated", positions="rotary")
    layers = [type(m) for m in model.modules()]
    assert layers.count(DropITGatedLinear) == (0 if gamma is None else 2) and layers.count(dropit.DropITRotary) == 2
    assert model.blocks[0].fc2.in_features == 2048
    before = [p.detach().clone() for p in model.parameters()]
    sps, peak, loss = vit.train_steps(model, 4, 2, warmup=1, optimizer=optimizer)
    dropit.check_device_status(cuda_device)
    assert sps > 0 and loss == loss
    assert all(bool(torch.isfinite(p).all()) for p in model.parameters())
    moved = [not torch.equal(p, b) for p, b in zip(model.parameters(), before)]
    assert sum(moved) >= len(moved) - 2


def test_the_dropping_saves_memory_in_gated_blocks(cuda_device):
    peaks = []
    for gamma in (None, 0.9):
        model = vit.build_vit_b16(gamma, device=cuda_device, depth=2, ffn="gated", positions="rotary")
        peaks.append(vit.train_steps(model, 32, 1, warmup=1)[1])
        del model
    assert peaks[1] < peaks[0]


def test_a_step_captured_whole(cuda_device):
    """Forward, backward and the optimizer's step in one graph: replays go on where the eager steps stopped, number of the step included."""
    def make():
        torch.manual_seed(0)
        model = vit.ViT(image=32, patch=8, dim=64, depth=1, heads=2, mlp=96, classes=10, ffn="gated", positions="rotary").to(cuda_device)
        old = model.blocks[0].fc1.both
        model.blocks[0].fc1 = DropITGatedLinear(64, 64, gamma=0.5, device=cuda_device)
        model.blocks[0].fc1.weight, model.blocks[0].fc1.bias = old.weight, old.bias
        return model, dropit.DropITAdamW(model.parameters(), lr=1e-3, state_bits=8)
    g = torch.Generator(device=cuda_device).manual_seed(1)
    images = [torch.randn(4, 3, 32, 32, generator=g, device=cuda_device) for _ in range(4)]
    label = torch.tensor([1, 2, 3, 4], device=cuda_device)

    def step(model, opt, image):
        opt.zero_grad(set_to_none=False)
        F.cross_entropy(model(image), label).backward()
        opt.step()
    eager, eager_opt = make()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):          # as the capture will run, so that the sums of its library kernels are the same
        for i in (0, 1, 2, 3):
            step(eager, eager_opt, images[i])
    torch.cuda.current_stream().wait_stream(stream)
    model, opt = make()
    static = images[0].clone()
    with torch.cuda.stream(stream):
        step(model, opt, static)
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(model, opt, static)
    for i in (1, 2, 3):
        static.copy_(images[i])
        graph.replay()
    torch.cuda.synchronize()
    dropit.check_device_status(cuda_device)
    assert all(int(opt.state[p]["step"]) == 4 for p in model.parameters())
    for p, q in zip(eager.parameters(), model.parameters()):
        # library kernels may add in another order under capture; four steps of 1e-3 move a parameter by 4e-3 at most
        assert float((p - q).abs().max()) <= 1e-3


def test_the_command(cuda_device, monkeypatch, capsys):
    monkeypatch.setattr(sys, "argv", ["vit", "--batch", "2", "--steps", "1", "--depth", "1", "--ffn", "gated", "--positions", "rotary", "--optimizer", "adamw8"])
    vit.main()
    out = json.loads(capsys.readouterr().out)
    assert out["config"]["ffn"] == "gated" and out["config"]["positions"] == "rotary" and out["config"]["optimizer"] == "adamw8"
    assert out["dropit"]["samples_per_s"] > 0


def test_what_the_options_refuse(cuda_device):
    with pytest.raises(ValueError):
        vit.ViT(ffn="moe")
    with pytest.raises(ValueError):
        vit.ViT(positions="none")
    with pytest.raises(ValueError):
        vit.make_optimizer(nn.Linear(2, 2), "lion", 1e-3)


def test_converting_the_stock_gated_block_keeps_its_gate(cuda_device):
    torch.manual_seed(3)
    block = vit.Block(64, 2, 96, "gated").to(cuda_device)
    x = torch.randn(2, 5, 64, device=cuda_device)
    want = block(x)
    convert_linear_layers(block, 0.0)
    got = block(x)
    assert float((got - want).detach().abs().max()) <= 1e-4 * float(want.detach().abs().max())


def test_layers_of_two_streams_at_once(cuda_device):
    """Two streams run the layer, the rotation and a step of their own at the same time: each gets what it gets alone."""
    def work(seed):
        g = torch.Generator(device=cuda_device).manual_seed(seed)
        torch.manual_seed(seed)
        layer = DropITGatedLinear(256, 384, gamma=0.8, device=cuda_device, dtype=torch.bfloat16).train()
        opt = dropit.DropITAdamW(layer.parameters(), lr=1e-2, state_bits=8, dither=True)
        rot = dropit.DropITRotary(64, (32, 32))
        x = torch.randn(2100, 256, generator=g, device=cuda_device).bfloat16().requires_grad_(True)
        dh = torch.randn(2100, 384, generator=g, device=cuda_device).bfloat16()
        at = torch.randint(0, 99, (2100, 2), generator=g, device=cuda_device)

        def once():
            x.grad = None
            opt.zero_grad()
            h = layer(x)
            h.backward(dh)
            opt.step()
            return [h.detach(), x.grad, rot(h.detach().view(2100, 6, 64), None, at)[0]] + [p.detach().clone() for p in layer.parameters()]
        return once
    alone = []
    for seed in (1, 2):
        once = work(seed)
        alone.append([once() for _ in range(4)])
    streams = [torch.cuda.Stream() for _ in range(2)]
    together = [work(1), work(2)]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(4):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(together[i]())
    torch.cuda.synchronize()
    dropit.check_device_status(cuda_device)
    for a, b in zip(alone, got):
        for one, other in zip(a, b):
            assert all(torch.equal(p, q) for p, q in zip(one, other))
