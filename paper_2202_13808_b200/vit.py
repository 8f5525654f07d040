"""A plain ViT-B/16 (12 blocks, hidden 768, MLP 3072, 12 heads, 1000 classes) on synthetic images, used to
measure a full training step with DropIT on every Linear layer against the same model with stock layers
(Sec. 3.5: fully-connected layers of attention and MLP and the classifier; LayerNorm, GELU and attention
keep their caches; the patch-projection convolution is left dense, App. A.6).

  python -m paper_2202_13808_b200.vit --batch 64 --gamma 0.9 --steps 5

Everything that DropIT does not touch is stock torch (LayerNorm, GELU, scaled-dot-product attention,
cross entropy, SGD).

  --ffn gated --positions rotary --optimizer adamw8

takes the parts of later ViTs instead: gated feed-forward blocks of the same cost (two thirds of the hidden width, SiLU), rotary
positions on rows and columns in the place of learned ones, and AdamW with its moments in 32 bits (adamw) or in 8 (adamw8).
"""
from __future__ import annotations

import argparse
import json

import torch
import torch.nn as nn
import torch.nn.functional as F

from .nn import DropITGatedLinear, DropITGeluLinear, DropITRotary, convert_linear_layers
from .optim import DropITAdamW


class StockGatedLinear(nn.Module):
    """silu(x Wg^T + bg) * (x Wu^T + bu) in stock operations: what DropITGatedLinear is compared with, and takes its parameters from."""

    def __init__(self, in_features: int, hidden_features: int, **kw):
        super().__init__()
        self.both = nn.Linear(in_features, 2 * hidden_features, **kw)

    def forward(self, x):
        a, u = self.both(x).chunk(2, -1)
        return F.silu(a) * u


class Block(nn.Module):
    def __init__(self, dim: int, heads: int, mlp: int, ffn: str = "gelu", rotary: bool = False):
        super().__init__()
        self.heads = heads
        self.norm1 = nn.LayerNorm(dim)
        self.qkv = nn.Linear(dim, 3 * dim)
        self.proj = nn.Linear(dim, dim)
        self.norm2 = nn.LayerNorm(dim)
        self.gated = ffn == "gated"
        if self.gated:
            mlp = 2 * mlp // 3
        self.fc1 = StockGatedLinear(dim, mlp) if self.gated else nn.Linear(dim, mlp)
        self.fc2 = nn.Linear(mlp, dim)
        self.gelu_in_fc2 = False      # True when fc2 is a DropITGeluLinear, which applies the GELU itself
        half = dim // heads // 4 * 2  # rows take one half of a head's channels, columns the other
        self.rotary = DropITRotary(dim // heads, (half, half), theta=100.0) if rotary else None

    def forward(self, x, positions=None):
        B, L, C = x.shape
        qkv = self.qkv(self.norm1(x)).reshape(B, L, 3, self.heads, C // self.heads)
        if self.rotary is None:
            q, k, v = qkv.permute(2, 0, 3, 1, 4)
        else:
            q, k = self.rotary(qkv[:, :, 0], qkv[:, :, 1], positions)
            q, k, v = q.transpose(1, 2), k.transpose(1, 2), qkv[:, :, 2].transpose(1, 2)
        a = F.scaled_dot_product_attention(q, k, v)
        x = x + self.proj(a.transpose(1, 2).reshape(B, L, C))
        h = self.fc1(self.norm2(x))
        return x + (self.fc2(h) if self.gelu_in_fc2 or self.gated else self.fc2(F.gelu(h)))


class ViT(nn.Module):
    def __init__(self, image=224, patch=16, dim=768, depth=12, heads=12, mlp=3072, classes=1000, ffn="gelu", positions="learned"):
        super().__init__()
        if ffn not in ("gelu", "gated") or positions not in ("learned", "rotary"):
            raise ValueError("ffn is 'gelu' or 'gated', positions 'learned' or 'rotary'")
        self.patch_embed = nn.Conv2d(3, dim, patch, stride=patch)
        side = image // patch
        self.cls = nn.Parameter(torch.zeros(1, 1, dim))
        if positions == "learned":
            self.pos = nn.Parameter(torch.randn(1, side * side + 1, dim) * 0.02)
            self.grid = None
        else:           # row and column of every patch, the class token at the origin
            self.pos = None
            at = torch.arange(side, dtype=torch.int32)
            grid = torch.stack(torch.meshgrid(at, at, indexing="ij"), -1).reshape(-1, 2)
            self.register_buffer("grid", torch.cat([grid.new_zeros(1, 2), grid]), persistent=False)
        self.blocks = nn.ModuleList([Block(dim, heads, mlp, ffn, positions == "rotary") for _ in range(depth)])
        self.norm = nn.LayerNorm(dim)
        self.head = nn.Linear(dim, classes)

    def forward(self, img):
        x = self.patch_embed(img).flatten(2).transpose(1, 2)
        x = torch.cat([self.cls.expand(x.shape[0], -1, -1), x], 1)
        if self.pos is not None:
            x = x + self.pos
        for b in self.blocks:
            x = b(x, self.grid)
        return self.head(self.norm(x)[:, 0])


def build_vit_b16(gamma=None, device="cuda", dtype=torch.bfloat16, depth=12, seed=0, fuse_gelu=False, ffn="gelu", positions="learned") -> ViT:
    """Random-initialised ViT-B/16; gamma=None keeps stock layers, otherwise every nn.Linear becomes DropITLinear.
    fuse_gelu: the MLP's GELU and second Linear become one DropITGeluLinear (the GELU kernel takes the selection
    statistics of its output, the compression reads that output once).  ffn="gated": gated blocks, whose two projections become one
    DropITGatedLinear each; positions="rotary": rotary positions on rows and columns."""
    torch.manual_seed(seed)
    model = ViT(depth=depth, ffn=ffn, positions=positions).to(device=device, dtype=dtype)
    if gamma is not None:
        for b in model.blocks:
            if b.gated:
                old = b.fc1.both
                b.fc1 = DropITGatedLinear(old.in_features, old.out_features // 2, gamma=gamma, device=old.weight.device, dtype=old.weight.dtype)
                b.fc1.weight, b.fc1.bias = old.weight, old.bias
        if fuse_gelu and ffn == "gelu":
            for b in model.blocks:
                old = b.fc2
                new = DropITGeluLinear(old.in_features, old.out_features, gamma=gamma, device=old.weight.device,
                                       dtype=old.weight.dtype)
                new.weight, new.bias = old.weight, old.bias
                b.fc2, b.gelu_in_fc2 = new, True
        convert_linear_layers(model, gamma)
    return model.train()


def make_optimizer(model: nn.Module, name: str, lr: float):
    """"sgd" (torch's); "adamw" and "adamw8" (moments in 32 and in 8 bits), where bf16 parameters are rounded with a dither, matrices and filters
    decay and vectors do not."""
    if name == "sgd":
        return torch.optim.SGD(model.parameters(), lr=lr)
    if name not in ("adamw", "adamw8"):
        raise ValueError("optimizer is 'sgd', 'adamw' or 'adamw8'")
    params = list(model.parameters())
    groups = [{"params": [p for p in params if p.dim() > 1], "weight_decay": 0.05}, {"params": [p for p in params if p.dim() <= 1], "weight_decay": 0.0}]
    return DropITAdamW(groups, lr=lr, state_bits=8 if name == "adamw8" else 32, dither=params[0].dtype == torch.bfloat16)


def train_steps(model: nn.Module, batch: int, steps: int, warmup: int = 2, lr: float = 1e-3, seed: int = 0, optimizer: str = "sgd"):
    """Run `steps` steps (SGD, or another of make_optimizer) on synthetic 224x224 images ~N(0,1) with random labels.
    Returns (samples/s, peak bytes allocated during a step beyond the resident state, last loss)."""
    dev = next(model.parameters()).device
    g = torch.Generator(device="cpu").manual_seed(seed)
    img = torch.randn(batch, 3, 224, 224, generator=g).to(dev, dtype=next(model.parameters()).dtype)
    lab = torch.randint(0, 1000, (batch,), generator=g).to(dev)
    opt = make_optimizer(model, optimizer, lr)

    def step():
        opt.zero_grad(set_to_none=True)
        loss = F.cross_entropy(model(img).float(), lab)
        loss.backward()
        opt.step()
        return loss

    for _ in range(warmup):
        step()
    torch.cuda.synchronize(dev)
    base = torch.cuda.memory_allocated(dev)
    torch.cuda.reset_peak_memory_stats(dev)
    e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    e0.record()
    for _ in range(steps):
        loss = step()
    e1.record()
    torch.cuda.synchronize(dev)
    peak = torch.cuda.max_memory_allocated(dev) - base
    return batch * steps / (e0.elapsed_time(e1) / 1e3), peak, float(loss.detach())


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--batch", type=int, default=64)
    ap.add_argument("--gamma", type=float, default=0.9)
    ap.add_argument("--steps", type=int, default=5)
    ap.add_argument("--depth", type=int, default=12)
    ap.add_argument("--ffn", choices=("gelu", "gated"), default="gelu")
    ap.add_argument("--positions", choices=("learned", "rotary"), default="learned")
    ap.add_argument("--optimizer", choices=("sgd", "adamw", "adamw8"), default="sgd")
    args = ap.parse_args()
    out = {}
    for name, gamma in (("dense", None), ("dropit", args.gamma)):
        model = build_vit_b16(gamma, depth=args.depth, ffn=args.ffn, positions=args.positions)
        sps, peak, loss = train_steps(model, args.batch, args.steps, optimizer=args.optimizer)
        out[name] = {"samples_per_s": sps, "peak_step_bytes": peak, "loss": loss}
        del model
        torch.cuda.empty_cache()
    out["config"] = {"model": "ViT-B/16", "batch": args.batch, "gamma": args.gamma, "dtype": "bf16", "depth": args.depth,
                     "ffn": args.ffn, "positions": args.positions, "optimizer": args.optimizer, "data": "synthetic"}
    out["peak_ratio"] = out["dropit"]["peak_step_bytes"] / max(out["dense"]["peak_step_bytes"], 1)
    out["speed_ratio"] = out["dropit"]["samples_per_s"] / out["dense"]["samples_per_s"]
    print(json.dumps(out))


if __name__ == "__main__":
    main()
