"""What a step of a gated, rotary transformer needs next to DropIT's layers, as timed cases.

  gated   DropITGatedLinear       h = gate(x Wg^T + bg) * (x Wu^T + bu), the first half of a gated feed-forward block, with the
                                  layer input cached as D(x): forward and backward, or the forward pass alone (tokens at inference)
  rotary  DropITRotary            rotary positions with several axes on queries and keys: forward and backward, or forward alone
  adamw   DropITAdamW.step        one AdamW step over all tensors of a model, moments in 32 bits or in 8

Sizes: the widths of the ViT-B/16 of this repository and of ViTDet at 1024 x 1024 pixels, with the hidden width of a gated block
of the same cost (two thirds of an ungated one's, 2048 for 768 channels), and what lies around them.  Values: activations after a
normalisation N(0, 1), weights N(0, 1 / fan-in), gradients N(0, 0.02^2); moments as they are in the middle of a training run.

`own` false: the operators in elementary torch operations, in 32 bits.  `own` true: the calls of the package.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

_DTYPE = {"bf16": torch.bfloat16, "f32": torch.float32}


# ---------------------------------------------------------------- cases

def _gated(name, tokens, channels, hidden, gate="silu", gamma=0.9, train=True, bias=True, dtype="bf16"):
    return {"name": name, "op": "gated", "M": tokens, "C": channels, "H": hidden, "gate": gate, "gamma": gamma, "train": train,
            "bias": bias, "dtype": dtype}


def _rotary(name, batch, length, heads, kv_heads, head_dim, sections, grid, interleaved=False, shared=False, train=True,
            dtype="bf16", start=0, theta=100.0):
    """`sections`: channels per axis; `grid`: tokens per axis, the last axis fastest; both as texts "a,b,.." (cases are plain values).
    Tokens in front of the grid (a class token) stand at the origin; `start` shifts the first axis."""
    return {"name": name, "op": "rotary", "B": batch, "L": length, "heads": heads, "kv_heads": kv_heads, "D": head_dim,
            "sections": sections, "grid": grid, "interleaved": interleaved, "shared": shared, "train": train, "dtype": dtype,
            "start": start, "theta": theta}


def _adamw(name, dim, hidden, depth, classes, p="f32", g="f32", bits=32, master=False, dither=False):
    return {"name": name, "op": "adamw", "dim": dim, "hidden": hidden, "depth": depth, "classes": classes, "p": p, "g": g,
            "bits": bits, "master": master, "dither": dither}


def listed():
    return [
        # a single token through the block at inference, where latency is what counts
        _gated("gated_token", 1, 768, 2048, train=False),
        # eight class tokens at inference
        _gated("gated_tokens_8", 8, 768, 2048, train=False),
        # a training step at batch 3 (3 x 197 tokens, an odd number)
        _gated("gated_591", 3 * 197, 768, 2048),
        # full-precision training of a narrow layer whose widths are odd
        _gated("gated_f32_odd", 197, 387, 771, gate="relu", gamma=0.8, dtype="f32"),
        # ViT-B/16 at batch 64, the ordinary call
        _gated("gated_vitb", 64 * 197, 768, 2048),
        # detection at 1024 x 1024 pixels, batch 8, a GELU gate without biases: the largest
        _gated("gated_vitdet", 8 * 4096, 768, 2048, gate="gelu", gamma=0.8, bias=False),
        # decoding: one token for each of 16 sequences far into a video, three axes of one frequency ladder, grouped keys
        _rotary("rotary_token", 16, 1, 16, 4, 128, "48,40,40", "1,1,1", shared=True, train=False, start=1000000, theta=10000.0),
        # ViT-B/16 at batch 64 with a class token: rows and columns, queries and keys where the qkv projection left them
        _rotary("rotary_vitb", 64, 197, 12, 12, 64, "32,32", "14,14"),
        # a clip of 13 frames of 31 x 45 tokens: three axes, pairs of neighbours, a head that is rotated in part
        _rotary("rotary_video", 1, 13 * 31 * 45, 16, 8, 128, "32,32,32", "13,31,45", interleaved=True, theta=10000.0),
        # the classifier and one block alone in full precision: fine-tuning, a few tensors
        _adamw("adamw_tune_f32", 192, 512, 1, 100),
        # all tensors of the ViT-B/16 with gated blocks, everything in 32 bits
        _adamw("adamw_vitb_f32", 768, 2048, 12, 1000),
        # the same with bf16 parameters and gradients, moments in 8 bits and parameters rounded with a dither: the least memory
        _adamw("adamw_vitb_8bit", 768, 2048, 12, 1000, p="bf16", g="bf16", bits=8, dither=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("gated", "gated", "gated", "rotary", "rotary", "adamw", "adamw"))
    if op == "gated":
        gate = rng.choice(("silu", "silu", "gelu", "relu"))
        kind = rng.choice(("train", "train", "train", "tokens", "f32"))
        gamma = round(rng.uniform(0.5, 0.95), 2)
        bias = rng.random() < 0.5
        if kind == "f32":
            case = _gated("", _log_int(rng, 16, 1024), _log_int(rng, 64, 512), _log_int(rng, 64, 1024), gate, gamma, True, bias, "f32")
        else:
            channels = 8 * _log_int(rng, 24, 128)           # 192 .. 1024
            hidden = 8 * (channels // 3)                     # 8/3 of the channels, in eights
            if kind == "tokens":
                case = _gated("", _log_int(rng, 1, 300), channels, hidden, gate, gamma, False, bias)
            else:
                tokens = min(_log_int(rng, 33, 32768), 32768 * 768 * 2048 // (channels * hidden))
                case = _gated("", tokens, channels, hidden, gate, gamma, True, bias)
    elif op == "rotary":
        axes = rng.choice((1, 2, 2, 3))
        head_dim = rng.choice((32, 48, 64, 80, 96, 128))
        unit = rng.choice((4, 8))
        per = head_dim // axes // unit * unit
        sections = [per] * axes
        if rng.random() < 0.5:
            sections[0] = head_dim - per * (axes - 1)
        if rng.random() < 0.4:
            grid, batch, train, start = [1] * axes, _log_int(rng, 1, 256), False, _log_int(rng, 1, 4000000)
        else:
            side = {1: (16, 8192), 2: (6, 96), 3: (4, 26)}[axes]
            grid, train, start = [_log_int(rng, *side) for _ in range(axes)], True, 0
            batch = _log_int(rng, 1, max(1, min(64, 16384 // math.prod(grid))))
        kv_heads = rng.choice((1, 2, 4, 8, 12))
        heads = kv_heads * rng.choice((1, 1, 2)) if train else kv_heads * rng.choice((1, 2, 4))
        length = math.prod(grid) + (1 if train and rng.random() < 0.5 else 0)
        case = _rotary("", batch, length, heads, kv_heads, head_dim, ",".join(map(str, sections)), ",".join(map(str, grid)),
                       rng.random() < 0.5, rng.random() < 0.3, train, rng.choice(("bf16", "bf16", "f32")), start,
                       rng.choice((100.0, 10000.0)))
    else:
        dim = _log_int(rng, 48, 768)
        bits = rng.choice((32, 8))
        p = rng.choice(("f32", "bf16"))
        master = p == "bf16" and rng.random() < 0.5
        case = _adamw("", dim, max(8, 8 * dim // 3), _log_int(rng, 1, 12), rng.choice((10, 100, 1000)), p,
                      p if rng.random() < 0.7 else rng.choice(("f32", "bf16")), bits, master,
                      p == "bf16" and not master and rng.random() < 0.6)
    del case["name"]
    return case


# ---------------------------------------------------------------- inputs

class _Draws:
    def __init__(self, seed):
        self.dev = torch.device("cuda")
        self.gen = torch.Generator(device=self.dev).manual_seed(int(seed))

    def normal(self, shape, std=1.0):
        return torch.randn(shape, generator=self.gen, device=self.dev, dtype=torch.float32).mul_(std)


def prepare(case, seed):
    return {"gated": _prepare_gated, "rotary": _prepare_rotary, "adamw": _prepare_adamw}[case["op"]](case, _Draws(seed))


def run(state):
    return {"gated": _run_gated, "rotary": _run_rotary, "adamw": _run_adamw}[state["case"]["op"]](state)


def exact(case, seed):
    return {"gated": _exact_gated, "rotary": _exact_rotary, "adamw": _exact_adamw}[case["op"]](case, seed)


def work(case):
    return {"gated": _work_gated, "rotary": _work_rotary, "adamw": _work_adamw}[case["op"]](case)


# ---------------------------------------------------------------- the gated linear

def _prepare_gated(case, draws):
    M, C, H, dtype = case["M"], case["C"], case["H"], _DTYPE[case["dtype"]]
    state = {"case": case, "x": draws.normal((M, C)).to(dtype), "w": draws.normal((2 * H, C), C ** -0.5).to(dtype), "b": None}
    if case["bias"]:
        state["b"] = draws.normal((2 * H,), 0.02).to(dtype)
    if case["train"]:
        state["dh"] = draws.normal((M, H), 0.02).to(dtype)
    if own:
        from paper_2202_13808_b200 import DropITGatedLinear
        layer = DropITGatedLinear(C, H, bias=case["bias"], gate=case["gate"], gamma=case["gamma"], device=draws.dev, dtype=dtype)
        with torch.no_grad():
            layer.weight.copy_(state["w"])
            if case["bias"]:
                layer.bias.copy_(state["b"])
        state["layer"] = layer.train(case["train"])
        state["x"].requires_grad_(case["train"])
    return state


def _kept(x, gamma):
    """Min-k: the k entries of the largest magnitude of the whole tensor (k = n - ceil(gamma n - 1e-6)), ties to the lower index."""
    n = x.numel()
    k = n - math.ceil(gamma * n - 1e-6)
    order = torch.sort(x.reshape(-1).abs(), descending=True, stable=True).indices
    keep = torch.zeros(n, dtype=torch.bool, device=x.device)
    keep[order[:k]] = True
    return keep.view_as(x)


def _gate_and_slope(a, gate):
    if gate == "silu":
        s = 1 / (1 + torch.exp(-a))
        return a * s, s * (1 + a * (1 - s))
    if gate == "gelu":
        phi = 0.5 * torch.erfc(-a * 0.5 ** 0.5)
        return a * phi, phi + a * torch.exp(-0.5 * a * a) * (2 * math.pi) ** -0.5
    return torch.where(a > 0, a, torch.zeros_like(a)), (a > 0).to(a.dtype)


def _run_gated(state):
    case = state["case"]
    if own:
        if not case["train"]:
            with torch.no_grad():
                return {"h": state["layer"](state["x"])}
        layer, x = state["layer"], state["x"]
        h = layer(x)
        leaves = (x, layer.weight) + ((layer.bias,) if case["bias"] else ())
        grads = torch.autograd.grad(h, leaves, state["dh"])
        return {"h": h.detach(), **dict(zip(("dx", "dw", "db"), grads))}
    dtype, H = state["x"].dtype, case["H"]
    x, w = state["x"].float(), state["w"].float()
    both = x @ w.t()
    if case["bias"]:
        both = both + state["b"].float()
    a, u = both[:, :H], both[:, H:]
    act, slope = _gate_and_slope(a, case["gate"])
    out = {"h": (act * u).to(dtype)}
    if case["train"]:
        dh = state["dh"].float()
        dboth = torch.cat([dh * u * slope, dh * act], 1)
        out["dx"] = (dboth @ w).to(dtype)
        out["dw"] = (dboth.t() @ (x * _kept(state["x"], case["gamma"]))).to(dtype)
        if case["bias"]:
            out["db"] = dboth.sum(0).to(dtype)
    return out


def _exact_gated(case, seed):
    state = _prepare_gated(case, _Draws(seed))
    x, w, H = state["x"].detach().double(), state["w"].double(), case["H"]
    a, u = x @ w[:H].t(), x @ w[H:].t()
    if case["bias"]:
        a, u = a + state["b"][:H].double(), u + state["b"][H:].double()
    if case["gate"] == "silu":
        act = a * torch.sigmoid(a)
        slope = torch.sigmoid(a) + act * torch.sigmoid(-a)
    elif case["gate"] == "gelu":
        cdf = torch.special.ndtr(a)
        act, slope = a * cdf, cdf + a * torch.exp(-a.square() / 2) / math.sqrt(2 * math.pi)
    else:
        act, slope = a.clamp_min(0), torch.heaviside(a, torch.zeros_like(a))
    out = {"h": act * u}
    if case["train"]:
        dh = state["dh"].double()
        da, du = dh * u * slope, dh * act
        # the threshold is the k-th magnitude; of the entries that share it the first ones stay
        size = x.abs().flatten()
        k = size.numel() - math.ceil(case["gamma"] * size.numel() - 1e-6)
        if k:
            least = size.sort(descending=True).values[k - 1]
            tied = size == least
            keep = (size > least) | (tied & (tied.long().cumsum(0) <= k - (size > least).sum()))
        else:
            keep = torch.zeros_like(size, dtype=torch.bool)
        kept = torch.where(keep, x.flatten(), torch.zeros_like(size)).view_as(x)
        out["dx"] = da @ w[:H] + du @ w[H:]
        out["dw"] = torch.cat([da.t() @ kept, du.t() @ kept])
        if case["bias"]:
            out["db"] = torch.cat([da.sum(0), du.sum(0)])
    return out


def _work_gated(case):
    """x, W, b (and dh) read once, h (and dx, dW, db) written once; the product and, in training, its two gradients."""
    M, C, H = case["M"], case["C"], case["H"]
    es = _DTYPE[case["dtype"]].itemsize
    values = M * C + 2 * H * C + M * H + (2 * H if case["bias"] else 0)
    return {"bytes": es * values * (2 if case["train"] else 1), "flops": 2 * M * C * 2 * H * (3 if case["train"] else 1)}


# ---------------------------------------------------------------- rotary positions with several axes

def _ints(text):
    return [int(v) for v in text.split(",")]


def _prepare_rotary(case, draws):
    B, L, D, dtype = case["B"], case["L"], case["D"], _DTYPE[case["dtype"]]
    heads, kv = case["heads"], case["kv_heads"]
    # queries, keys and values side by side, as one projection writes them
    qkv = draws.normal((B, L, (heads + 2 * kv) * D)).to(dtype)
    q = qkv[..., :heads * D].unflatten(-1, (heads, D))
    k = qkv[..., heads * D:(heads + kv) * D].unflatten(-1, (kv, D))
    grid = _ints(case["grid"])
    axes = [torch.arange(g, dtype=torch.int32, device=draws.dev) for g in grid]
    axes[0] = axes[0] + case["start"]
    positions = torch.stack(torch.meshgrid(*axes, indexing="ij"), -1).reshape(-1, len(grid))
    extra = L - positions.shape[0]
    positions = torch.cat([positions.new_zeros(extra, len(grid)), positions]).contiguous()
    if case["start"]:       # every sequence at a place of its own
        shift = torch.randint(0, 1000, (B, 1, len(grid)), generator=draws.gen, device=draws.dev, dtype=torch.int32)
        positions = (positions + shift).contiguous()
    state = {"case": case, "q": q, "k": k, "positions": positions}
    if case["train"]:
        state["dq"], state["dk"] = draws.normal((B, L, heads, D), 0.02).to(dtype), draws.normal((B, L, kv, D), 0.02).to(dtype)
    if own:
        from paper_2202_13808_b200 import DropITRotary
        state["rotary"] = DropITRotary(D, _ints(case["sections"]), theta=case["theta"], interleaved=case["interleaved"],
                                       shared=case["shared"])
        if case["train"]:
            state["q"], state["k"] = q.detach().requires_grad_(True), k.detach().requires_grad_(True)
    return state


def _angles(case, positions):
    """Angle of every pair, in 64 bits: position on the pair's axis times theta^(-2 i / d), i counted within the axis with d its
    channels, or over all rotated channels where the axes share one ladder."""
    sections = _ints(case["sections"])
    axis = [a for a, d in enumerate(sections) for _ in range(d // 2)]
    if case["shared"]:
        power = [2 * i / sum(sections) for i in range(len(axis))]
    else:
        power = [2 * i / d for d in sections for i in range(d // 2)]
    speed = torch.tensor([case["theta"] ** -e for e in power], dtype=torch.float64, device=positions.device)
    return positions.double()[..., axis] * speed


def _turn(x, cos, sin, interleaved):
    """Pairs (2 j, 2 j + 1), or (j, j + half of the rotated channels); what lies behind stays as it is."""
    rotated = 2 * cos.shape[-1]
    if interleaved:
        first, second = x[..., 0:rotated:2], x[..., 1:rotated:2]
        turned = torch.stack([first * cos - second * sin, first * sin + second * cos], -1).flatten(-2)
    else:
        first, second = x[..., :rotated // 2], x[..., rotated // 2:rotated]
        turned = torch.cat([first * cos - second * sin, first * sin + second * cos], -1)
    return torch.cat([turned, x[..., rotated:]], -1)


def _run_rotary(state):
    case = state["case"]
    if own:
        q, k = state["rotary"](state["q"], state["k"], state["positions"])
        if not case["train"]:
            return {"q": q, "k": k}
        dq, dk = torch.autograd.grad((q, k), (state["q"], state["k"]), (state["dq"], state["dk"]))
        return {"q": q.detach(), "k": k.detach(), "dq": dq, "dk": dk}
    dtype = state["q"].dtype
    angle = _angles(case, state["positions"]).unsqueeze(-2)
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    out = {n: _turn(state[n].float(), cos, sin, case["interleaved"]).to(dtype) for n in ("q", "k")}
    if case["train"]:
        out.update({n: _turn(state[n].float(), cos, -sin, case["interleaved"]).to(dtype) for n in ("dq", "dk")})
    return out


def _exact_rotary(case, seed):
    state = _prepare_rotary(case, _Draws(seed))
    sections = _ints(case["sections"])
    rotated, out = sum(sections), {}
    for name in ("q", "k", "dq", "dk"):
        if name not in state:
            continue
        x = state[name].detach().double()
        y, at = x.clone(), 0
        for a, d in enumerate(sections):
            p = state["positions"][..., a].double().unsqueeze(-1)           # one value per token, for all heads
            for i in range(d // 2):
                j = at + i
                speed = case["theta"] ** (-2 * j / rotated if case["shared"] else -2 * i / d)
                c, s = torch.cos(p * speed), torch.sin(p * speed)
                if name[0] == "d":
                    s = -s
                one, two = (2 * j, 2 * j + 1) if case["interleaved"] else (j, j + rotated // 2)
                y[..., one] = x[..., one] * c - x[..., two] * s
                y[..., two] = x[..., one] * s + x[..., two] * c
            at += d // 2
        out[name] = y
    return out


def _work_rotary(case):
    """Queries and keys (and their gradients) read and written once, the positions read; six operations a pair."""
    n = case["B"] * case["L"] * (case["heads"] + case["kv_heads"]) * case["D"] * (2 if case["train"] else 1)
    axes = len(_ints(case["grid"]))
    return {"bytes": 2 * n * _DTYPE[case["dtype"]].itemsize + 4 * case["L"] * axes * (case["B"] if case["start"] else 1), "flops": 3 * n}


# ---------------------------------------------------------------- AdamW over all tensors of a model

_LR, _BETAS, _EPS, _DECAY, _STEP, _SEED = 1e-3, (0.9, 0.999), 1e-8, 0.05, 1000, 1234
_BLOCK = 256        # values that share one scale where moments are held in 8 bits


def _shapes(case):
    """The tensors of a ViT with gated blocks, as an optimizer's two groups have them: what is decayed, then what is not."""
    C, H, all_of = case["dim"], case["hidden"], []
    all_of += [(1, 1, C), (1, 197, C), (C, 3, 16, 16), (C,)]
    for _ in range(case["depth"]):
        all_of += [(C,), (C,), (3 * C, C), (3 * C,), (C, C), (C,), (C,), (C,), (2 * H, C), (2 * H,), (C, H), (C,)]
    all_of += [(C,), (C,), (case["classes"], C), (case["classes"],)]
    return [s for s in all_of if len(s) > 1] + [s for s in all_of if len(s) == 1]


def _blocks_of(n):
    return (n + _BLOCK - 1) // _BLOCK


def _e4m3(x, scale):
    """Values over their blocks' scales, to the nearest 8-bit float."""
    inv = torch.where(scale > 0, 1 / scale, torch.zeros_like(scale))
    return (x.view(-1, _BLOCK) * inv[:, None]).clamp(-448, 448).to(torch.float8_e4m3fn).view(-1)


def _prepare_adamw(case, draws):
    shapes = _shapes(case)
    sizes = [math.prod(s) for s in shapes]
    starts, blocks, total = [], [], 0
    for n in sizes:         # every tensor begins on a block of its own
        starts.append(total * _BLOCK)
        blocks.append(total)
        total += _blocks_of(n)
    inside = torch.zeros(total * _BLOCK, dtype=torch.float32, device=draws.dev)
    for a, n in zip(starts, sizes):
        inside[a:a + n] = 1
    p32 = draws.normal((total * _BLOCK,), 0.02) * inside
    state = {"case": case, "shapes": shapes, "sizes": sizes, "starts": starts, "blocks": blocks,
             "p": p32.to(_DTYPE[case["p"]]), "g": (draws.normal((total * _BLOCK,), 0.02) * inside).to(_DTYPE[case["g"]])}
    # the moments of a run under way: the first a tenth of the gradients' size, the second near their square
    m = draws.normal((total * _BLOCK,), 0.005) * inside
    v = (0.02 * (1 + 0.3 * draws.normal((total * _BLOCK,))) * inside).square()
    if case["master"]:
        state["master"] = p32
    if case["bits"] == 8:
        root = v.sqrt()
        state["m_scale"] = m.view(-1, _BLOCK).abs().amax(1) / 448
        state["r_scale"] = root.view(-1, _BLOCK).amax(1) / 448
        state["m"], state["r"] = _e4m3(m, state["m_scale"]), _e4m3(root, state["r_scale"])
    else:
        state["m"], state["v"] = m, v
    state["step"] = _STEP
    if own:
        from paper_2202_13808_b200 import DropITAdamW
        params = [torch.nn.Parameter(state["p"][a:a + n].view(s)) for a, n, s in zip(starts, sizes, shapes)]
        for q, a, n, s in zip(params, starts, sizes, shapes):
            q.grad_dtype = None         # gradients of another type than the parameter's
            q.grad = state["g"][a:a + n].view(s)
        groups = [{"params": [q for q in params if q.dim() > 1], "weight_decay": _DECAY},
                  {"params": [q for q in params if q.dim() == 1], "weight_decay": 0.0}]
        state["opt"] = opt = DropITAdamW(groups, lr=_LR, betas=_BETAS, eps=_EPS, state_bits=case["bits"], master=case["master"],
                                         dither=case["dither"], seed=_SEED)
        # the optimizer's own state takes the run's: what a checkpoint would bring
        for q, a, n, at in zip(params, starts, sizes, blocks):
            s = opt.init_state(q)
            s["step"].fill_(_STEP)
            s["exp_avg"].view(-1).copy_(state["m"][a:a + n])
            last = at + _blocks_of(n)
            if case["bits"] == 8:
                s["exp_avg_root"].view(-1).copy_(state["r"][a:a + n])
                s["exp_avg_scale"].copy_(state["m_scale"][at:last])
                s["exp_avg_root_scale"].copy_(state["r_scale"][at:last])
            else:
                s["exp_avg_sq"].view(-1).copy_(state["v"][a:a + n])
            if case["master"]:
                s["master"].view(-1).copy_(state["master"][a:a + n])
        state["params"] = params
    return state


def _mix(x):
    """A mixing function of 32-bit words (two multiplications, three shifts), in 64-bit integers."""
    x = x ^ (x >> 16)
    x = (x * 0x7FEB352D) & 0xFFFFFFFF
    x = x ^ (x >> 15)
    x = (x * 0x846CA68B) & 0xFFFFFFFF
    return x ^ (x >> 16)


def _words(ordinal, step, n, device):
    """One random word per value, from the seed, the step, the tensor's number and the value's place."""
    key = _mix(_mix(_mix(_SEED) + step & 0xFFFFFFFF) + ordinal & 0xFFFFFFFF)
    return _mix(torch.arange(n, dtype=torch.int64, device=device) ^ key)


def _to_8_bits(x, bits16, floor_at_one):
    """Blocks of 256 under a scale that makes the largest magnitude 448; a value lies between two 8-bit floats (3 bits of mantissa,
    steps of 2^-9 below 2^-6) and goes to the upper one where its place between them plus a 16-bit random fraction reaches one.
    `floor_at_one`: what is not zero gets the smallest code at least."""
    n = x.numel()
    pad = torch.zeros(_blocks_of(n) * _BLOCK, dtype=x.dtype, device=x.device)
    pad[:n] = x
    scale = pad.view(-1, _BLOCK).abs().amax(1) / 448
    scale = torch.where(scale * 448 < 1e-30, torch.zeros_like(scale), scale)
    inv = torch.where(scale > 0, 1 / scale, torch.zeros_like(scale))
    y = (pad.view(-1, _BLOCK) * inv[:, None]).view(-1)[:n]
    size = y.abs()
    exponent = torch.frexp(size).exponent - 1
    step = torch.ldexp(torch.ones_like(size), exponent.clamp_min(-6) - 3)
    down = torch.floor(size / step)
    up = (size / step - down) + bits16.to(size.dtype) / 65536 >= 1
    value = ((down + up.to(size.dtype)) * step).clamp_max(448)
    if floor_at_one:
        value = torch.where((x > 0) & (value == 0) & (y > 0), torch.full_like(value, 2.0 ** -9), value)
    return (torch.sign(y) * value), scale


def _adamw_values(state):
    """One step of every tensor; yields (its number, p before rounding, m, v, random words)."""
    case = state["case"]
    b1, b2 = _BETAS
    step = state["step"] + 1
    for i, (a, n, at) in enumerate(zip(state["starts"], state["sizes"], state["blocks"])):
        p = (state["master"] if case["master"] else state["p"])[a:a + n].float()
        g = state["g"][a:a + n].float()
        m = state["m"][a:a + n].float()
        if case["bits"] == 8:
            last = at + _blocks_of(n)
            m = m * state["m_scale"][at:last].float().repeat_interleave(_BLOCK)[:n]
            v = (state["r"][a:a + n].float() * state["r_scale"][at:last].float().repeat_interleave(_BLOCK)[:n]).square()
        else:
            v = state["v"][a:a + n].float()
        m = b1 * m + (1 - b1) * g
        v = b2 * v + (1 - b2) * g * g
        decay = _DECAY if len(state["shapes"][i]) > 1 else 0.0
        move = (m / (1 - b1 ** step)) / ((v / (1 - b2 ** step)).sqrt() + _EPS)
        p = p * (1 - _LR * decay) - _LR * move
        words = _words(i, step, n, p.device) if case["bits"] == 8 or case["dither"] else None
        yield i, p, m, v, words


def _run_adamw(state):
    case = state["case"]
    if own:
        opt = state["opt"]
        opt.step()
        out = {"p": state["p"]}
        for name, key in (("m", "exp_avg"), ("v", "exp_avg_sq"), ("r", "exp_avg_root"), ("m_scale", "exp_avg_scale"),
                          ("r_scale", "exp_avg_root_scale"), ("master", "master")):
            whole = opt.whole_state(key)
            if whole is not None:
                out[name] = whole
        return out
    for i, p, m, v, words in _adamw_values(state):
        a, n, at = state["starts"][i], state["sizes"][i], state["blocks"][i]
        if case["master"]:
            state["master"][a:a + n] = p
        if case["dither"]:
            bits = p.view(torch.int32).long() + ((words * 0x9E3779B1 & 0xFFFFFFFF) >> 16)
            p = (bits & ~0xFFFF).to(torch.int32).view(torch.float32)
        state["p"][a:a + n] = p
        if case["bits"] == 8:
            last = at + _blocks_of(n)
            for name, x, bits16 in (("m", m, words >> 16), ("r", v.sqrt(), words & 0xFFFF)):
                codes, scale = _to_8_bits(x, bits16, name == "r")
                state[name][a:a + n] = codes.to(torch.float8_e4m3fn)
                state[name + "_scale"][at:last] = scale
        else:
            state["m"][a:a + n], state["v"][a:a + n] = m, v
    state["step"] += 1
    return {k: state[k] for k in ("p", "m", "v", "r", "m_scale", "r_scale", "master") if k in state}


def _exact_words(ordinal, step, n, device):
    """The same words in the wrapping arithmetic of 32-bit integers."""
    def mix(x):
        x = (x ^ x >> np.uint32(16)) * np.uint32(0x7FEB352D)
        x = (x ^ x >> np.uint32(15)) * np.uint32(0x846CA68B)
        return x ^ x >> np.uint32(16)
    with np.errstate(over="ignore"):
        key = mix(np.array([_SEED], dtype=np.uint32))
        for part in (step, ordinal):
            key = mix(key + np.uint32(part))
        words = mix(np.arange(n, dtype=np.uint32) ^ key)
        other = words * np.uint32(0x9E3779B1)
    return [torch.from_numpy(x.astype(np.uint16).view(np.int16)).to(device).int().bitwise_and_(0xFFFF).double() / 65536
            for x in (words >> np.uint32(16), words & np.uint32(0xFFFF), other >> np.uint32(16))]


def _exact_codes(x, fraction, smallest):
    """Blocks under their scales, by the list of all 8-bit floats: the one below, or the next where the place between the two plus the
    random fraction reaches one."""
    n = x.numel()
    values = [m / 512 for m in range(8)] + [(8 + m) / 8 * 2.0 ** e for e in range(-6, 9) for m in range(8)][:-1]
    grid = torch.tensor(values, dtype=torch.float64, device=x.device)
    padded = torch.nn.functional.pad(x, (0, -n % _BLOCK)).view(-1, _BLOCK)
    top = padded.abs().max(1).values
    scale = torch.where(top >= 1e-30, top / 448, torch.zeros_like(top))
    y = torch.where(scale[:, None] > 0, padded / scale[:, None], torch.zeros_like(padded)).view(-1)[:n]
    below = torch.searchsorted(grid, y.abs().contiguous(), right=True) - 1
    below = below.clamp(0, len(values) - 2)
    low, high = grid[below], grid[below + 1]
    code = torch.where((y.abs() - low) / (high - low) + fraction >= 1, high, low)
    if smallest:
        code = torch.where(y != 0, code.clamp_min(values[1]), code)
    return torch.copysign(code, y), scale


def _exact_adamw(case, seed):
    """The step in its published form: decay, exponential averages by interpolation, averages freed of their bias."""
    state = _prepare_adamw(case, _Draws(seed))
    out = {k: state[k].double() for k in ("p", "m", "v", "r", "m_scale", "r_scale", "master") if k in state}
    t = _STEP + 1
    for i, shape in enumerate(state["shapes"]):
        n = math.prod(shape)
        own_part = slice(state["starts"][i], state["starts"][i] + n)
        scales = slice(state["blocks"][i], state["blocks"][i] + -(-n // _BLOCK))
        p, g, m = out["master" if case["master"] else "p"][own_part].clone(), state["g"][own_part].double(), out["m"][own_part]
        if case["bits"] == 8:
            block = torch.arange(n, device=p.device) // _BLOCK
            m, v = m * out["m_scale"][scales][block], (out["r"][own_part] * out["r_scale"][scales][block]) ** 2
        else:
            v = out["v"][own_part]
        if len(shape) > 1:
            p = p - _LR * _DECAY * p
        m = m + (1 - _BETAS[0]) * (g - m)
        v = v + (1 - _BETAS[1]) * (g ** 2 - v)
        p = p - _LR * (m / (1 - _BETAS[0] ** t)) / ((v / (1 - _BETAS[1] ** t)) ** 0.5 + _EPS)
        if case["master"]:
            out["master"][own_part] = p
        if case["bits"] == 8 or case["dither"]:
            for_m, for_r, for_p = _exact_words(i, t, n, p.device)
        if case["dither"]:      # a bf16 has 8 significant bits
            unit = torch.exp2(torch.floor(torch.log2(p.abs().clamp_min(1e-38))) - 7)
            p = torch.copysign(torch.floor(p.abs() / unit + for_p) * unit, p)
        out["p"][own_part] = p
        if case["bits"] == 8:
            out["m"][own_part], out["m_scale"][scales] = _exact_codes(m, for_m, False)
            out["r"][own_part], out["r_scale"][scales] = _exact_codes(v ** 0.5, for_r, True)
        else:
            out["m"][own_part], out["v"][own_part] = m, v
    return out


def _work_adamw(case):
    """Gradients read; parameters (and their 32-bit copies) and moments read and written; fifteen operations a value."""
    n = sum(math.prod(s) for s in _shapes(case))
    p, g = _DTYPE[case["p"]].itemsize, _DTYPE[case["g"]].itemsize
    moments = 2 * (1 + 4 / _BLOCK) if case["bits"] == 8 else 8
    # with a 32-bit copy the parameters themselves are written only
    params = p + 8 if case["master"] else 2 * p
    return {"bytes": int(n * (g + params + 2 * moments)), "flops": 15 * n}
