"""AdamW whose whole step is one kernel launch, with moments in 32 bits or in 8 (`dropit_adamw_step`).

What a layer caches is one part of a training step's memory, the optimizer's state the other: 8 bytes a parameter for two fp32 moments,
2.03 for two in 8 bits.
"""
from __future__ import annotations

import torch
from torch.optim import optimizer as _optimizer

from . import api

_profiler_enabled = torch.autograd._profiler_enabled
BLOCK = 256         # values that share one scale where moments are held in 8 bits; every tensor begins on a block of its own


class DropITAdamW(torch.optim.Optimizer):
    """torch.optim.AdamW's step (decoupled decay, bias correction) for bf16 and fp32 parameters on one CUDA device.

    state_bits: 32 (state: exp_avg, exp_avg_sq) or 8 (exp_avg, exp_avg_root = sqrt(exp_avg_sq), 8-bit floats whose values are code *
        scale with one fp32 scale per 256 values: exp_avg_scale, exp_avg_root_scale).  Codes are rounded with a dither (a random
        fraction from `seed`, the step, the tensor and the place, so that a run can be repeated): to the nearest code an average that
        moves by a thousandth of itself would not move at all.
    master: bf16 parameters have an fp32 copy that is stepped in their place (state: master); fp32 ones need none.  The copy is made when the state is
        laid out: what is written to a parameter later is overwritten from it, and a parameter whose type has changed is refused.
    dither: bf16 parameters are rounded with a dither, which keeps small steps on average without a copy; else to nearest.
    lr may be a CUDA tensor of one fp32 value, which a captured step reads when it replays; other hyperparameters are part of the graph.  step(grad_factor=t): gradients times t, a CUDA
    tensor of one fp32 value (clipping, unscaling).  Parameters without a gradient stay as they are.  An infinite or NaN gradient
    spoils its own value, and in 8 bits the moments of its block of 256.

    The state lies in arenas, one per kind, in the order of the parameters, blocks of 256 values; state[p] holds views of them.  A group that is
    added later moves them, which a captured step forbids."""

    def __init__(self, params, lr=1e-3, betas=(0.9, 0.999), eps: float = 1e-8, weight_decay: float = 1e-2, state_bits: int = 32,
                 master: bool = False, dither: bool = False, seed: int = 0):
        if state_bits not in (8, 32):
            raise ValueError("state_bits must be 8 or 32, got %r" % (state_bits,))
        self.state_bits, self.master, self.dither, self.seed = int(state_bits), bool(master), bool(dither), int(seed) & 0xFFFFFFFF
        self._plan, self._arenas, self._captured = None, {}, False
        super().__init__(params, dict(lr=lr, betas=betas, eps=eps, weight_decay=weight_decay))

    def add_param_group(self, param_group):
        if self._captured:
            raise RuntimeError("a captured step holds the places of the state, which another group would move: add groups, then capture")
        super().add_param_group(param_group)
        try:
            self._check_group(self.param_groups[-1])
        except Exception:
            self.param_groups.pop()
            raise
        self._plan = None       # the arenas grow when they are next needed

    def _check_group(self, group):
        b1, b2 = group["betas"]
        if not (0 <= b1 < 1 and 0 <= b2 < 1):
            raise ValueError("betas must be in [0, 1), got %r" % (group["betas"],))
        if not group["eps"] >= 0 or not group["weight_decay"] >= 0:
            raise ValueError("eps and weight_decay must not be negative")
        lr = group["lr"]
        if not isinstance(lr, torch.Tensor) and not lr >= 0:
            raise ValueError("lr must not be negative, got %r" % (lr,))
        if len({id(p) for p in group["params"]}) != len(group["params"]):
            raise ValueError("a parameter is given twice")
        for p in group["params"]:
            if p.dtype not in (torch.bfloat16, torch.float32):
                raise TypeError("parameters are bf16 or fp32, got %s" % p.dtype)
            if not torch.ops.aten.is_non_overlapping_and_dense(p):
                raise ValueError("a parameter's values must fill its memory without gaps or overlaps")
            if p.numel() >= 2 ** 31:
                raise ValueError("a parameter has 2^31 values or more")

    def __getstate__(self):
        own = ("state_bits", "master", "dither", "seed")
        return {**super().__getstate__(), **{k: getattr(self, k) for k in own}}

    def __setstate__(self, state):
        super().__setstate__(state)
        self._plan, self._arenas = None, {}      # laid out anew, from the state, when they are next needed
        self.__dict__.setdefault("_captured", False)

    # ---- state ----

    def _kinds(self):
        """Arena name -> (type, values per block)."""
        if self.state_bits == 8:
            kinds = {"exp_avg": (torch.float8_e4m3fn, BLOCK), "exp_avg_root": (torch.float8_e4m3fn, BLOCK),
                     "exp_avg_scale": (torch.float32, 1), "exp_avg_root_scale": (torch.float32, 1)}
        else:
            kinds = {"exp_avg": (torch.float32, BLOCK), "exp_avg_sq": (torch.float32, BLOCK)}
        if self.master:
            kinds["master"] = (torch.float32, BLOCK)
        return kinds

    def _all_params(self):
        return [p for g in self.param_groups for p in g["params"]]

    @torch.no_grad()
    def _build(self):
        """Lay out the arenas for the parameters there are; what earlier ones held keeps its values."""
        params = self._all_params()
        if not params:
            raise ValueError("the optimizer has no parameters")
        device = params[0].device
        if any(p.device != device for p in params) or device.type != "cuda":
            raise ValueError("all parameters must be on one CUDA device (there is no CPU path)")
        if self._captured:
            raise RuntimeError("a captured step holds the places of the state, which cannot be laid out again")
        if torch.cuda.is_current_stream_capturing():        # the zeros and copies below would be part of the graph, and every replay begin anew
            raise RuntimeError("the state must be laid out before a step is captured: call init_state()")
        spans = sorted((p.data_ptr(), p.data_ptr() + p.numel() * p.element_size()) for p in params if p.numel())
        if any(a[1] > b[0] for a, b in zip(spans, spans[1:])):
            raise ValueError("two parameters share memory: one step would take it in turns with itself")
        before = {id(p): self.state[p] for p in params if self.state.get(p)}
        first, total = [], 0
        for p in params:
            first.append(total)
            total += (p.numel() + BLOCK - 1) // BLOCK
        kinds = self._kinds()
        arenas = {k: torch.zeros(max(total, 1) * unit, dtype=t, device=device) for k, (t, unit) in kinds.items()}
        steps = torch.zeros(len(params), dtype=torch.int32, device=device)
        for i, p in enumerate(params):
            state = {"step": steps[i]}
            n, blocks = p.numel(), (p.numel() + BLOCK - 1) // BLOCK
            for k, (_, unit) in kinds.items():
                if k == "master" and p.dtype != torch.bfloat16:
                    continue
                if unit == 1:
                    state[k] = arenas[k][first[i]:first[i] + blocks]
                else:
                    state[k] = arenas[k][first[i] * BLOCK:first[i] * BLOCK + n].as_strided(p.shape, p.stride())
            held = before.get(id(p), {})
            for k in state:
                if k in held:
                    state[k].copy_(held[k])
            if "master" in state and "master" not in held:      # new, or fp32 when it was laid out before
                state["master"].copy_(p)
            self.state[p] = state
        self._arenas, self._steps = arenas, steps
        self._ticket = torch.zeros(4, dtype=torch.int32, device=device)
        group_of = [i for i, g in enumerate(self.param_groups) for _ in g["params"]]
        self._plan = api._native().AdamWParams(params, first, group_of)

    def init_state(self, p=None):
        """Lay out the state now; returns state[p].  The first step does it otherwise, and the first one after add_param_group, but not under capture."""
        if self._plan is None or not self.state:
            self._build()
        return None if p is None else self.state[p]

    def whole_state(self, kind: str):
        """The arena of one kind of state (None if this optimizer has none of it): every parameter's values from a block of its own on, in
        the order of the parameters."""
        self.init_state()
        return self._arenas.get(kind)

    @torch.no_grad()
    def load_state_dict(self, state_dict):
        """Takes the hyperparameters and copies the state into this optimizer's arenas, type for type.  State and learning rates that are tensors
        keep their places, so that a captured step goes on from what is loaded.  Parameters that the checkpoint has no state for begin anew; a checkpoint
        that does not fit is refused before anything changes."""
        state_dict, hooks = dict(state_dict), (self._optimizer_load_state_dict_pre_hooks, self._optimizer_load_state_dict_post_hooks)
        for hook in hooks[0].values():
            changed = hook(self, state_dict)
            state_dict = state_dict if changed is None else changed
        self.init_state()
        params, groups, lrs = self._all_params(), state_dict["param_groups"], [g["lr"] for g in self.param_groups]
        if [len(g["params"]) for g in groups] != [len(g["params"]) for g in self.param_groups]:
            raise ValueError("the checkpoint has other groups of parameters")
        given = [state_dict["state"].get(i) for g in groups for i in g["params"]]
        for i, (p, held) in enumerate(zip(params, given)):
            mine = self.state[p]
            if held and set(held) != set(mine):
                raise ValueError("the state has %s, this optimizer %s" % (sorted(held), sorted(mine)))
            for k, v in (held or {}).items():
                if v.shape != mine[k].shape or v.dtype != mine[k].dtype:
                    raise ValueError("%s of parameter %d is %s %s, expected %s %s" % (k, i, v.dtype, tuple(v.shape), mine[k].dtype, tuple(mine[k].shape)))
        if self._captured and any(lr is other and float(g["lr"]) != float(h["lr"]) for g, lr in zip(groups, lrs) for h, other in zip(groups, lrs)
                                  if isinstance(lr, torch.Tensor)):
            raise ValueError("groups whose learning rate a captured step reads from one tensor are to have different ones")
        # nothing has changed up to here
        laid_out = self.state, self._plan, self._arenas
        empty = type(hooks[0])()
        try:            # the base class takes the groups; its hooks see the whole of it, from here
            self._optimizer_load_state_dict_pre_hooks = self._optimizer_load_state_dict_post_hooks = empty
            super().load_state_dict({**state_dict, "state": {}})
        finally:
            self._optimizer_load_state_dict_pre_hooks, self._optimizer_load_state_dict_post_hooks = hooks
            self.state, self._plan, self._arenas = laid_out
        self._keep_lr_tensors(lrs)
        for p, held in zip(params, given):
            for k, v in self.state[p].items():
                if held:
                    v.copy_(held[k])
                elif k == "master":
                    v.copy_(p)
                else:
                    v.zero_()
        for hook in hooks[1].values():
            hook(self)

    def _keep_lr_tensors(self, before):
        """Learning rates that were tensors take the loaded values; groups that shared one and no longer agree get tensors of their own."""
        loaded = [float(g["lr"]) for g in self.param_groups]
        for g, lr, value in zip(self.param_groups, before, loaded):
            if isinstance(lr, torch.Tensor):
                agree = all(v == value for v, other in zip(loaded, before) if other is lr)
                g["lr"] = lr.fill_(value) if agree else torch.full_like(lr, value)

    # ---- the step ----

    def step(self, closure=None, grad_factor=None):
        if self._optimizer_step_pre_hooks or self._optimizer_step_post_hooks or _optimizer._global_optimizer_pre_hooks or \
                _optimizer._global_optimizer_post_hooks or _profiler_enabled():
            return _hooked_step(self, closure, grad_factor)
        return self._step(closure, grad_factor)

    step.hooked = True      # the base class would wrap every call for hooks and a profiler's label: 10 us, twice what a small step takes

    def _step(self, closure=None, grad_factor=None):
        loss = None
        if closure is not None:
            with torch.enable_grad():
                loss = closure()
        if self._plan is None or not self.state:        # emptied by the caller: begins anew
            self._build()
        settings = []
        for g in self.param_groups:
            lr, device_lr = g["lr"], None
            if isinstance(lr, torch.Tensor):
                lr, device_lr = 0.0, self._scalar(lr, "lr")
            settings.append((lr, device_lr, g["weight_decay"], *g["betas"], g["eps"]))
        a = self._arenas
        captured = api._native().adamw_step(
            self._plan, settings, self.state_bits, self.dither, self.seed, a["exp_avg"], a["exp_avg_root" if self.state_bits == 8 else "exp_avg_sq"],
            a.get("exp_avg_scale"), a.get("exp_avg_root_scale"), a.get("master"), self._steps, self._ticket,
            None if grad_factor is None else self._scalar(grad_factor, "grad_factor"))
        if captured:
            self._captured = True
        return loss

    def _scalar(self, t, name):
        if not isinstance(t, torch.Tensor) or t.device != self._steps.device or t.dtype != torch.float32 or t.numel() != 1:
            raise ValueError("%s must be one fp32 value on the parameters' device" % name)
        return t


_hooked_step = torch.optim.Optimizer.profile_hook_step(DropITAdamW._step)
