"""AdamW as a ``torch.optim.Optimizer`` whose whole step is one launch of the library for up to 480 tensors (``binding.pacer_adamw``), for
training programs.

Parameters are f32 or bf16, contiguous, on GPUs; gradients f32, bf16 or f16.  A bf16 parameter has an f32 master among the states,
unless ``master=False``; the parameter is that master rounded, so that a program which writes to it between steps has to write
``state[p]["master"]`` too, or drop the state.  States are f32, or with ``states="8bit"`` 8-bit codes with a scale for 256 elements
(tensors of fewer than 4096 elements keep f32 states).  8-bit states and bf16 parameters without a master are rounded at random
with ``seed``; with ``seed=None`` to nearest, which leaves second moments too large (20 % after 2000 steps) and loses updates below half
a step of a parameter.
"""
from __future__ import annotations

import operator
from typing import Optional

import torch

from . import binding

SMALL = 4096                       # elements below which a tensor's states stay in 32 bits


class AdamW(torch.optim.Optimizer):
    """max_norm: the gradients of all groups are scaled to at most this global norm (0: not at all); a step whose norm is not finite changes
    nothing but the count.  capturable: the count is kept on the device and lr may be an f32 scalar there, so that ``step`` can be
    captured into a CUDA graph, each parameter's first step excepted, which makes its state (gradients must then stay where they are: zero
    them, don't drop them)."""

    def __init__(self, params, lr=1e-3, betas=(0.9, 0.999), eps: float = 1e-8, weight_decay: float = 1e-2, *, states: str = "f32",
                 master: bool = True, seed: Optional[int] = 0, max_norm: float = 0.0, capturable: bool = False):
        if states not in ("f32", "8bit"):
            raise ValueError("states: 'f32' or '8bit'")
        if not all(0.0 <= b < 1.0 for b in betas) or eps < 0.0 or max_norm < 0.0 or (not torch.is_tensor(lr) and lr < 0.0):
            raise ValueError("betas in [0, 1); eps, lr and max_norm at least 0")
        if torch.is_tensor(lr) and not capturable:
            raise ValueError("lr on the device: only with capturable")
        self.states, self.master, self.seed, self.max_norm, self.capturable = states, master, seed, max_norm, capturable
        self._tables = {}
        super().__init__(params, dict(lr=lr, betas=tuple(betas), eps=eps, weight_decay=weight_decay))

    def add_param_group(self, param_group):
        super().add_param_group(param_group)
        for p in self.param_groups[-1]["params"]:
            if not (p.is_cuda and p.dtype in (torch.float32, torch.bfloat16) and p.is_contiguous()):
                self.param_groups.pop()
                raise ValueError("params: f32 or bf16, contiguous, on the GPU")

    def __getstate__(self):
        own = ("states", "master", "seed", "max_norm", "capturable")
        return dict(super().__getstate__(), **{k: getattr(self, k) for k in own})

    def __setstate__(self, state):
        super().__setstate__(state)
        self._tables = {}

    def _state_of(self, p, fresh):
        """fresh: the count that parameters met for the first time in this step share, by device."""
        s = self.state[p]
        if not s:
            if torch.cuda.is_current_stream_capturing():                # (a replay would set the moments to 0 again)
                raise RuntimeError("AdamW: a captured step has to come after a first one of each of its parameters")
            small = self.states == "f32" or p.numel() < SMALL
            s["step"] = 0
            if self.capturable:
                if p.device not in fresh:
                    fresh[p.device] = torch.zeros((), dtype=torch.int32, device=p.device)
                s["step"] = fresh[p.device]
            for name in ("exp_avg", "exp_avg_sq"):
                s[name] = torch.zeros(p.shape, dtype=torch.float32 if small else torch.uint8, device=p.device)
            if not small:
                s["scales"] = torch.zeros(-(-p.numel() // 256), 2, device=p.device)
            if p.dtype == torch.bfloat16 and self.master:
                s["master"] = p.detach().float()
        return s

    def load_state_dict(self, state_dict):
        """States keep their types (torch would take them to their parameter's); a bf16 parameter whose state has no master gets one of its value
        now.  Registered hooks run as torch's do: ours see what the ones before loading return, and are done before those after it."""
        seen = []
        last = self.register_load_state_dict_pre_hook(lambda _, d: seen.append(d))
        first = self.register_load_state_dict_post_hook(lambda _: self._take(seen[-1]), prepend=True)
        try:
            super().load_state_dict(state_dict)
        finally:
            last.remove()
            first.remove()

    def _take(self, state_dict):
        params = [p for g in self.param_groups for p in g["params"]]
        place = dict(zip([n for g in state_dict["param_groups"] for n in g["params"]], params))
        counts = {}
        for k, held in state_dict["state"].items():
            p = place[k]
            for name, x in held.items():
                if name != "step":
                    self.state[p][name] = x.detach().to(p.device, copy=True)
                elif self.capturable:                                   # (equal counts are one tensor)
                    key = (p.device, int(x))
                    if key not in counts:
                        counts[key] = torch.full((), int(x), dtype=torch.int32, device=p.device)
                    self.state[p][name] = counts[key]
                else:
                    self.state[p][name] = int(x)
            if held and p.dtype == torch.bfloat16 and self.master and "master" not in held:
                self.state[p]["master"] = p.detach().float()
        self._tables = {}

    def _buckets(self):
        """Lists of parameters that one call takes: those of a group, device, count and kind of state."""
        buckets, fresh = {}, {}
        for gi, group in enumerate(self.param_groups):
            for p in group["params"]:
                if p.grad is None:
                    continue
                if p.grad.is_sparse:
                    raise RuntimeError("AdamW: no sparse gradients")
                if not p.is_contiguous():                               # (a parameter may get other strides where it lies)
                    raise RuntimeError("AdamW: params contiguous, as they were given")
                s = self._state_of(p, fresh)
                buckets.setdefault((gi, p.device, id(s["step"]) if self.capturable else s["step"], "scales" in s), []).append(p)
        if self.capturable:
            # a count on the device is shared by the parameters that have had the same steps: where some of them have none now, the others go on
            # with a copy of it
            now = {p for ps in buckets.values() for p in ps}
            stay = {id(s["step"]) for p, s in self.state.items() if p not in now and s}
            copies = {}
            for p in now:
                t = self.state[p]["step"]
                if id(t) in stay:
                    if torch.cuda.is_current_stream_capturing():
                        raise RuntimeError("AdamW: a captured step has to have the gradients of the steps before it")
                    self.state[p]["step"] = copies.setdefault(id(t), t.clone())
        return buckets

    def _table(self, key, ps, coded):
        """The tensors that a call takes, kept between steps while the state holds these very ones (a program may drop or exchange them)."""
        st = [self.state[p] for p in ps]
        copies = [p if "master" in s else None for p, s in zip(ps, st)]
        now = ([s.get("master", p) for p, s in zip(ps, st)], copies if any(c is not None for c in copies) else None, [s["exp_avg"] for s in st],
               [s["exp_avg_sq"] for s in st], [s["scales"] for s in st] if coded else None)
        kept = self._tables.get(key)
        if kept is None or not all(x is y or (x is not None and y is not None and all(map(operator.is_, x, y))) for x, y in zip(kept.tensors, now)):
            if kept is not None or len(self._tables) >= 64:             # (others may hold on to what was dropped; programs whose parameters take turns)
                self._tables.clear()
            params, copies, exp_avg, exp_avg_sq, scales = now
            kept = self._tables[key] = binding.AdamwTensors(params, exp_avg, exp_avg_sq, scales, copies)
        return kept

    @torch.no_grad()
    def step(self, closure=None):
        loss = None
        if closure is not None:
            with torch.enable_grad():
                loss = closure()
        if not self.capturable and torch.cuda.is_current_stream_capturing():
            raise RuntimeError("AdamW: captured steps need capturable=True (else every replay has the count and rate of now)")
        buckets = self._buckets()
        # (before anything is counted: a state that does not fit is refused)
        tables = [self._table((gi, device, coded, *map(id, ps)), ps, coded) for (gi, device, _, coded), ps in buckets.items()]
        grads = {p: p.grad.contiguous() for ps in buckets.values() for p in ps}
        norm = None
        if self.max_norm > 0 and grads:
            if len({p.device for p in grads}) > 1:
                raise RuntimeError("AdamW: max_norm with parameters on one GPU only")
            norm = binding.pacer_grad_norm(list(grads.values()))
        if self.capturable:
            for t in {id(s["step"]): s["step"] for s in map(self.state.__getitem__, grads)}.values():
                t += 1
        else:
            for p in grads:
                self.state[p]["step"] += 1
        for ((gi, *_), ps), table in zip(buckets.items(), tables):
            group = self.param_groups[gi]
            binding.pacer_adamw(table, [grads[p] for p in ps], self.state[ps[0]]["step"], group["lr"], group["betas"], group["eps"],
                                group["weight_decay"], self.seed, norm, self.max_norm)
        return loss
