"""AdamW as a ``torch.optim.Optimizer`` whose whole step is one launch of the library for up to 480 tensors (``binding.pacer_adamw``), for
training programs.

Parameters are f32 or bf16, contiguous, on GPUs; gradients f32, bf16 or f16.  A bf16 parameter has an f32 master among the states,
unless ``master=False``.  States are f32, or with ``states="8bit"`` 8-bit codes with a scale for 256 elements (tensors of fewer
than 4096 elements keep f32 states).  With ``seed`` 8-bit states and bf16 parameters without a master are rounded at random.
"""
from __future__ import annotations

from typing import Optional

import torch

from . import binding

SMALL = 4096                       # elements below which a tensor's states stay in 32 bits


class AdamW(torch.optim.Optimizer):
    """max_norm: the gradients of all groups are scaled to at most this global norm (0: not at all); a step whose norm is not finite changes
    nothing but the count.  capturable: the count is kept on the device and lr may be an f32 scalar there, so that ``step`` can be
    captured into a CUDA graph (gradients must then stay where they are: zero them, don't drop them)."""

    def __init__(self, params, lr=1e-3, betas=(0.9, 0.999), eps: float = 1e-8, weight_decay: float = 1e-2, *, states: str = "f32",
                 master: bool = True, seed: Optional[int] = None, max_norm: float = 0.0, capturable: bool = False):
        if states not in ("f32", "8bit"):
            raise ValueError("states: 'f32' or '8bit'")
        if not all(0.0 <= b < 1.0 for b in betas) or eps < 0.0 or max_norm < 0.0 or (not torch.is_tensor(lr) and lr < 0.0):
            raise ValueError("betas in [0, 1); eps, lr and max_norm at least 0")
        if torch.is_tensor(lr) and not capturable:
            raise ValueError("lr on the device: only with capturable")
        super().__init__(params, dict(lr=lr, betas=tuple(betas), eps=eps, weight_decay=weight_decay))
        self.states, self.master, self.seed, self.max_norm, self.capturable = states, master, seed, max_norm, capturable
        for group in self.param_groups:
            for p in group["params"]:
                if not (p.is_cuda and p.dtype in (torch.float32, torch.bfloat16) and p.is_contiguous()):
                    raise ValueError("params: f32 or bf16, contiguous, on the GPU")
        self._tables = {}

    def _state_of(self, p):
        s = self.state[p]
        if not s:
            small = self.states == "f32" or p.numel() < SMALL
            s["step"] = torch.zeros((), dtype=torch.int32, device=p.device) if self.capturable else 0
            for name in ("exp_avg", "exp_avg_sq"):
                s[name] = torch.zeros(p.shape, dtype=torch.float32 if small else torch.uint8, device=p.device)
            if not small:
                s["scales"] = torch.zeros(-(-p.numel() // 256), 2, device=p.device)
            if p.dtype == torch.bfloat16 and self.master:
                s["master"] = p.detach().float()
        return s

    def load_state_dict(self, state_dict):
        """States keep their types (torch would take them to their parameter's)."""
        held = [k for k in state_dict["state"]]
        super().load_state_dict(state_dict)
        params = [p for g in self.param_groups for p in g["params"]]
        numbers = [n for g in state_dict["param_groups"] for n in g["params"]]
        place = dict(zip(numbers, params))
        for k in held:
            p = place[k]
            for name, x in state_dict["state"][k].items():
                if name == "step":
                    x = int(x)
                    self.state[p][name] = torch.full((), x, dtype=torch.int32, device=p.device) if self.capturable else x
                else:
                    self.state[p][name] = x.detach().to(p.device, copy=True)
        self._tables = {}

    def _buckets(self):
        """Lists of parameters that one call takes: those of a group, device, count and kind of state."""
        buckets = {}
        for gi, group in enumerate(self.param_groups):
            for p in group["params"]:
                if p.grad is None:
                    continue
                if p.grad.is_sparse:
                    raise RuntimeError("AdamW: no sparse gradients")
                s = self._state_of(p)
                buckets.setdefault((gi, p.device, None if self.capturable else s["step"], "scales" in s), []).append(p)
        return buckets

    @torch.no_grad()
    def step(self, closure=None):
        loss = None
        if closure is not None:
            with torch.enable_grad():
                loss = closure()
        buckets = self._buckets()
        grads = {p: p.grad.contiguous() for ps in buckets.values() for p in ps}
        norm = None
        if self.max_norm > 0 and grads:
            if len({p.device for p in grads}) > 1:
                raise RuntimeError("AdamW: max_norm with parameters on one GPU only")
            norm = binding.pacer_grad_norm(list(grads.values()))
        for (gi, device, count, coded), ps in buckets.items():
            group = self.param_groups[gi]
            key = (gi, device, coded, *map(id, ps))
            if key not in self._tables:
                self._tables = {k: t for k, t in self._tables.items() if k[:3] != key[:3]}
                st = [self.state[p] for p in ps]
                copies = [p if "master" in s else None for p, s in zip(ps, st)]
                self._tables[key] = binding.AdamwTensors([s.get("master", p) for p, s in zip(ps, st)], [s["exp_avg"] for s in st],
                                                         [s["exp_avg_sq"] for s in st], [s["scales"] for s in st] if coded else None,
                                                         copies if any(c is not None for c in copies) else None)
            for p in ps:
                self.state[p]["step"] += 1
            # (a capturable optimiser's parameters may have different counts: one call for each count would need to read them back)
            step = self.state[ps[0]]["step"] if self.capturable else count + 1
            binding.pacer_adamw(self._tables[key], [grads[p] for p in ps], step, group["lr"], group["betas"], group["eps"], group["weight_decay"],
                                self.seed, norm, self.max_norm)
        return loss
