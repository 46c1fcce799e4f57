"""Momentum whose steps are orthogonalised (orthogonal.h): the optimiser for the matrices of a policy.

    m <- momentum m + g        u = g + momentum m  (or m)        w <- (1 - lr decay) w - lr sqrt(max(1, rows / cols)) orth(u)

Every direction of the update has about the same size, so that few strong directions of the gradient do not crowd out
the rest.  Vectors (biases, norms, rates) and matrices whose rows are looked up one by one belong to another optimiser.
Matrices of one shape go through the products together.
"""
from __future__ import annotations

import math

import torch

from . import orthogonal


class OrthogonalMomentum(torch.optim.Optimizer):
    """params: float32 CUDA matrices [rows, cols].  A parameter without a gradient is left as it is."""

    def __init__(self, params, lr: float = 0.02, momentum: float = 0.95, nesterov: bool = True, weight_decay: float = 0.0,
                 steps: int = 5):
        if not lr >= 0.0 or not 0.0 <= momentum < 1.0 or not weight_decay >= 0.0:
            raise ValueError("lr and weight_decay must not be negative, momentum must lie in [0, 1)")
        super().__init__(params, dict(lr=lr, momentum=momentum, nesterov=nesterov, weight_decay=weight_decay, steps=steps))
        self._ops = {}

    def __setstate__(self, state):
        super().__setstate__(state)
        self.__dict__.setdefault("_ops", {})       # a copy has handles of its own

    def add_param_group(self, group):
        super().add_param_group(group)
        params = self.param_groups[-1]["params"]
        if len(set(map(id, params))) != len(params):
            self.param_groups.pop()
            raise ValueError("a parameter appears twice")
        for p in params:
            if p.dim() != 2 or p.dtype is not torch.float32:
                self.param_groups.pop()
                raise ValueError("parameters must be float32 matrices, got %s %s" % (p.dtype, tuple(p.shape)))

    def _op(self, p, steps):
        key = (tuple(p.shape), p.device, steps)
        if key not in self._ops:
            self._ops[key] = orthogonal.Orthogonal(p.shape[0], p.shape[1], dtype=torch.float32, steps=steps, device=str(p.device))
        return self._ops[key]

    @torch.no_grad()
    def step(self, closure=None):
        loss = None
        if closure is not None:
            with torch.enable_grad():
                loss = closure()
        for group in self.param_groups:
            alike = {}
            for p in group["params"]:
                if p.grad is not None:
                    alike.setdefault((tuple(p.shape), p.device), []).append(p)
            for params in alike.values():
                rows, cols = params[0].shape
                wanted = torch.empty((len(params), rows, cols), dtype=torch.float32, device=params[0].device)
                for p, u in zip(params, wanted):
                    state = self.state[p]
                    if "momentum" not in state:
                        state["momentum"] = torch.zeros_like(p, memory_format=torch.contiguous_format)
                    m = state["momentum"].mul_(group["momentum"]).add_(p.grad)
                    if group["nesterov"]:
                        torch.add(p.grad, m, alpha=group["momentum"], out=u)
                    else:
                        u.copy_(m)
                updates = self._op(params[0], group["steps"]).update(wanted)
                scale = group["lr"] * math.sqrt(max(1.0, rows / cols))
                for p, o in zip(params, updates):
                    if group["weight_decay"]:
                        p.mul_(1.0 - group["lr"] * group["weight_decay"])
                    p.add_(o, alpha=-scale)
        return loss

    def check(self):
        """Synchronises; raises if a kernel gave up a wait."""
        for op in self._ops.values():
            op.status()
