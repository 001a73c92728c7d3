"""AdamW over the tensors of a model, one library call a step (``ntc.adamw``).

Parameters in 16 bits get fp32 masters, in which the steps add up; the parameter itself
receives the master rounded.  Moments take 8 bytes an element, or 2 (and 8 bytes for
every 256 of a tensor) with ``bits=8``.  Gradients come with the call, as the
``*_backward`` functions return them.

Eight bits are too few for a slow decay: where the gradients of a block of 256 have one size,
the roots of the second moment settle 1.12 times too high with beta2 = 0.999, 1.17 times with
0.995, 1.37 times with 0.99 and 1.66 times with 0.98 (medians after 4,000 steps of normally
distributed gradients, beta1 = 0.9), and the steps are 5, 12, 25 and 36 % too small.
"""
from __future__ import annotations

import warnings

import torch

from . import ntc


class AdamW:
    """`params`: a dict or a list of contiguous CUDA tensors in fp32, fp16 or bf16; updated in place.

    captured=True counts the steps and holds the rate on the device, so that a step captured in a CUDA graph counts on
    with every replay; set_lr then changes the rate between replays."""

    def __init__(self, params, *, lr: float = 1e-3, beta1: float = 0.9, beta2: float = 0.999, eps: float = 1e-8,
                 weight_decay: float = 0.01, bits: int = 32, masters: bool = True, captured: bool = False):
        if bits not in (8, 32):
            raise ValueError(f"bits must be 8 or 32, not {bits!r}")
        if bits == 8 and beta2 < 0.995:
            warnings.warn(f"moments in 8 bits with beta2 = {beta2}: the second moment decays in part only, and steps may be "
                          "a quarter (0.99) or more (below) too small; 0.995 or more is meant for them", stacklevel=2)
        self.names = list(params) if isinstance(params, dict) else None
        self.params = list(params.values()) if isinstance(params, dict) else list(params)
        self.hyper = dict(beta1=beta1, beta2=beta2, eps=eps, weight_decay=weight_decay)
        keep = [masters and p.dtype != torch.float32 for p in self.params]
        self.masters = [p.detach().float() if k else p for p, k in zip(self.params, keep)]
        self.copies = [p if k else None for p, k in zip(self.params, keep)]
        kind = torch.float8_e4m3fn if bits == 8 else torch.float32
        self.m = [torch.zeros(p.shape, dtype=kind, device=p.device) for p in self.params]
        self.v = [torch.zeros(p.shape, dtype=kind, device=p.device) for p in self.params]
        self.scales = [torch.zeros(2, -(-p.numel() // ntc.NTC_ADAMW_BLOCK), device=p.device)
                       for p in self.params] if bits == 8 else None
        self.steps, self.captured = 0, captured
        if captured:
            if not self.params:
                raise ValueError("a captured step needs a parameter")
            dev = self.params[0].device
            self.steps = torch.zeros(1, dtype=torch.int32, device=dev)
            self.lr = torch.empty(1, device=dev)
        self.set_lr(lr)

    def set_lr(self, lr: float):
        """The rate is held in fp32, captured or not, so that both take the same steps."""
        if self.captured:
            self.lr.fill_(lr)
        else:
            self.lr = torch.tensor(lr, dtype=torch.float32).item()

    def step(self, grads, grad_scale=1.0):
        """One step for `grads` (as `params` were given: by name, or in order), times grad_scale (a number, or an fp32
        CUDA tensor of one element)."""
        if self.names is not None:
            grads = [grads[n] for n in self.names]
        steps = self.steps.add_(1) if self.captured else self.steps + 1
        try:
            ntc.adamw(self.masters, grads, self.m, self.v, scales=self.scales, copies=self.copies, step=steps, lr=self.lr,
                      grad_scale=grad_scale, **self.hyper)
        except Exception:
            if self.captured:
                self.steps.sub_(1)  # a step that was refused is none
            raise
        self.steps = steps

    def state(self) -> dict:
        """What a checkpoint holds beside the parameters (references, not copies)."""
        return dict(m=self.m, v=self.v, scales=self.scales, masters=[p for p, c in zip(self.masters, self.copies) if c is not None],
                    steps=int(self.steps))

    def load(self, state: dict):
        """Takes over a state(), or, where it does not fit, nothing of it; the parameters become their masters, rounded."""
        mine = self.state()
        if (mine["scales"] is None) != (state["scales"] is None):
            raise ValueError("the state's moments have another number of bits")
        pairs = []  # all of the state is looked at before any of it is taken
        for k in ("m", "v", "scales", "masters"):
            if mine[k] is None:
                continue
            if len(mine[k]) != len(state[k]):
                raise ValueError(f"the state has {len(state[k])} {k}, not {len(mine[k])}")
            for to, of in zip(mine[k], state[k]):
                if to.shape != of.shape:
                    raise ValueError(f"{k}: shape {tuple(of.shape)}, not {tuple(to.shape)}")
                if (to.dtype == torch.float8_e4m3fn) != (of.dtype == torch.float8_e4m3fn):
                    raise ValueError(f"{k}: {of.dtype}, not {to.dtype}: codes mean nothing without their scales")
                pairs.append((to, of))
        steps = int(state["steps"])
        if steps < 0:
            raise ValueError(f"steps must not be negative: {steps}")
        with torch.no_grad():
            for to, of in pairs:
                to.copy_(of)
            for p, c in zip(self.masters, self.copies):
                if c is not None:
                    c.copy_(p)
        if self.captured:
            self.steps.fill_(steps)
        else:
            self.steps = steps
