"""A layer of routed experts: the calls of ``experts`` put together.

    out = residual + sum_j w_j (W2_e act(W1_e x + b1_e) + b2_e),   e = the token's j-th expert

with the experts and their weights from a linear router.  ``forward`` keeps what
``backward`` needs when asked to; ``backward`` returns every gradient.  Every product,
routing, ordering and blending step is one library call; torch holds the tensors.
Every result between the calls is rounded to the layer's type, the router's logits among
them; gradients are computed by ``backward``, not by autograd.  After a step
``ntc.ntc_linear_status`` says whether a kernel gave up a wait, which makes results invalid.
"""
from __future__ import annotations

import torch

from . import ntc


class RoutedExperts:
    """Parameters in `dtype` (biases fp32) on the current CUDA device, drawn from `generator`."""

    NAMES = ("router", "router_bias", "w1", "b1", "w2", "b2")

    def __init__(self, d_in: int, hidden: int, d_out: int, num_experts: int, top_k: int, *, activation: str = "silu",
                 score: str = "softmax", dtype=torch.bfloat16, generator=None):
        dev = torch.device("cuda", torch.cuda.current_device())

        def normal(*shape, std):
            return torch.randn(*shape, generator=generator, device=dev) * std

        self.num_experts, self.top_k, self.activation, self.score = num_experts, top_k, activation, score
        self.router = normal(num_experts, d_in, std=d_in ** -0.5).to(dtype)
        self.router_bias = torch.zeros(num_experts, device=dev)
        self.w1 = normal(num_experts, hidden, d_in, std=d_in ** -0.5).to(dtype)
        self.b1 = torch.zeros(num_experts, hidden, device=dev)
        self.w2 = normal(num_experts, d_out, hidden, std=hidden ** -0.5).to(dtype)
        self.b2 = torch.zeros(num_experts, d_out, device=dev)
        # steers the choice towards experts that too few tokens take; no gradient (see balance)
        self.choice_bias = torch.zeros(num_experts, device=dev)

    def forward(self, x, residual=None, keep: bool = False):
        """The layer's rows for x [tokens, d_in]; with keep, also what backward takes."""
        logits = ntc.linear(x, self.router, self.router_bias)
        ids, weights = ntc.route(logits, self.top_k, bias=self.choice_bias, score=self.score)
        rows, place, offsets = ntc.expert_order(ids, self.num_experts)
        h = ntc.linear(x, self.w1, self.b1, rows=rows, offsets=offsets, activation=self.activation, save=keep)
        h, z = h if keep else (h, None)
        y = ntc.linear(h, self.w2, self.b2, offsets=offsets)
        out = ntc.combine(y, place, weights, offsets, residual=residual)
        return (out, (x, logits, ids, weights, rows, place, offsets, h, z, y)) if keep else out

    def backward(self, dout, kept):
        """The gradients of the parameters (a dict by NAMES) and of x; the residual's is dout itself."""
        x, logits, ids, weights, rows, place, offsets, h, z, y = kept
        dy, dweights = ntc.combine_backward(dout, y, place, weights, offsets)
        dh, dw2, db2 = ntc.linear_backward(dy, h, self.w2, offsets=offsets)
        dx, dw1, db1 = ntc.linear_backward(dh, x, self.w1, z=z, rows=rows, offsets=offsets, activation=self.activation)
        dlogits = ntc.route_backward(logits, ids, dweights, score=self.score)
        dx_router, drouter, dbias = ntc.linear_backward(dlogits, x, self.router)
        # a token's gradient: the sum of its entries', and the router's
        dx = ntc.combine(dx, place, None, offsets, residual=dx_router)
        return dict(router=drouter, router_bias=dbias, w1=dw1, b1=db1, w2=dw2, b2=db2), dx

    def balance(self, offsets, rate: float = 1e-3):
        """Moves the choice's bias against the load of the last batch (offsets of its order)."""
        load = (offsets[1:] - offsets[:-1]).float()
        self.choice_bias += rate * torch.sign(load.mean() - load)
