"""The routed-expert calls of libntc on torch tensors (also names of ``ntc``).

Each function checks its tensors, allocates its outputs and workspace with torch
and makes the one library call of its name (``include/ntc.h`` has the
definitions); all of that is compiled (``csrc/torch/experts_binding.cpp``), for in a
serving step the host is the bound.  ``stream`` (default: the current stream) is where the
call is queued and where those allocations live; tensors of another stream are the
caller's to order, as for any torch call.  Matrices may have any row stride; their
last dimension is contiguous.  Wrong tensors and values raise ValueError, what the
library refuses NtcError.

Autograd does not record these calls: a result has no gradient, and an input that requires
one draws a warning.  The ``*_backward`` functions compute the gradients.  A call returns
before its kernels have run; ``ntc.ntc_linear_status`` tells whether one of ``linear`` or
``linear_backward`` gave up a wait since it was last asked, which makes results invalid
(a fault of the machine, for valid calls get on).
"""
from __future__ import annotations

import torch

from . import ntc  # loads libntc.so, which _experts needs
from ._build import _experts as _c

_SCORES, _ACTIVATIONS = ntc.SCORES, ntc.ACTIVATIONS


def _choice(table, key, name):
    try:
        return table[key]
    except (KeyError, TypeError):
        raise ValueError(f"{name} must be one of {', '.join(table)}, not {key!r}") from None


def _needs(need, names):
    for n in need:
        if n not in names:
            raise ValueError(f"need must name {', '.join(names)}, not {n!r}")


def route(logits, top_k: int, *, bias=None, score: str = "softmax", groups: int = 1, top_groups: int = 1,
          renormalize: bool = True, scale: float = 1.0, stream=None):
    """ids [n, top_k] int32 and weights [n, top_k] fp32 of each row of logits [n, experts]: see ntc_route."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return route(logits, top_k, bias=bias, score=score, groups=groups, top_groups=top_groups,
                         renormalize=renormalize, scale=scale)
    return _c.route(logits, top_k, bias, _choice(_SCORES, score, "score"), groups, top_groups, bool(renormalize), scale)


def route_backward(logits, ids, dweights, *, score: str = "softmax", renormalize: bool = True, scale: float = 1.0,
                   stream=None):
    """The gradient of route's logits for the gradient of its weights: see ntc_route_backward."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return route_backward(logits, ids, dweights, score=score, renormalize=renormalize, scale=scale)
    return _c.route_backward(logits, ids, dweights, _choice(_SCORES, score, "score"), bool(renormalize), scale)


def expert_order(ids, num_experts: int, *, stream=None):
    """rows [n * k], place [n, k] and offsets [num_experts + 1] (int32) of ids [n, k]: see ntc_expert_order."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return expert_order(ids, num_experts)
    return _c.expert_order(ids, num_experts)


def linear(x, w, bias=None, *, rows=None, offsets=None, activation: str = "none", leaky_slope: float = 0.01,
           residual=None, save: bool = False, stream=None):
    """act(x[rows] w^T + bias) + residual, with each expert's weights for its rows: see ntc_linear.

    x [n, K]; w [E, N, K] (or [N, K]); bias fp32 [E, N] (or [N]); rows int32: the row of x of each row of the
    result (default: the same); offsets int32 [E + 1]: where each expert's rows begin; residual [rows, N].
    save=True also returns the input of the activation, which linear_backward takes as z."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return linear(x, w, bias, rows=rows, offsets=offsets, activation=activation, leaky_slope=leaky_slope,
                          residual=residual, save=save)
    return _c.linear(x, w, bias, rows, offsets, _choice(_ACTIVATIONS, activation, "activation"), leaky_slope, residual,
                     save)


def linear_backward(dy, x, w, *, z=None, rows=None, offsets=None, activation: str = "none", leaky_slope: float = 0.01,
                    need=("dx", "dw", "db"), stream=None):
    """(dx, dw, db) of linear for the gradient dy of its result: see ntc_linear_backward.

    z is what linear(save=True) returned beside the result (not needed without an activation).  dx has a row per
    row of dy; where rows gathered x, combine(dx, place, None, offsets) sums a token's.  dw and db have the shapes
    of w and of its bias; gradients that `need` does not name are None."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return linear_backward(dy, x, w, z=z, rows=rows, offsets=offsets, activation=activation,
                                   leaky_slope=leaky_slope, need=need)
    _needs(need, ("dx", "dw", "db"))
    return _c.linear_backward(dy, x, w, z, rows, offsets, _choice(_ACTIVATIONS, activation, "activation"), leaky_slope,
                              "dx" in need, "dw" in need, "db" in need)


def combine(y, place, weights=None, offsets=None, *, residual=None, stream=None):
    """residual + the sum of y[place[t, j]] times weights[t, j] (1 without weights): see ntc_combine.

    Places from offsets[-1] on (rows of no expert) are left out."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return combine(y, place, weights, offsets, residual=residual)
    return _c.combine(y, place, weights, offsets, residual)


def combine_backward(dout, y, place, weights=None, offsets=None, *, need=("dy", "dweights"), stream=None):
    """(dy, dweights) of combine for the gradient dout of its result: see ntc_combine_backward."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return combine_backward(dout, y, place, weights, offsets, need=need)
    _needs(need, ("dy", "dweights"))
    return _c.combine_backward(dout, y, place, weights, offsets, "dy" in need, "dweights" in need)
