"""The routed-expert calls of libntc on torch tensors (also names of ``ntc``).

Each function checks its tensors, allocates its outputs and workspace with torch
and makes the one library call of its name (``include/ntc.h`` has the
definitions).  ``stream`` (default: the current stream) is where the call is
queued and where those allocations live; tensors of another stream are the
caller's to order, as for any torch call.  Matrices may have any row stride; their
last dimension is contiguous.

A small call is bound by what the host does, so the descriptors are packed with
``struct`` (1.2 us less a call than ctypes structures) and each tensor is looked at
once.
"""
from __future__ import annotations

import struct

import torch

from . import ntc

_TYPES = {torch.float32: ntc.NTC_TYPE_FP32, torch.float16: ntc.NTC_TYPE_FP16, torch.bfloat16: ntc.NTC_TYPE_BF16}
_I32, _F32 = torch.int32, torch.float32

# ntc_route_desc, ntc_linear_desc and ntc_combine_desc in the host's own layout
_ROUTE = struct.Struct("@6Ifi")
_LINEAR = struct.Struct("@i4If8Q")
_COMBINE = struct.Struct("@i3I5Q")

_lib = ntc._lib
_raw_stream = torch._C._cuda_getCurrentRawStream


def _on(stream):
    return torch.cuda.stream(stream)


def _check(status):
    if status:
        raise ntc.NtcError(status, ntc.ntc_last_error())


def _pack(layout, *values):
    try:
        return layout.pack(*values)
    except struct.error:
        raise ValueError("an argument is out of range or not of its type") from None


def _device(t, name):
    d = t.device
    if d.type != "cuda":
        raise ValueError(f"{name} must be a CUDA tensor")
    if d.index != torch.cuda.current_device():
        raise ValueError(f"{name} is on {d}, which is not the current device")
    return d


def _matrix(t, name, rows, cols, dtype, device):
    """The row stride of a [rows, cols] matrix argument, after its checks."""
    if t.dtype is not dtype or t.device != device:
        raise ValueError(f"{name} must be {dtype} on {device}, not {t.dtype} on {t.device}")
    if t.shape != (rows, cols):
        raise ValueError(f"{name} must have shape [{rows}, {cols}], not {list(t.shape)}")
    ld, step = t.stride()
    if step != 1 and cols > 1:
        raise ValueError(f"{name} must be contiguous along its last dimension")
    if rows <= 1:
        return cols
    if ld < cols:
        raise ValueError(f"{name} has overlapping rows")
    return ld


def _array(t, name, shape, dtype, device):
    """The address of a contiguous array argument of this shape (None stays None), after its checks."""
    if t is None:
        return None
    if t.dtype is not dtype or t.device != device:
        raise ValueError(f"{name} must be {dtype} on {device}, not {t.dtype} on {t.device}")
    if t.shape != shape:
        raise ValueError(f"{name} must have shape {list(shape)}, not {list(t.shape)}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


def _two(t, name):
    s = t.shape
    if len(s) != 2:
        raise ValueError(f"{name} must have two dimensions, not {len(s)}")
    return s


def _type(t, name):
    try:
        return _TYPES[t.dtype]
    except KeyError:
        raise ValueError(f"{name} must be float32, float16 or bfloat16, not {t.dtype}") from None


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
        with _on(stream):
            return route(logits, top_k, bias=bias, score=score, groups=groups, top_groups=top_groups,
                         renormalize=renormalize, scale=scale)
    dev = _device(logits, "logits")
    n, E = _two(logits, "logits")
    ld = _matrix(logits, "logits", n, E, logits.dtype, dev)
    d = _pack(_ROUTE, E, top_k, groups, top_groups, _choice(ntc.SCORES, score, "score"), bool(renormalize), scale,
              _type(logits, "logits"))
    b = _array(bias, "bias", (E,), _F32, dev)
    ids = torch.empty((n, top_k), dtype=_I32, device=dev)
    weights = torch.empty((n, top_k), dtype=_F32, device=dev)
    _check(_lib.ntc_route(d, n, logits.data_ptr(), ld, b, ids.data_ptr(), weights.data_ptr(), _raw_stream(dev.index)))
    return ids, weights


def route_backward(logits, ids, dweights, *, score: str = "softmax", renormalize: bool = True, scale: float = 1.0,
                   stream=None):
    """The gradient of route's logits for the gradient of its weights: see ntc_route_backward."""
    if stream is not None:
        with _on(stream):
            return route_backward(logits, ids, dweights, score=score, renormalize=renormalize, scale=scale)
    dev = _device(logits, "logits")
    n, E = _two(logits, "logits")
    k = _two(ids, "ids")[1]
    ld = _matrix(logits, "logits", n, E, logits.dtype, dev)
    d = _pack(_ROUTE, E, k, 1, 1, _choice(ntc.SCORES, score, "score"), bool(renormalize), scale, _type(logits, "logits"))
    i = _array(ids, "ids", (n, k), _I32, dev)
    g = _array(dweights, "dweights", (n, k), _F32, dev)
    out = torch.empty((n, E), dtype=logits.dtype, device=dev)
    _check(_lib.ntc_route_backward(d, n, logits.data_ptr(), ld, i, g, out.data_ptr(), _raw_stream(dev.index)))
    return out


def expert_order(ids, num_experts: int, *, stream=None):
    """rows [n * k], place [n, k] and offsets [num_experts + 1] (int32) of ids [n, k]: see ntc_expert_order."""
    if stream is not None:
        with _on(stream):
            return expert_order(ids, num_experts)
    dev = _device(ids, "ids")
    n, k = _two(ids, "ids")
    if not 1 <= num_experts <= ntc.NTC_MAX_EXPERTS:
        raise ValueError(f"num_experts must be in 1..{ntc.NTC_MAX_EXPERTS}, not {num_experts}")
    i = _array(ids, "ids", (n, k), _I32, dev)
    m = n * k
    rows = torch.empty((m,), dtype=_I32, device=dev)
    place = torch.empty((n, k), dtype=_I32, device=dev)
    offsets = torch.empty((num_experts + 1,), dtype=_I32, device=dev)
    size = _lib.ntc_expert_order_workspace(m, num_experts)
    ws = torch.empty((size,), dtype=torch.uint8, device=dev) if size else None
    _check(_lib.ntc_expert_order(i, m, k, num_experts, rows.data_ptr(), place.data_ptr(), offsets.data_ptr(),
                                 ws.data_ptr() if size else None, size, _raw_stream(dev.index)))
    return rows, place, offsets


def _operands(x, w, dev):
    """E, N, K and the strides of x and w, after their checks."""
    s = w.shape
    if len(s) == 3:
        E, N, K = s
        step, ldw, one = w.stride()
    elif len(s) == 2:
        (N, K), E = s, 1
        ldw, one = w.stride()
        step = 0
    else:
        raise ValueError(f"w must have two or three dimensions, not {len(s)}")
    dt = x.dtype
    if w.dtype is not dt or w.device != dev:
        raise ValueError(f"w must be {dt} on {dev}, not {w.dtype} on {w.device}")
    if one != 1 and K > 1:
        raise ValueError("w must be contiguous along its last dimension")
    if N <= 1:
        ldw = K
    if E <= 1:
        step = N * ldw
    n = _two(x, "x")[0]
    return E, N, K, n, _matrix(x, "x", n, K, dt, dev), ldw, step


def linear(x, w, bias=None, *, rows=None, offsets=None, activation: str = "none", leaky_slope: float = 0.01,
           residual=None, save: bool = False, stream=None):
    """act(x[rows] w^T + bias) + residual, with each expert's weights for its rows: see ntc_linear.

    x [n, K]; w [E, N, K] (or [N, K]); bias fp32 [E, N] (or [N]); rows int32: the row of x of each row of the
    result (default: the same); offsets int32 [E + 1]: where each expert's rows begin; residual [rows, N].
    save=True also returns the input of the activation, which linear_backward takes as z."""
    if stream is not None:
        with _on(stream):
            return linear(x, w, bias, rows=rows, offsets=offsets, activation=activation, leaky_slope=leaky_slope,
                          residual=residual, save=save)
    dev = _device(x, "x")
    E, N, K, n, ldx, ldw, step = _operands(x, w, dev)
    dt = x.dtype
    m = n if rows is None else rows.shape[0]
    r = _array(rows, "rows", (m,), _I32, dev)
    o = _array(offsets, "offsets", (E + 1,), _I32, dev)
    b = None
    if bias is not None:
        b = _array(bias, "bias", (N,) if bias.dim() == 1 and E == 1 else (E, N), _F32, dev)
    ldr, res = N, None
    if residual is not None:
        ldr, res = _matrix(residual, "residual", m, N, dt, dev), residual.data_ptr()
    d = _pack(_LINEAR, _type(x, "x"), K, N, E, _choice(ntc.ACTIVATIONS, activation, "activation"), leaky_slope, m, n,
              ldx, ldw, step, N, N, ldr)
    px, pw = x.data_ptr(), w.data_ptr()
    y = torch.empty((m, N), dtype=dt, device=dev)
    z = torch.empty((m, N), dtype=dt, device=dev) if save else None
    size = _lib.ntc_linear_workspace(d, px, r, pw)
    ws = torch.empty((size,), dtype=torch.uint8, device=dev) if size else None
    _check(_lib.ntc_linear(d, px, r, o, pw, b, res, y.data_ptr(), z.data_ptr() if save else None,
                           ws.data_ptr() if size else None, size, _raw_stream(dev.index)))
    return (y, z) if save else y


def linear_backward(dy, x, w, *, z=None, rows=None, offsets=None, activation: str = "none", leaky_slope: float = 0.01,
                    need=("dx", "dw", "db"), stream=None):
    """(dx, dw, db) of linear for the gradient dy of its result: see ntc_linear_backward.

    z is what linear(save=True) returned beside the result (not needed without an activation).  dx has a row per
    row of dy; where rows gathered x, combine(dx, place, None, offsets) sums a token's.  dw and db have the shapes
    of w and of its bias; gradients that `need` does not name are None."""
    if stream is not None:
        with _on(stream):
            return linear_backward(dy, x, w, z=z, rows=rows, offsets=offsets, activation=activation,
                                   leaky_slope=leaky_slope, need=need)
    dev = _device(x, "x")
    E, N, K, n, ldx, ldw, step = _operands(x, w, dev)
    dt = x.dtype
    m = _two(dy, "dy")[0]
    r = _array(rows, "rows", (m,), _I32, dev)
    o = _array(offsets, "offsets", (E + 1,), _I32, dev)
    ldy = _matrix(dy, "dy", m, N, dt, dev)
    act = _choice(ntc.ACTIVATIONS, activation, "activation")
    ldz, pz = N, None
    if act:
        if z is None:
            raise ValueError(f"activation {activation!r} needs z")
        ldz, pz = _matrix(z, "z", m, N, dt, dev), z.data_ptr()
    _needs(need, ("dx", "dw", "db"))
    d = _pack(_LINEAR, _type(x, "x"), K, N, E, act, leaky_slope, m, n, ldx, ldw, step, ldy, ldz, N)
    py, px, pw = dy.data_ptr(), x.data_ptr(), w.data_ptr()
    dx = torch.empty((m, K), dtype=dt, device=dev) if "dx" in need else None
    dw = torch.empty(w.shape, dtype=dt, device=dev) if "dw" in need else None
    db = torch.empty(w.shape[:-1], dtype=_F32, device=dev) if "db" in need else None
    size = _lib.ntc_linear_backward_workspace(d, py, px, r, pw)
    ws = torch.empty((size,), dtype=torch.uint8, device=dev) if size else None
    _check(_lib.ntc_linear_backward(d, py, pz, px, r, o, pw, None if dx is None else dx.data_ptr(),
                                    None if dw is None else dw.data_ptr(), None if db is None else db.data_ptr(),
                                    ws.data_ptr() if size else None, size, _raw_stream(dev.index)))
    return dx, dw, db


def combine(y, place, weights=None, offsets=None, *, residual=None, stream=None):
    """residual + the sum of y[place[t, j]] times weights[t, j] (1 without weights): see ntc_combine.

    Places from offsets[-1] on (rows of no expert) are left out."""
    if stream is not None:
        with _on(stream):
            return combine(y, place, weights, offsets, residual=residual)
    dev = _device(y, "y")
    m, D = _two(y, "y")
    T, k = _two(place, "place")
    dt = y.dtype
    E = 1 if offsets is None else offsets.shape[0] - 1
    ldy = _matrix(y, "y", m, D, dt, dev)
    p = _array(place, "place", (T, k), _I32, dev)
    g = _array(weights, "weights", (T, k), _F32, dev)
    o = _array(offsets, "offsets", (E + 1,), _I32, dev)
    ldr, res = D, None
    if residual is not None:
        ldr, res = _matrix(residual, "residual", T, D, dt, dev), residual.data_ptr()
    d = _pack(_COMBINE, _type(y, "y"), D, k, E, T, m, ldy, D, ldr)
    out = torch.empty((T, D), dtype=dt, device=dev)
    _check(_lib.ntc_combine(d, y.data_ptr(), p, g, o, res, out.data_ptr(), _raw_stream(dev.index)))
    return out


def combine_backward(dout, y, place, weights=None, offsets=None, *, need=("dy", "dweights"), stream=None):
    """(dy, dweights) of combine for the gradient dout of its result: see ntc_combine_backward."""
    if stream is not None:
        with _on(stream):
            return combine_backward(dout, y, place, weights, offsets, need=need)
    dev = _device(y, "y")
    m, D = _two(y, "y")
    T, k = _two(place, "place")
    dt = y.dtype
    E = 1 if offsets is None else offsets.shape[0] - 1
    ldy = _matrix(y, "y", m, D, dt, dev)
    ldo = _matrix(dout, "dout", T, D, dt, dev)
    p = _array(place, "place", (T, k), _I32, dev)
    g = _array(weights, "weights", (T, k), _F32, dev)
    o = _array(offsets, "offsets", (E + 1,), _I32, dev)
    _needs(need, ("dy", "dweights"))
    d = _pack(_COMBINE, _type(y, "y"), D, k, E, T, m, ldy, ldo, D)
    dy = torch.empty((m, D), dtype=dt, device=dev) if "dy" in need else None
    dw = torch.empty((T, k), dtype=_F32, device=dev) if "dweights" in need else None
    _check(_lib.ntc_combine_backward(d, dout.data_ptr(), y.data_ptr(), p, g, o, None if dy is None else dy.data_ptr(),
                                     None if dw is None else dw.data_ptr(), _raw_stream(dev.index)))
    return dy, dw
