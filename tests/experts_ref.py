"""Plain 64-bit forms of the routed-expert calls, and the bounds their tests use.

Bounds are per element, from the arithmetic alone: u is the unit roundoff of the
result's type, a sum of n fp32 products in any order is off by at most
n * 2^-23 * (the sum of the terms' magnitudes) (2^-23, not 2^-24: a tensor core
may truncate), exp, erf and division cost a few 2^-23 of their result and are
allowed 2^-18 of the activation's input or result.
"""
import math

import torch

F32 = 2.0 ** -23
SPECIAL = 2.0 ** -18
UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 2.0 ** -126, torch.bfloat16: 2.0 ** -126, torch.float16: 2.0 ** -24}


def act(name, z, slope=0.01):
    if name == "none":
        return z
    if name == "relu":
        return torch.where(z < 0, torch.zeros_like(z), z)
    if name == "leaky":
        return torch.where(z > 0, z, slope * z)
    if name == "gelu":
        return z * torch.special.ndtr(z)
    return z / (1 + torch.exp(-z))


def act_slope(name, z, slope=0.01):
    if name == "none":
        return torch.ones_like(z)
    if name == "relu":
        return (z > 0).to(z.dtype)
    if name == "leaky":
        return torch.where(z > 0, torch.ones_like(z), torch.full_like(z, slope))
    if name == "gelu":
        return torch.special.ndtr(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    s = 1 / (1 + torch.exp(-z))
    return s * (1 + z * (1 - s))


def order(ids, E):
    """rows, place, offsets by a stable sort; ids outside 0..E-1 last."""
    T, k = ids.shape
    key = torch.where((ids >= 0) & (ids < E), ids, E).reshape(-1).long()
    at = torch.sort(key, stable=True).indices
    place = torch.empty_like(at)
    place[at] = torch.arange(at.numel(), device=ids.device)
    counts = torch.bincount(key, minlength=E + 1)
    offsets = torch.zeros(E + 1, dtype=torch.long, device=ids.device)
    offsets[1:] = counts[:E].cumsum(0)
    return (at // k).int(), place.view(T, k).int(), offsets.int()


def segments(offsets, m):
    if offsets is None:
        return [(0, 0, m)]
    o = offsets.tolist()
    return [(e, o[e], o[e + 1]) for e in range(len(o) - 1)]


def gathered(x, rows):
    """x's rows in the order of rows, zeros for an index outside x."""
    if rows is None:
        return x.double()
    r = rows.long()
    inside = (r >= 0) & (r < x.shape[0])
    return torch.where(inside[:, None], x.double()[r.clamp(0, x.shape[0] - 1)], torch.zeros((), dtype=torch.float64, device=x.device))


def linear(x, w, bias=None, rows=None, offsets=None, activation="none", slope=0.01, residual=None):
    """y, z and their bounds (|got - want| <= bound) for results of x's type."""
    if w.dim() == 2:
        w = w[None]
    xs = gathered(x, rows)
    m, (E, N, K) = xs.shape[0], w.shape
    z = torch.zeros(m, N, dtype=torch.float64, device=x.device)
    mag = torch.zeros_like(z)
    live = torch.zeros(m, dtype=torch.bool, device=x.device)
    for e, a, o in segments(offsets, m):
        we = w[e].double()
        z[a:o] = xs[a:o] @ we.t()
        mag[a:o] = xs[a:o].abs() @ we.abs().t()
        if bias is not None:
            b = bias.view(E, N)[e].double()
            z[a:o] += b
            mag[a:o] += b.abs()
        live[a:o] = True
    y = act(activation, z, slope)
    r = torch.zeros_like(y)
    if residual is not None:
        r = torch.where(live[:, None], residual.double(), r)
    u, tiny = UNIT[x.dtype], TINY[x.dtype]
    zb = (K + 8) * F32 * mag
    yb = 1.2 * zb + SPECIAL * z.abs() + 4 * F32 * r.abs()
    y = torch.where(live[:, None], y, torch.zeros_like(y)) + r
    return y, z, yb + u * (y.abs() + yb) + tiny, zb + u * (z.abs() + zb) + tiny


def linear_backward(dy, x, w, z, rows, offsets, activation, slope=0.01):
    """dx, dw, db and their bounds."""
    if w.dim() == 2:
        w = w[None]
    E, N, K = w.shape
    m = dy.shape[0]
    xs = gathered(x, rows)
    dz = dy.double() * (act_slope(activation, z.double(), slope) if activation != "none" else 1.0)
    u, tiny = UNIT[x.dtype], TINY[x.dtype]
    off = dz.abs() * F32 * 4 + (SPECIAL * dy.double().abs() * (1 + (z.double().abs() if z is not None else 0))
                                if activation in ("gelu", "silu") else 0)
    rounded = 0.0 if activation == "none" else u * (dz.abs() + off) + tiny  # dz, rounded for the products
    e_dz = off + rounded
    dev = x.device
    dx, bx = (torch.zeros(m, K, dtype=torch.float64, device=dev) for _ in range(2))
    dw, bw = (torch.zeros(E, N, K, dtype=torch.float64, device=dev) for _ in range(2))
    db, bb = (torch.zeros(E, N, dtype=torch.float64, device=dev) for _ in range(2))
    for e, a, o in segments(offsets, m):
        we = w[e].double()
        n = o - a
        dx[a:o] = dz[a:o] @ we
        bx[a:o] = (e_dz[a:o] + (N + 8) * F32 * dz[a:o].abs()) @ we.abs()
        dw[e] = dz[a:o].t() @ xs[a:o]
        bw[e] = (e_dz[a:o] + (n + 8) * F32 * dz[a:o].abs()).t() @ xs[a:o].abs()
        db[e] = dz[a:o].sum(0)
        bb[e] = (off[a:o] + (n + 8) * F32 * dz[a:o].abs()).sum(0)
    return (dx, bx * 1.01 + u * dx.abs() * 1.01 + tiny), (dw, bw * 1.01 + u * dw.abs() * 1.01 + tiny), (db, bb + 1e-37)


def scores(logits, score):
    """64-bit scores; masked experts (-inf, NaN) have 0."""
    l = logits.double()
    dead = ~(l > -math.inf)
    l = l.clamp(max=torch.finfo(torch.float32).max)
    if score == "sigmoid":
        s = 1 / (1 + torch.exp(-l))
    else:
        m = torch.where(dead, torch.full_like(l, -math.inf), l).max(1, keepdim=True).values
        m = torch.where(torch.isfinite(m), m, torch.zeros_like(m))
        e = torch.where(dead, torch.zeros_like(l), torch.exp(l - m))
        s = e / e.sum(1, keepdim=True).clamp_min(1e-300)
    return torch.where(dead, torch.zeros_like(s), s), dead


def route(logits, k, bias=None, score="softmax", groups=1, top_groups=1, renormalize=True, scale=1.0):
    """ids and weights, row by row and expert by expert as the definition says it."""
    s, dead = scores(logits, score)
    c = s if bias is None else s + bias.double()
    T, E = s.shape
    ids = torch.full((T, k), -1, dtype=torch.int32)
    w = torch.zeros(T, k, dtype=torch.float64)
    sl, cl, dl = s.tolist(), c.tolist(), dead.tolist()
    per = E // groups
    for t in range(T):
        alive = [e for e in range(E) if not dl[t][e] and cl[t][e] == cl[t][e]]
        if groups > 1:
            value = []
            for g in range(groups):
                top = sorted((cl[t][e] for e in alive if e // per == g), reverse=True)[:2]
                if top:
                    value.append((-sum(top), g))
            kept = {g for _, g in sorted(value)[:top_groups]}
            alive = [e for e in alive if e // per in kept]
        alive.sort(key=lambda e: (-cl[t][e], e))
        pick = alive[:k]
        total = sum(sl[t][e] for e in pick)
        for j, e in enumerate(pick):
            ids[t, j] = e
            w[t, j] = scale * (sl[t][e] / total if renormalize and total > 0 else 0.0 if renormalize else sl[t][e])
    return ids, w


def route_weights(logits, ids, score, renormalize, scale):
    """The weights of given ids as a differentiable 64-bit function of the logits."""
    l = logits
    s = torch.sigmoid(l) if score == "sigmoid" else torch.softmax(l, 1)
    p = s.gather(1, ids.clamp_min(0).long()) * (ids >= 0)
    return scale * (p / p.sum(1, keepdim=True) if renormalize else p)


def assert_within(got, want, bound, what=""):
    d = (got.double() - want).abs()
    bad = ~(d <= bound)
    assert not bad.any(), (what, int(bad.sum()), "of", bad.numel(), "worst", float((d / bound)[bad].max()),
                           bad.nonzero()[0].tolist())
