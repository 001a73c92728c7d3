"""Plain 64-bit forms of the balance loss, the AdamW step and the weights in 4 bits, with bounds from the arithmetic.

u32 = 2^-24 is half a step of fp32; a sum of n fp32 terms in any order is off by at most n u32 of their magnitudes; exp
and the division by a sum are allowed R.SPECIAL = 2^-18 of their result, as for the router."""
import math

import torch

import tests.experts_ref as R

U32 = 2.0 ** -24
# The balance loss adds a lane's tokens, the lanes and warps of a CTA and the CTAs' rows: below 640 additions in a
# chain for 65,536 tokens on 304 CTAs (28 + 5 + 8 + 76 + 512).
CHAIN = 640


def probabilities(logits, score):
    s, dead = R.scores(logits, score)
    if score == "sigmoid":  # from logarithms: a row far below 0 has its ratios, too
        l = torch.where(dead, torch.full_like(s, -math.inf), torch.nn.functional.logsigmoid(logits.double().clamp(max=3e38)))
        top = l.max(1, keepdim=True).values
        s = torch.where(dead, torch.zeros_like(s), torch.exp(l - torch.where(torch.isfinite(top), top, torch.zeros_like(top))))
    total = s.sum(1, keepdim=True)
    return torch.where(total > 0, s / total.clamp_min(1e-300), torch.zeros_like(s)), dead


def counts(ids, E):
    live = (ids >= 0) & (ids < E)
    c = torch.bincount(ids[live].long(), minlength=E)
    return c, live.any(1) if ids.numel() else torch.zeros(ids.shape[0], dtype=torch.bool, device=ids.device)


def balance_loss(logits, ids, score="softmax", scale=1.0):
    """loss, counts, mean and the bounds of loss and mean."""
    E = logits.shape[1]
    p, _ = probabilities(logits, score)
    c, live = counts(ids, E)
    n, C = int(live.sum()), int(c.sum())
    mean = p[live].sum(0) / max(n, 1)
    loss = scale * E * float((c.double() * mean).sum()) / max(C, 1)
    b_mean = mean * (R.SPECIAL + CHAIN * U32) + 1e-37
    b_loss = abs(scale) * E * float((c.double() * b_mean).sum()) / max(C, 1) + abs(loss) * (E + 8) * U32 + 1e-37
    return loss, torch.cat([c, live.sum()[None]]).int(), mean, b_loss, b_mean


def balance_loss_backward(logits, ids, score="softmax", scale=1.0, dloss=1.0, residual=None):
    """dlogits and their bounds."""
    E = logits.shape[1]
    p, dead = probabilities(logits, score)
    c, live = counts(ids, E)
    a = dloss * scale * E / (max(int(live.sum()), 1) * max(int(c.sum()), 1))
    d = c.double() - c.double()[p.argmax(1)][:, None]
    dot = (p * d).sum(1, keepdim=True)
    slope = torch.sigmoid(-logits.double()) if score == "sigmoid" else torch.ones_like(p)
    g = a * p * (d - dot) * slope
    off = abs(a) * p * slope * ((d - dot).abs() * 3 * R.SPECIAL + (p * d.abs()).sum(1, keepdim=True) * (2 * R.SPECIAL + (E + 8) * U32))
    keep = live[:, None] & ~dead
    g, off = torch.where(keep, g, torch.zeros_like(g)), torch.where(keep, off, torch.zeros_like(g))
    if residual is not None:
        g = g + residual.double()
        off = off + U32 * g.abs()
    u, tiny = R.UNIT[logits.dtype], R.TINY[logits.dtype]
    return g, off + u * (g.abs() + off) + tiny


def adamw(p, g, m, v, step, lr, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01, grad_scale=1.0):
    """p, m, v of one step and their bounds in fp32 (p before it is rounded to its type).

    Each constant is rounded once and each operation once: three roundings of a term and one of the sum for m, one more
    for v, and for the change of p those of m and v (half of v's in the root) and eight of its own."""
    p, g, m, v = (t.double() for t in (p, g, m, v))
    f = g * grad_scale
    m1 = beta1 * m + (1 - beta1) * f
    v1 = beta2 * v + (1 - beta2) * f * f
    b_m = 4 * U32 * ((beta1 * m).abs() + ((1 - beta1) * f).abs()) + 1e-38
    b_v = 6 * U32 * v1 + 1e-38
    c1, c2 = 1 - beta1 ** step, 1 - beta2 ** step
    down = v1.sqrt() / math.sqrt(c2) + eps
    change = lr / c1 * m1 / down
    p1 = (1 - lr * weight_decay) * p - change
    # a root of a v that is off by b_v: sqrt(v + b) - sqrt(v) <= min(b / (2 sqrt(v)), sqrt(b))
    b_root = torch.minimum(b_v / (2 * v1.sqrt()).clamp_min(1e-300), b_v.sqrt()) / math.sqrt(c2)
    b_change = lr / c1 * b_m / down + change.abs() * (b_root / down + 12 * U32)
    return p1, m1, v1, b_change + 4 * U32 * (p.abs() + change.abs()) + 1e-38, b_m, b_v


def scale_of(w, group):
    """Groups [..., G, group] of weights [..., K], padded with zeros, in 64 bits."""
    K = w.shape[-1]
    G = -(-K // group)
    return torch.nn.functional.pad(w.double(), (0, G * group - K)).unflatten(-1, (G, group))


def pack4(w, group, dtype):
    """q [..., K] and the scales, as ntc_pack4 defines them."""
    f = scale_of(w, group)
    top = f.abs().amax(-1)
    bad = ~torch.isfinite(f).all(-1)
    # the largest magnitude times 1/7, rounded to fp32 and to 16 bits
    s = (top.float() * torch.tensor(1.0 / 7.0, dtype=torch.float32)).to(dtype)
    s = torch.where(bad, torch.full_like(s, math.nan), s)
    at = s.double()[..., None]
    q = torch.where(at > 0, torch.round(torch.where(at > 0, f / at, torch.zeros_like(f))), torch.zeros_like(f)).clamp(-8, 7)
    return q.flatten(-2)[..., :w.shape[-1]], s


def nibbles(packed, K):
    return torch.stack([packed & 15, packed >> 4], -1).flatten(-2)[..., :K].double() - 8


def values(packed, scales, K, group):
    """The weights in 64 bits."""
    return nibbles(packed, K) * scales.double().repeat_interleave(group, -1)[..., :K]
