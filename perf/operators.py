"""Performance cases of routed experts: the router, the experts' products, and their blend.

A router gives every token (a texel's latent features, or any other row) the
``top_k`` of E experts and their weights; the tokens' entries are ordered by
expert; each expert's rows go through its linear layers (bias, activation and
residual in the product's epilogue); a token's rows are blended with its weights.

``op`` of a case names the call:
  route         ids and weights from logits, and the order by expert made from the ids
  route_back    the gradient of the logits
  linear        one product of every expert with its rows (or a dense one, experts=1)
  linear_back   the gradients of its input, weights and bias
  combine       the weighted sum of each token's rows
  combine_back  the gradients of the rows and of the weights
  layer         route, order, linear (gathering its rows), linear, combine

``exact()`` evaluates the definitions in 64 bits, expert by expert.
"""
import math

import torch

own = False

DTYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}

# Every field of a case, with the value it has when a case does not name it.
DEFAULTS = dict(
    op="linear", tokens=1, experts=1, top_k=1, dtype="bf16",
    # router
    score="softmax", bias=False, groups=1, top_groups=1, renorm=True, scale=1.0,
    # products: width in, width out (layer: model width, hidden width)
    d_in=0, d_out=0, act="none", residual=False, save=False,
    padding=0.0,  # share of the tokens that are padding: no expert takes them
)


def full(case):
    return dict(DEFAULTS, **{k: v for k, v in case.items() if k != "name"})


def listed():
    return [
        # one serving step of a batch of 16 sequences: launches and latency are the whole cost
        dict(name="route-step", op="route", tokens=16, experts=128, top_k=8, dtype="fp32"),
        # a prefill chunk through a large router: sigmoid scores, balance bias, half of the groups
        dict(name="route-prefill", op="route", tokens=32768, experts=256, top_k=8, dtype="bf16", score="sigmoid",
             bias=True, groups=8, top_groups=4, scale=2.5),
        # the router's gradient in a training step
        dict(name="route-back-train", op="route_back", tokens=65536, experts=64, top_k=6, dtype="fp32"),
        # one token through its 8 experts: the weights' bytes are the cost
        dict(name="linear-token", op="linear", tokens=1, experts=64, top_k=8, d_in=2048, d_out=1024, act="silu"),
        # a serving step of 64 sequences, a few rows per expert, padding slots in the batch
        dict(name="linear-step", op="linear", tokens=64, experts=32, top_k=4, d_in=1024, d_out=2048, dtype="fp16",
             act="gelu", residual=True, padding=0.125),
        # a dense layer whose sizes fit no tile and no vector load
        dict(name="linear-dense-odd", op="linear", tokens=1999, d_in=771, d_out=1027, dtype="fp16", act="leaky",
             residual=True),
        # the experts' first product in a training step, its input to the activation kept for the gradient
        dict(name="linear-experts-train", op="linear", tokens=16384, experts=16, top_k=2, d_in=2048, d_out=4096,
             act="gelu", save=True),
        # the gradients of such a product
        dict(name="linear-back-train", op="linear_back", tokens=8192, experts=8, top_k=2, d_in=1024, d_out=4096,
             act="gelu"),
        # the gradients of a small dense layer of odd sizes
        dict(name="linear-back-odd", op="linear_back", tokens=777, d_in=301, d_out=513, dtype="fp16", act="relu"),
        # the blend of eight experts' rows with the residual stream
        dict(name="combine-prefill", op="combine", tokens=16384, experts=64, top_k=8, d_out=2048, residual=True),
        # its gradient
        dict(name="combine-back-train", op="combine_back", tokens=8192, experts=32, top_k=4, d_out=1024, dtype="fp16",
             padding=0.05),
        # the whole routed layer over a prefill chunk
        dict(name="layer-prefill", op="layer", tokens=4096, experts=32, top_k=4, d_in=1024, d_out=2048, act="silu"),
    ]


def draw(rng):
    def logu(lo, hi):
        return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))

    def width(lo, hi):  # half of them multiples of 64, the others as they fall
        w = logu(lo, hi)
        w = max(lo, w // 64 * 64) if rng.random() < 0.5 else w
        return w + 64 if w == 3072 else w

    op = rng.choice(["route", "route", "route_back", "linear", "linear", "linear", "linear_back", "linear_back",
                     "combine", "combine_back", "layer"])
    c = dict(op=op, dtype=rng.choice(["bf16", "fp16"]))
    if op in ("route", "route_back"):
        c["dtype"] = rng.choice(["fp32", "bf16", "fp16"])
        c["tokens"] = logu(1, 65536)
        if rng.random() < 0.4:
            c["groups"] = rng.choice([2, 4, 8])
            c["experts"] = c["groups"] * logu(2, 32)
            c["top_groups"] = rng.randint(1, c["groups"])
        else:
            c["experts"] = logu(2, 586)
        reach = c["experts"] // c.get("groups", 1) * c.get("top_groups", 1)
        c["top_k"] = rng.randint(1, min(10, reach))
        c["score"] = rng.choice(["softmax", "sigmoid"])
        c["renorm"] = rng.random() < 0.7
        c["scale"] = rng.choice([1.0, 2.5])
        if op == "route":
            c["bias"] = rng.random() < 0.5
        return c
    dense = op in ("linear", "linear_back") and rng.random() < 0.3
    c["experts"] = 1 if dense else logu(2, 128)
    c["top_k"] = 1 if dense else rng.randint(1, min(8, c["experts"]))
    c["d_out"] = width(16, 4096)
    if op in ("combine", "combine_back"):
        c["tokens"] = logu(1, 16384)
        c["residual"] = op == "combine" and rng.random() < 0.5
        c["padding"] = rng.choice([0.0, 0.1])
        return c
    c["d_in"] = width(16, 4096)
    while c["experts"] * c["d_in"] * c["d_out"] > 1 << 27:  # the weights stay below 256 MB
        c["experts"] = max(1, c["experts"] // 2)
    c["top_k"] = min(c["top_k"], c["experts"])
    # as many tokens as keep the pass below the largest listed one
    per = 2.0 * c["top_k"] * c["d_in"] * c["d_out"] * (1 if op == "linear" else 2)
    c["tokens"] = logu(1, int(max(1, min(16384, 2.0e11 / per, (1 << 27) / (c["top_k"] * max(c["d_in"], c["d_out"]))))))
    c["act"] = rng.choice(["none", "relu", "leaky", "gelu", "silu"])
    if op == "linear":
        c["residual"] = rng.random() < 0.4
        c["save"] = rng.random() < 0.3
    c["padding"] = 0.0 if dense else rng.choice([0.0, 0.1])
    return c


# ------------------------------------------------------------------ inputs

SLOPE = 0.01  # leaky activation


def choices(c, logits, bias):
    """Scores, the values that the choice goes by, and the ids in descending order, all in the logits' type."""
    s = torch.sigmoid(logits) if c["score"] == "sigmoid" else torch.softmax(logits, 1)
    v = s if bias is None else s + bias.to(s.dtype)
    group = None
    if c["groups"] > 1:
        T, G = v.shape[0], c["groups"]
        per = c["experts"] // G
        group = v.view(T, G, per).sort(dim=2, descending=True).values[:, :, :2].sum(2)
        kept = torch.zeros_like(group, dtype=torch.bool).scatter_(
            1, group.sort(dim=1, descending=True, stable=True).indices[:, :c["top_groups"]], True)
        v = v.masked_fill(~kept.repeat_interleave(per, dim=1), -math.inf)
    val, ids = v.sort(dim=1, descending=True, stable=True)
    return s, val, ids, group


def separate(c, logits, bias):
    """Rows whose choice hangs on a relative difference below 1e-5 -- where two correct evaluations in 32 bits may
    choose differently -- are replaced by rows that do not."""
    _, val, _, group = choices(c, logits.double(), bias)
    k = c["top_k"]
    top = val[:, :k + 1]
    top = torch.where(torch.isfinite(top), top, torch.full_like(top, -1.0))
    close = ((top[:, :-1] - top[:, 1:]) < 1e-5 * top[:, :-1].abs().clamp_min(1e-3)).any(1) if top.shape[1] > 1 else \
        torch.zeros(logits.shape[0], dtype=torch.bool, device=logits.device)
    if group is not None and c["top_groups"] < c["groups"]:
        g = group.sort(dim=1, descending=True).values
        a, b = g[:, c["top_groups"] - 1], g[:, c["top_groups"]]
        close |= (a - b) < 1e-5 * a.abs().clamp_min(1e-3)
    good = (~close).nonzero().view(-1)
    bad = close.nonzero().view(-1)
    if bad.numel() and good.numel():
        logits[bad] = logits[good[torch.arange(bad.numel(), device=logits.device) % good.numel()]]
    return logits


def route_ids(c, g, dev):
    """top_k distinct experts per token, some experts more popular than others; padding tokens have -1."""
    T, E, k = c["tokens"], c["experts"], c["top_k"]
    noise = -torch.log(-torch.log(torch.rand(T, E, generator=g, device=dev).clamp(1e-7, 1 - 1e-7)))
    ids = (noise + 0.5 * torch.randn(E, generator=g, device=dev)).topk(k, dim=1).indices.to(torch.int32)
    if c["padding"]:
        ids[torch.rand(T, generator=g, device=dev) < c["padding"]] = -1
    return ids


def order_of(ids, E):
    """rows (token of each ordered entry), place (ordered position of each entry), offsets (first entry of each expert)."""
    T, k = ids.shape
    key = torch.where((ids >= 0) & (ids < E), ids, E).view(-1).long()
    order = key.sort(stable=True).indices
    place = torch.empty_like(order)
    place[order] = torch.arange(order.numel(), device=ids.device)
    offsets = (key[None, :] < torch.arange(E + 1, device=ids.device)[:, None]).sum(1) if T * k * E <= 1 << 24 else \
        torch.bincount(key, minlength=E + 1).cumsum(0).roll(1).scatter(0, torch.zeros(1, dtype=torch.long, device=ids.device), 0)
    return (order // k).to(torch.int32), place.view(T, k).to(torch.int32), offsets.to(torch.int32)


def prepare(case, seed):
    c = full(case)
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(seed)
    dt = DTYPES[c["dtype"]]
    T, E, k, op = c["tokens"], c["experts"], c["top_k"], c["op"]

    def normal(*shape, std=1.0, dtype=None):
        return (torch.randn(*shape, generator=g, device=dev) * std).to(dtype or dt)

    st = dict(case=c)
    if op in ("route", "route_back", "layer"):
        st["bias"] = normal(E, std=0.02, dtype=torch.float32) if c["bias"] else None
        st["logits"] = separate(c, normal(T, E), st["bias"])
    if op == "route_back":
        st["ids"] = choices(c, st["logits"].double(), None)[2][:, :k].to(torch.int32).contiguous()
        st["dweights"] = normal(T, k, dtype=torch.float32)
    if op in ("linear", "linear_back", "combine", "combine_back"):
        if E > 1 or op.startswith("combine"):
            ids = route_ids(c, g, dev)
            st["rows"], st["place"], st["offsets"] = order_of(ids, E)
            # the largest number of rows of one expert: what a padded batch is sized by
            st["most"] = int((st["offsets"][1:] - st["offsets"][:-1]).max())
        else:
            st["rows"] = st["offsets"] = None
    n = T * k
    if op in ("linear", "linear_back"):
        K, N = c["d_in"], c["d_out"]
        st["x"] = normal(T, K)
        st["w"] = normal(E, N, K, std=K ** -0.5)
        st["b"] = normal(E, N, std=0.1, dtype=torch.float32)
        if op == "linear":
            st["r"] = normal(n, N) if c["residual"] else None
        else:
            st["z"] = normal(n, N) if c["act"] != "none" else None
            st["dy"] = normal(n, N)
    if op == "layer":
        D, H = c["d_in"], c["d_out"]
        st["x"] = normal(T, D)
        st["w1"], st["b1"] = normal(E, H, D, std=D ** -0.5), normal(E, H, std=0.1, dtype=torch.float32)
        st["w2"], st["b2"] = normal(E, D, H, std=H ** -0.5), normal(E, D, std=0.1, dtype=torch.float32)
    if op in ("combine", "combine_back"):
        D = c["d_out"]
        st["y"] = normal(n, D)
        st["weights"] = torch.softmax(normal(T, k, dtype=torch.float32), 1)
        if op == "combine":
            st["r"] = normal(T, D) if c["residual"] else None
        else:
            st["dout"] = normal(T, D)
    return st


# ------------------------------------------------------------- the plain form

def act_of(a, z):
    if a == "none":
        return z
    if a == "relu":
        return z.clamp_min(0)
    if a == "leaky":
        return torch.where(z > 0, z, SLOPE * z)
    if a == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    return z * torch.sigmoid(z)


def act_slope(a, z):
    if a == "relu":
        return (z > 0).to(z.dtype)
    if a == "leaky":
        return torch.where(z > 0, torch.ones_like(z), torch.full_like(z, SLOPE))
    if a == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi))
    s = torch.sigmoid(z)
    return s * (1 + z * (1 - s))


def plain_route(c, logits, bias):
    s, _, order, _ = choices(c, logits.float(), bias)
    ids = order[:, :c["top_k"]]
    w = s.gather(1, ids)
    if c["renorm"]:
        w = w / w.sum(1, keepdim=True)
    return ids.to(torch.int32), w * c["scale"]


def padded(st, E):
    """Each expert's rows in a batch [E, most]: the ordered row in every slot, whether it is one, and each row's slot."""
    off = st["offsets"].long()
    dev = off.device
    at = off[:-1, None] + torch.arange(st["most"], device=dev)
    is_row = at < off[1:, None]
    n = st["rows"].shape[0]
    i = torch.arange(n, device=dev)
    e = torch.bucketize(i, off[1:], right=True)
    live = e < E
    e = e.clamp_max(E - 1)
    return at.clamp_max(n - 1), is_row, e, (i - off[e]).clamp_max(st["most"] - 1).clamp_min(0), live


def plain_linear(st, x, w, b, act, rows, residual, save):
    dt, E = x.dtype, w.shape[0]
    if st["offsets"] is None:
        z = x.float() @ w[0].float().t() + b[0]
        live = None
    else:
        at, is_row, e, slot, live = padded(st, E)
        src = rows if rows is not None else torch.arange(x.shape[0], device=x.device, dtype=torch.int32)
        if src.shape[0] <= E:  # few rows: only the weights that they need
            z = torch.bmm(w[e].float(), x[src.long()].float()[:, :, None])[:, :, 0] + b[e]
        else:
            z = torch.bmm(x[src.long()[at]].float(), w.float().transpose(1, 2)) + b[:, None, :]
            z = z[e, slot]
        z = torch.where(live[:, None], z, torch.zeros((), device=z.device))
    y = act_of(act, z)
    if residual is not None:
        y = y + (residual.float() if live is None else torch.where(live[:, None], residual.float(), torch.zeros((), device=z.device)))
    return (y.to(dt), z.to(dt)) if save else y.to(dt)


def plain_linear_back(st, act):
    x, w, dy = st["x"], st["w"], st["dy"]
    E, dt = w.shape[0], x.dtype
    dz = dy.float() if act == "none" else dy.float() * act_slope(act, st["z"].float())
    if st["offsets"] is None:
        return {"dx": (dz @ w[0].float()).to(dt), "dw": (dz.t() @ x.float())[None].to(dt), "db": dz.sum(0)[None]}
    at, is_row, e, slot, live = padded(st, E)
    dzp = torch.where(is_row[:, :, None], dz[at], torch.zeros((), device=dz.device))
    xp = x[st["rows"].long()[at]].float()
    dx = torch.bmm(dzp, w.float())[e, slot]
    dx = torch.where(live[:, None], dx, torch.zeros((), device=dx.device))
    return {"dx": dx.to(dt), "dw": torch.bmm(dzp.transpose(1, 2), xp).to(dt), "db": dzp.sum(1)}


def plain_combine(y, place, weights, offsets, residual):
    p = place.long()
    live = p < offsets[-1]
    rows = y[p].float() * torch.where(live, weights, torch.zeros((), device=y.device))[:, :, None]
    out = rows.sum(1)
    return (out if residual is None else out + residual.float()).to(y.dtype)


def plain_combine_back(st):
    y, p, w, dout = st["y"], st["place"].long(), st["weights"], st["dout"].float()
    live = p < st["offsets"][-1]
    zero = torch.zeros((), device=y.device)
    dw = torch.where(live, (y[p].float() * dout[:, None, :]).sum(2), zero)
    dy = torch.empty_like(y)
    dy[p.view(-1)] = (torch.where(live, w, zero)[:, :, None] * dout[:, None, :]).to(y.dtype).view(-1, y.shape[1])
    return {"dy": dy, "dweights": dw}


def plain(st):
    c = st["case"]
    op = c["op"]
    if op == "route":
        ids, w = plain_route(c, st["logits"], st["bias"])
        rows, place, offsets = order_of(ids, c["experts"])
        return {"ids": ids, "weights": w, "rows": rows, "place": place, "offsets": offsets}
    if op == "route_back":
        l, ids, dw = st["logits"].float(), st["ids"].long(), st["dweights"] * c["scale"]
        s = torch.sigmoid(l) if c["score"] == "sigmoid" else torch.softmax(l, 1)
        sel = s.gather(1, ids)
        if c["renorm"]:
            S = sel.sum(1, keepdim=True)
            dw = (dw - (dw * sel).sum(1, keepdim=True) / S) / S
        ds = torch.zeros_like(s).scatter(1, ids, dw)
        dl = ds * s * (1 - s) if c["score"] == "sigmoid" else s * (ds - (ds * s).sum(1, keepdim=True))
        return dl.to(st["logits"].dtype)
    if op == "linear":
        r = plain_linear(st, st["x"], st["w"], st["b"], c["act"], st["rows"], st["r"], c["save"])
        return {"y": r[0], "z": r[1]} if c["save"] else r
    if op == "linear_back":
        return plain_linear_back(st, c["act"])
    if op == "combine":
        return plain_combine(st["y"], st["place"], st["weights"], st["offsets"], st["r"])
    if op == "combine_back":
        return plain_combine_back(st)
    ids, w = plain_route(c, st["logits"], st["bias"])
    rows, place, offsets = order_of(ids, c["experts"])
    s2 = dict(rows=rows, offsets=offsets, most=int((offsets[1:] - offsets[:-1]).max()))
    h = plain_linear(s2, st["x"].float(), st["w1"], st["b1"], c["act"], rows, None, False)
    y = plain_linear(s2, h, st["w2"], st["b2"], "none", None, None, False)
    return {"out": plain_combine(y, place, w, offsets, st["x"]).to(st["x"].dtype), "weights": w}


# ---------------------------------------------------------------- one pass

def run(st):
    if not own:
        return plain(st)
    from paper_2608_27888_gb300 import ntc
    c = st["case"]
    op = c["op"]
    how = dict(score=c["score"], renormalize=c["renorm"], scale=c["scale"])
    pick = dict(how, bias=st.get("bias"), groups=c["groups"], top_groups=c["top_groups"])
    if op == "route":
        ids, w = ntc.route(st["logits"], c["top_k"], **pick)
        rows, place, offsets = ntc.expert_order(ids, c["experts"])
        return {"ids": ids, "weights": w, "rows": rows, "place": place, "offsets": offsets}
    if op == "route_back":
        return ntc.route_backward(st["logits"], st["ids"], st["dweights"], **how)
    if op == "linear":
        r = ntc.linear(st["x"], st["w"], st["b"], rows=st["rows"], offsets=st["offsets"], activation=c["act"],
                       leaky_slope=SLOPE, residual=st["r"], save=c["save"])
        return {"y": r[0], "z": r[1]} if c["save"] else r
    if op == "linear_back":
        dx, dw, db = ntc.linear_backward(st["dy"], st["x"], st["w"], z=st["z"], rows=st["rows"],
                                         offsets=st["offsets"], activation=c["act"], leaky_slope=SLOPE)
        return {"dx": dx, "dw": dw, "db": db}
    if op == "combine":
        return ntc.combine(st["y"], st["place"], st["weights"], st["offsets"], residual=st["r"])
    if op == "combine_back":
        dy, dw = ntc.combine_backward(st["dout"], st["y"], st["place"], st["weights"], st["offsets"])
        return {"dy": dy, "dweights": dw}
    ids, w = ntc.route(st["logits"], c["top_k"], **pick)
    rows, place, offsets = ntc.expert_order(ids, c["experts"])
    h = ntc.linear(st["x"], st["w1"], st["b1"], rows=rows, offsets=offsets, activation=c["act"], leaky_slope=SLOPE)
    y = ntc.linear(h, st["w2"], st["b2"], offsets=offsets)
    return {"out": ntc.combine(y, place, w, offsets, residual=st["x"]), "weights": w}


# ------------------------------------------------------------- the true values

def exact_act(a, z):
    if a == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if a == "leaky":
        return torch.where(z > 0, z, z * SLOPE)
    if a == "gelu":
        return z * torch.special.ndtr(z)
    if a == "silu":
        return z / (1 + torch.exp(-z))
    return z


def exact_slope(a, z):
    if a == "none":
        return torch.ones_like(z)
    if a in ("relu", "leaky"):
        return torch.where(z > 0, 1.0, 0.0 if a == "relu" else SLOPE)
    if a == "gelu":
        return torch.special.ndtr(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    s = 1 / (1 + torch.exp(-z))
    return s + z * s * (1 - s)


def segments(st, E, n):
    """(expert, first row, one past its last row), and how many rows have an expert."""
    if st["offsets"] is None:
        return [(0, 0, n)], n
    o = st["offsets"].tolist()
    return [(e, o[e], o[e + 1]) for e in range(E) if o[e + 1] > o[e]], o[E]


def exact_product(st, x, w, b, rows):
    n = x.shape[0] if rows is None else rows.shape[0]
    z = torch.zeros(n, w.shape[1], dtype=torch.float64, device=x.device)
    seg, live = segments(st, w.shape[0], n)
    for e, a, o in seg:
        src = x[a:o] if rows is None else x[rows[a:o].long()]
        z[a:o] = src.double() @ w[e].double().t() + b[e].double()
    return z, live


def exact_scores(c, l):
    return 1 / (1 + torch.exp(-l)) if c["score"] == "sigmoid" else torch.exp(l - torch.logsumexp(l, 1, keepdim=True))


def exact_weights(c, logits, bias):
    s = exact_scores(c, logits.double())
    ids = choices(c, logits.double(), bias)[2][:, :c["top_k"]]
    w = torch.take_along_dim(s, ids, 1)
    return ids.to(torch.int32), c["scale"] * (w / w.sum(1, keepdim=True) if c["renorm"] else w)


def exact(case, seed):
    c = full(case)
    op = c["op"]
    work_ = work(case)["flops"]
    if work_ > 6e12:  # 64-bit products at about 1 TFLOP/s
        return None
    st = prepare(case, seed)
    E = c["experts"]
    if op == "route":
        return {"ids": None, "weights": exact_weights(c, st["logits"], st["bias"])[1], "rows": None, "place": None,
                "offsets": None}
    if op == "route_back":
        l = st["logits"].double()
        ids, dw = st["ids"].long(), st["dweights"].double() * c["scale"]
        s = exact_scores(c, l)
        sel = torch.take_along_dim(s, ids, 1)
        if c["renorm"]:
            p = sel / sel.sum(1, keepdim=True)
            dw = (dw - (dw * p).sum(1, keepdim=True)) / sel.sum(1, keepdim=True)
        if c["score"] == "sigmoid":
            return torch.zeros_like(l).scatter(1, ids, dw * sel * (1 - sel))
        return torch.zeros_like(l).scatter(1, ids, sel * dw) - s * (sel * dw).sum(1, keepdim=True)
    if op == "linear":
        z, live = exact_product(st, st["x"], st["w"], st["b"], st["rows"])
        y = exact_act(c["act"], z)
        if st["r"] is not None:
            y[:live] += st["r"][:live].double()
        return {"y": y, "z": z} if c["save"] else y
    if op == "linear_back":
        x, w = st["x"], st["w"]
        n = st["dy"].shape[0]
        rows = st["rows"].long() if st["rows"] is not None else torch.arange(n, device=x.device)
        dx = torch.zeros(n, w.shape[2], dtype=torch.float64, device=x.device)
        dw = torch.zeros(w.shape, dtype=torch.float64, device=x.device)
        db = torch.zeros(w.shape[:2], dtype=torch.float64, device=x.device)
        for e, a, o in segments(st, E, n)[0]:
            dz = st["dy"][a:o].double()
            if c["act"] != "none":
                dz = dz * exact_slope(c["act"], st["z"][a:o].double())
            dx[a:o] = dz @ w[e].double()
            dw[e] = dz.t() @ x[rows[a:o]].double()
            db[e] = dz.sum(0)
        return {"dx": dx, "dw": dw, "db": db}
    if op == "combine":
        live = int(st["offsets"][-1])
        y, p = st["y"], st["place"].long()
        out = torch.zeros(y.shape[0] // c["top_k"], y.shape[1], dtype=torch.float64, device=y.device)
        for j in range(c["top_k"]):
            m = p[:, j] < live
            out[m] += st["weights"][m, j, None].double() * y[p[m, j]].double()
        return out if st["r"] is None else out + st["r"].double()
    if op == "combine_back":
        live = int(st["offsets"][-1])
        y, p, d = st["y"], st["place"].long(), st["dout"].double()
        dy = torch.zeros(y.shape, dtype=torch.float64, device=y.device)
        dw = torch.zeros(p.shape, dtype=torch.float64, device=y.device)
        for j in range(c["top_k"]):
            m = p[:, j] < live
            dy[p[m, j]] = st["weights"][m, j, None].double() * d[m]
            dw[m, j] = torch.einsum("td,td->t", d[m], y[p[m, j]].double())
        return {"dy": dy, "dweights": dw}
    ids, w = exact_weights(c, st["logits"], st["bias"])
    x = st["x"].double()
    out = x.clone()
    for e in range(E):
        t, j = (ids == e).nonzero(as_tuple=True)
        if t.numel():
            h = exact_act(c["act"], x[t] @ st["w1"][e].double().t() + st["b1"][e].double())
            out.index_add_(0, t, w[t, j][:, None] * (h @ st["w2"][e].double().t() + st["b2"][e].double()))
    return {"out": out, "weights": w}


# ------------------------------------------------------------------- its work

def work(case):
    """Bytes and operations of one pass: every input read once, every output written once."""
    c = full(case)
    T, E, k, op = c["tokens"], c["experts"], c["top_k"], c["op"]
    size = 4 if c["dtype"] == "fp32" else 2
    n = T * k
    order = 8 * n + 4 * (E + 1)
    if op == "route":
        return {"bytes": T * E * size + (4 * E if c["bias"] else 0) + 8 * n + order, "flops": 8 * T * E}
    if op == "route_back":
        return {"bytes": 2 * T * E * size + 8 * n, "flops": 10 * T * E}
    live = n * (1 - c["padding"])
    hit = E * (1 - (1 - min(1.0, k / E)) ** (T * (1 - c["padding"])))  # experts that some token takes
    N, K = c["d_out"], c["d_in"]
    index = 0 if E == 1 else 4 * n + 4 * (E + 1)
    if op == "linear":
        b = T * K * size + hit * (N * K * size + 4 * N) + n * N * size * (1 + c["residual"] + c["save"]) + index
        return {"bytes": b, "flops": 2 * live * N * K}
    if op == "linear_back":
        b = T * K * size + hit * N * K * size + n * N * size * (1 + (c["act"] != "none")) + n * K * size
        return {"bytes": b + E * (N * K * size + 4 * N) + index, "flops": 4 * live * N * K}
    if op == "combine":
        return {"bytes": (live * N + T * N * (1 + c["residual"])) * size + 8 * n, "flops": 2 * live * N}
    if op == "combine_back":
        return {"bytes": (live + T + n) * N * size + 12 * n, "flops": 3 * live * N}
    b = T * E * size + T * K * size * 2 + hit * (2 * N * K * size + 4 * (N + K)) + 4 * n
    return {"bytes": b, "flops": 4 * live * N * K}
