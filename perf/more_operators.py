"""Performance cases of training and serving a layer of routed experts.

Beside the router, the experts' products and their blend: the loss that spreads the
tokens over the experts, with its gradient; the optimizer's step over all parameters
at once; and the experts' weights in 4 bits, made, read back and multiplied.

``op`` of a case names the call:
  balance       loss, counts and mean probabilities of a batch's logits and choices
  balance_back  the gradient of the logits, added to the one that they have already
  adamw         one step over the parameters of `layers` routed layers, moments in 32 or in 8 bits
  linear4       one product of every expert's 4-bit weights with its rows (or a dense one, experts=1)
  pack4         weights to 4 bits with a scale for each group, and back

``exact()`` evaluates the definitions in 64 bits: gradients by autograd, products
expert by expert.
"""
import math

import torch

own = False

DTYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}

# Every field of a case, with the value it has when a case does not name it.
DEFAULTS = dict(
    op="linear4", tokens=1, experts=1, top_k=1, dtype="bf16",
    padding=0.0,  # share of the tokens that are padding: no expert takes them
    # balance loss
    score="softmax", masked=0.0, residual=False,
    # products and weights: width in, width out, weights of a scale
    d_in=0, d_out=0, group=128, act="none",
    # optimizer: routed layers d_in -> hidden -> d_out; masters: fp32 parameters with 16-bit copies of the matrices
    layers=1, hidden=0, bits=32, masters=True,
)


def full(case):
    return dict(DEFAULTS, **{k: v for k, v in case.items() if k != "name"})


def listed():
    return [
        # one micro-batch of a small router: launches and latency are the whole cost
        dict(name="balance-step", op="balance", tokens=512, experts=60, top_k=4, dtype="fp32"),
        # a training batch through a large router, sigmoid scores, a twentieth of the tokens padding
        dict(name="balance-train", op="balance", tokens=65536, experts=256, top_k=8, score="sigmoid", padding=0.05),
        # its gradient, added to the router's own
        dict(name="balance-back-train", op="balance_back", tokens=32768, experts=128, top_k=8, masked=0.02, residual=True),
        # the parameters of a small distilled layer (widths of a texture decoder): six tensors, latency
        dict(name="adamw-decoders", op="adamw", layers=1, experts=8, d_in=16, hidden=128, d_out=9),
        # a training step's parameters: fp32 masters, bf16 gradients and copies
        dict(name="adamw-train", op="adamw", layers=2, experts=8, d_in=2048, hidden=2048, d_out=2048),
        # widths that end inside a block, moments in 8 bits
        dict(name="adamw-train-8bit", op="adamw", layers=4, experts=7, d_in=1111, hidden=2049, d_out=999, bits=8),
        # one token through its 8 experts: the weights' bytes are the cost
        dict(name="linear4-token", op="linear4", tokens=1, experts=64, top_k=8, d_in=2048, d_out=1024, act="silu"),
        # a serving step of 64 sequences, a few rows per expert, padding slots in the batch
        dict(name="linear4-step", op="linear4", tokens=64, experts=32, top_k=4, d_in=1024, d_out=2048, dtype="fp16",
             group=64, act="gelu", residual=True, padding=0.125),
        # a dense layer whose sizes fit no tile, no group and no vector load
        dict(name="linear4-dense-odd", op="linear4", tokens=13, d_in=771, d_out=1027, dtype="fp16", group=32, act="leaky",
             residual=True),
        # a prefill chunk: arithmetic counts, too
        dict(name="linear4-prefill", op="linear4", tokens=1024, experts=16, top_k=2, d_in=2048, d_out=2048, group=128),
        # the experts' weights of a layer made ready to serve, and read back
        dict(name="pack4-experts", op="pack4", experts=32, d_in=1024, d_out=2048, group=64),
        # rows that end inside a group and inside a byte
        dict(name="pack4-odd", op="pack4", experts=3, d_in=771, d_out=1027, dtype="fp16", group=32),
    ]


def draw(rng):
    def logu(lo, hi):
        return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))

    def width(lo, hi):  # half of them multiples of 64, the others as they fall
        w = logu(lo, hi)
        return max(lo, w // 64 * 64) if rng.random() < 0.5 else w

    op = rng.choice(["balance", "balance_back", "adamw", "adamw", "linear4", "linear4", "linear4", "pack4"])
    c = dict(op=op, dtype=rng.choice(["bf16", "fp16"]))
    if op in ("balance", "balance_back"):
        c["dtype"] = rng.choice(["fp32", "bf16", "fp16"])
        c["experts"] = logu(4, 1024)
        c["tokens"] = logu(1, max(1, min(65536, (1 << 24) // c["experts"])))
        c["top_k"] = rng.randint(1, min(10, c["experts"] - 1))
        c["score"] = rng.choice(["softmax", "sigmoid"])
        c["padding"] = rng.choice([0.0, 0.1]) if c["tokens"] >= 64 else 0.0
        c["masked"] = rng.choice([0.0, 0.05]) if c["experts"] > 32 else 0.0
        c["residual"] = op == "balance_back" and rng.random() < 0.5
        return c
    if op == "adamw":
        c["layers"] = rng.randint(1, 12)
        c["experts"] = logu(1, 32)
        c["d_in"], c["hidden"], c["d_out"] = width(8, 2048), width(16, 4096), width(3, 2048)
        while c["layers"] * c["experts"] * c["hidden"] * (c["d_in"] + c["d_out"]) > 1 << 26:
            c["experts"], c["hidden"] = max(1, c["experts"] // 2), max(16, c["hidden"] * 3 // 4)
        c["bits"] = rng.choice([32, 8])
        c["masters"] = rng.random() < 0.7
        return c
    c["group"] = rng.choice([32, 64, 128])
    c["experts"] = 1 if rng.random() < 0.3 else logu(2, 64)
    c["d_in"], c["d_out"] = width(16, 4096), width(16, 4096)
    while c["experts"] * c["d_in"] * c["d_out"] > 1 << 26:
        c["experts"], c["d_out"] = max(1, c["experts"] // 2), max(16, c["d_out"] * 3 // 4)
    if op == "pack4":
        return c
    c["top_k"] = rng.randint(1, min(8, c["experts"]))
    per = 2.0 * c["top_k"] * c["d_in"] * c["d_out"]
    c["tokens"] = logu(1, int(max(1, min(1024, 1.6e10 / per))))
    c["act"] = rng.choice(["none", "relu", "leaky", "gelu", "silu"])
    c["residual"] = rng.random() < 0.4
    c["padding"] = 0.0 if c["experts"] == 1 else rng.choice([0.0, 0.1])
    return c


# ------------------------------------------------------------------ inputs

SLOPE = 0.01  # leaky activation
BETA1, BETA2, EPS, DECAY, RATE = 0.9, 0.999, 1e-8, 0.01, 1e-3
BLOCK = 256  # moments of a scale


def route_ids(c, g, dev):
    """top_k distinct experts per token, some experts more popular than others; padding tokens have -1."""
    T, E, k = c["tokens"], c["experts"], c["top_k"]
    noise = -torch.log(-torch.log(torch.rand(T, E, generator=g, device=dev).clamp(1e-7, 1 - 1e-7)))
    ids = (noise + 0.5 * torch.randn(E, generator=g, device=dev)).topk(k, dim=1).indices.to(torch.int32)
    if c["padding"]:
        ids[torch.rand(T, generator=g, device=dev) < c["padding"]] = -1
    return ids


def order_of(ids, E):
    """rows (token of each ordered entry) and offsets (first entry of each expert)."""
    key = torch.where((ids >= 0) & (ids < E), ids, E).view(-1).long()
    order = key.sort(stable=True).indices
    offsets = torch.searchsorted(key[order], torch.arange(E + 1, device=ids.device))
    return (order // ids.shape[1]).to(torch.int32), offsets.to(torch.int32)


def quantised(w, group, dtype):
    """Whole numbers -8..7 [..., K] and scales [..., ceil(K / group)] of weights w [..., K]."""
    K = w.shape[-1]
    G = -(-K // group)
    f = torch.zeros(w.shape[:-1] + (G * group,), device=w.device)
    f[..., :K] = w.float()
    f = f.view(w.shape[:-1] + (G, group))
    s = (f.abs().amax(-1) * (1.0 / 7.0)).to(dtype)
    at = s.float()[..., None]
    q = torch.where(at > 0, torch.round(f / at), torch.zeros_like(f)).clamp(-8, 7)
    return q.view(w.shape[:-1] + (G * group,))[..., :K], s


def packed(q):
    """Two numbers a byte, the even one in the low half, as q + 8; rows begin on 16 bytes."""
    K = q.shape[-1]
    n = -(-K // 2)
    u = torch.full(q.shape[:-1] + (-(-n // 16) * 32,), 8, dtype=torch.uint8, device=q.device)
    u[..., :K] = (q + 8).to(torch.uint8)
    return (u[..., 0::2] | (u[..., 1::2] << 4))[..., :n]


def unpacked(p, scales, K, group):
    """The weights in 32 bits."""
    q = torch.stack([p & 15, p >> 4], -1).flatten(-2)[..., :K].float() - 8.0
    return q * scales.float().repeat_interleave(group, -1)[..., :K]


def blocks_of(x):
    """A moment's blocks of BLOCK values, the last one filled with zeros."""
    n = x.numel()
    f = torch.zeros(-(-n // BLOCK) * BLOCK, device=x.device)
    f[:n] = x.reshape(-1)
    return f.view(-1, BLOCK)


def encoded(x, positive):
    """e4m3 values and the blocks' scales of a moment; a positive one that is not 0 stays so."""
    f = blocks_of(x)
    top = f.abs().amax(1, keepdim=True)
    top = torch.where(top < 2.0 ** -100, torch.zeros_like(top), top)
    y = f * torch.where(top > 0, torch.div(torch.full_like(top, 448.0), top), torch.zeros_like(top))
    if positive:
        y = torch.where(y > 0, y.clamp_min(2.0 ** -9), y)
    code = y.to(torch.float8_e4m3fn).view(-1)[:x.numel()].view(x.shape)
    return code, (top * (1.0 / 448.0)).view(-1)


def decoded(code, scale):
    f = blocks_of(code.float()) * scale[:, None]
    return f.view(-1)[:code.numel()].view(code.shape)


def shapes_of(c):
    """The optimizer's tensors: router, its bias, the two matrices of every expert and their biases."""
    E, D, H, O = c["experts"], c["d_in"], c["hidden"], c["d_out"]
    return [(E, D), (E,), (E, H, D), (E, H), (E, O, H), (E, O)] * c["layers"]


def prepare(case, seed):
    c = full(case)
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(seed)
    dt = DTYPES[c["dtype"]]
    T, E, k, op = c["tokens"], c["experts"], c["top_k"], c["op"]

    def normal(*shape, std=1.0, dtype=None):
        return (torch.randn(*shape, generator=g, device=dev) * std).to(dtype or dt)

    st = dict(case=c)
    if op in ("balance", "balance_back"):
        l = normal(T, E, dtype=torch.float32) + 0.5 * normal(E, dtype=torch.float32)
        if c["masked"]:
            l[torch.rand(T, E, generator=g, device=dev) < c["masked"]] = -math.inf
        st["ids"] = l.topk(k, dim=1).indices.to(torch.int32)
        if c["padding"]:  # a padding token has no choice, and often no logit
            out = torch.rand(T, generator=g, device=dev) < c["padding"]
            st["ids"][out] = -1
            l[out & (torch.rand(T, generator=g, device=dev) < 0.5)] = -math.inf
        st["logits"] = l.to(dt)
        if op == "balance_back":
            st["counts"] = counts_of(st["ids"], E)
            scale = 0.1 * (65536 if c["dtype"] == "fp16" else 1)  # fp16 trains with its loss scaled
            st["dloss"] = torch.rand(1, generator=g, device=dev)[0] * scale + scale
            st["dlogits"] = normal(T, E, std=scale / (T * E)) if c["residual"] else None
    elif op == "adamw":
        # every kind of tensor in one buffer, as an optimizer keeps them, each tensor from a block's start on
        shapes = shapes_of(c)
        n = sum(-(-math.prod(s) // BLOCK) * BLOCK for s in shapes)
        eight, pt = c["bits"] == 8, torch.float32 if c["masters"] else dt
        flat = {"m": torch.zeros(n, device=dev), "v": torch.zeros(n, device=dev), "weights": torch.zeros(n, dtype=pt, device=dev),
                "vectors": torch.zeros(n, device=dev), "copies": torch.zeros(n, dtype=dt, device=dev) if c["masters"] else None}
        st.update(flat=flat, params=[], grads=[], copies=[], m=[], v=[], scales=[], step=100)
        at = 0
        for s in shapes:
            matrix = len(s) == 3
            size = torch.exp(normal(*s[-1:], dtype=torch.float32)) * 1e-3  # gradients differ from column to column
            here = slice(at, at + math.prod(s))
            p = flat["weights" if matrix else "vectors"][here].view(s)
            p.copy_(normal(*s, std=0.05, dtype=torch.float32))
            st["params"].append(p)
            st["copies"].append(flat["copies"][here].view(s).copy_(p) if c["masters"] and matrix else None)
            st["grads"].append((normal(*s, dtype=torch.float32) * size).to(dt if matrix else torch.float32))
            flat["m"][here].view(s).copy_(normal(*s, dtype=torch.float32) * size * 0.3)
            flat["v"][here].view(s).copy_((normal(*s, dtype=torch.float32).abs() + 0.05) * size)
            at += -(-math.prod(s) // BLOCK) * BLOCK
        if eight:
            (flat["m"], a), (flat["v"], b) = encoded(flat["m"], False), encoded(flat["v"], True)
            flat["scales"] = torch.stack([a, b])
        else:
            flat["v"].square_()
        at = 0
        for s in shapes:
            here = slice(at, at + math.prod(s))
            st["m"].append(flat["m"][here].view(s))
            st["v"].append(flat["v"][here].view(s))
            if eight:
                st["scales"].append(flat["scales"][:, at // BLOCK:at // BLOCK - -math.prod(s) // BLOCK])
            at += -(-math.prod(s) // BLOCK) * BLOCK
    else:
        N, K = c["d_out"], c["d_in"]
        w = normal(E, N, K, std=K ** -0.5)
        if op == "pack4":
            st["w"] = w
            return st
        q, st["scales"] = quantised(w, c["group"], dt)
        st["packed"] = packed(q)
        st["x"] = normal(T, K)
        st["b"] = normal(E, N, std=0.1, dtype=torch.float32)
        st["rows"] = st["offsets"] = None
        if E > 1:
            st["rows"], st["offsets"] = order_of(route_ids(c, g, dev), E)
            # the largest number of rows of one expert: what a padded batch is sized by
            st["most"] = int((st["offsets"][1:] - st["offsets"][:-1]).max())
        st["r"] = normal(T * k, N) if c["residual"] else None
    return st


# ------------------------------------------------------------- the plain form

def counts_of(ids, E):
    """Entries of each expert, and after them the tokens that have one."""
    live = (ids >= 0) & (ids < E)
    key = torch.where(live, ids, E).view(-1).long()
    n = torch.zeros(E + 1, dtype=torch.int32, device=ids.device)
    n.scatter_add_(0, key, torch.ones_like(key, dtype=torch.int32))
    n[E] = live.any(1).sum()
    return n


def probabilities(c, logits):
    """Scores of a token that sum to 1 (0 where no logit is left), and a sigmoid's slope over its value."""
    l = logits.float()
    dead = l == -math.inf
    top = l.amax(1, keepdim=True)
    if c["score"] == "softmax":
        s = torch.where(dead, torch.zeros_like(l), torch.exp(l - torch.where(top == -math.inf, torch.zeros_like(top), top)))
        slope = None
    else:
        s, slope = torch.sigmoid(l), torch.sigmoid(-l)
    sum_ = s.sum(1, keepdim=True)
    return torch.where(sum_ > 0, s / sum_, torch.zeros_like(s)), slope


def plain_balance(st):
    c, ids = st["case"], st["ids"]
    E = c["experts"]
    p, _ = probabilities(c, st["logits"])
    n = counts_of(ids, E)
    live = ((ids >= 0) & (ids < E)).any(1, keepdim=True)
    total = torch.where(live, p, torch.zeros_like(p)).sum(0, dtype=torch.float64)
    tokens = n[E].double().clamp_min(1)
    f = n[:E].double() / n[:E].double().sum().clamp_min(1)
    return {"loss": (E * (f * total).sum() / tokens).float(), "counts": n, "mean": (total / tokens).float()}


def plain_balance_back(st):
    c, ids, n = st["case"], st["ids"], st["counts"].float()
    E = c["experts"]
    p, slope = probabilities(c, st["logits"])
    live = ((ids >= 0) & (ids < E)).any(1, keepdim=True)
    a = st["dloss"] * E / (n[E].clamp_min(1) * n[:E].sum().clamp_min(1))
    n = n[:E] - n[p.argmax(1)][:, None]  # differences: their mean keeps its digits where one p is near 1
    d = a * p * (n - (p * n).sum(1, keepdim=True))
    d = torch.where(live, d if slope is None else d * slope, torch.zeros_like(d))
    return (d if st["dlogits"] is None else d + st["dlogits"].float()).to(st["logits"].dtype)


def plain_step(st, i):
    """One tensor's step; every operation is rounded to 32 bits, the parameter and the moments once more where they are held in less."""
    p, g, m, v, copy = (st[n][i] for n in ("params", "grads", "m", "v", "copies"))
    bits8, t = st["case"]["bits"] == 8, st["step"]
    f = g.float()
    m0, v0 = m, v
    if bits8:
        s = st["scales"][i]
        m0, v0 = decoded(m, s[0]), decoded(v, s[1])
        v0 = v0 * v0
    m1 = m0 * BETA1 + f * (1 - BETA1)
    v1 = v0 * BETA2 + (f * (1 - BETA2)) * f
    root = torch.sqrt(v1)
    down = root * (1 / math.sqrt(1 - BETA2 ** t)) + EPS
    p1 = p.float() * (1 - RATE * DECAY) - torch.div(m1 * (RATE / (1 - BETA1 ** t)), down)
    p.copy_(p1)
    if copy is not None:
        copy.copy_(p1)
    if bits8:
        m1, a = encoded(m1, False)
        v1, b = encoded(root, True)
        s.copy_(torch.stack([a, b]))
    m.copy_(m1)
    v.copy_(v1)


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


def plain_linear4(st):
    c, x, rows, off = st["case"], st["x"], st["rows"], st["offsets"]
    E, K, group = c["experts"], c["d_in"], c["group"]
    if off is None:
        z = x.float() @ unpacked(st["packed"][0], st["scales"][0], K, group).t() + st["b"][0]
        live = None
    else:
        off = off.long()
        n = rows.shape[0]
        i = torch.arange(n, device=x.device)
        e = torch.bucketize(i, off[1:], right=True)
        live = (e < E)[:, None]
        e = e.clamp_max(E - 1)
        if n <= E:  # few rows: only the weights that they need
            w = unpacked(st["packed"][e], st["scales"][e], K, group)
            z = torch.bmm(w, x[rows.long()].float()[:, :, None])[:, :, 0] + st["b"][e]
        else:  # every expert's rows in a padded batch
            at = (off[:-1, None] + torch.arange(st["most"], device=x.device)).clamp_max(n - 1)
            w = unpacked(st["packed"], st["scales"], K, group)
            z = torch.bmm(x[rows.long()[at]].float(), w.transpose(1, 2)) + st["b"][:, None, :]
            z = z[e, (i - off[e]).clamp(0, st["most"] - 1)]
    y = act_of(c["act"], z)
    if st["r"] is not None:
        y = y + st["r"].float()
    return (y if live is None else torch.where(live, y, torch.zeros_like(y))).to(x.dtype)


def plain(st):
    c = st["case"]
    op = c["op"]
    if op == "balance":
        return plain_balance(st)
    if op == "balance_back":
        return plain_balance_back(st)
    if op == "adamw":
        _ = [plain_step(st, i) for i in range(len(st["params"]))]
        return st["flat"]
    if op == "linear4":
        return plain_linear4(st)
    q, s = quantised(st["w"], c["group"], st["w"].dtype)
    return {"scales": s, "w": unpacked(packed(q), s, c["d_in"], c["group"]).to(st["w"].dtype)}


# ---------------------------------------------------------------- one pass

def run(st):
    c = st["case"]
    op = c["op"]
    if op == "adamw":
        st["step"] += 1
    if not own:
        return plain(st)
    from paper_2608_27888_gb300 import ntc
    if op == "balance":
        loss, counts, mean = ntc.balance_loss(st["logits"], st["ids"], score=c["score"])
        return {"loss": loss, "counts": counts, "mean": mean}
    if op == "balance_back":
        return ntc.balance_loss_backward(st["logits"], st["ids"], st["counts"], dloss=st["dloss"],
                                         residual=st["dlogits"], score=c["score"])
    if op == "adamw":
        ntc.adamw(st["params"], st["grads"], st["m"], st["v"], scales=st["scales"] or None, copies=st["copies"],
                  step=st["step"], lr=RATE, beta1=BETA1, beta2=BETA2, eps=EPS, weight_decay=DECAY)
        return st["flat"]
    if op == "linear4":
        return ntc.linear4(st["x"], st["packed"], st["scales"], st["b"], group=c["group"], rows=st["rows"],
                           offsets=st["offsets"], activation=c["act"], leaky_slope=SLOPE, residual=st["r"])
    p, s = ntc.pack4(st["w"], group=c["group"])
    return {"scales": s, "w": ntc.unpack4(p, s, c["d_in"], group=c["group"])}


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


def exact_balance(c, st, logits):
    """The loss and the mean probabilities as a differentiable function of 64-bit logits."""
    E, ids = c["experts"], st["ids"].long()
    here = (ids[:, :, None] == torch.arange(E, device=ids.device)).any(1) if ids.numel() * E < 1 << 27 else \
        torch.zeros(ids.shape[0], E + 1, dtype=torch.bool, device=ids.device).scatter_(1, ids.clamp_min(-1) % (E + 1), True)[:, :E]
    token = here.any(1)
    l = logits[token]
    s = torch.sigmoid(l) if c["score"] == "sigmoid" else torch.exp(l - torch.logsumexp(l, 1, keepdim=True))
    p = s / s.sum(1, keepdim=True)
    share = here.sum(0).double() / here.sum().clamp_min(1)  # a token's ids are distinct
    mean = p.sum(0) / token.sum().clamp_min(1)
    return E * (share * mean).sum(), mean


def exact(case, seed):
    c = full(case)
    op = c["op"]
    st = prepare(case, seed)
    if op == "balance":
        loss, mean = exact_balance(c, st, st["logits"].double())
        return {"loss": loss, "counts": None, "mean": mean}
    if op == "balance_back":
        l = st["logits"].double().requires_grad_()
        d = torch.autograd.grad(exact_balance(c, st, l)[0], l)[0] * st["dloss"].double()
        return d if st["dlogits"] is None else d + st["dlogits"].double()
    if op == "adamw":
        t, eight, flat = st["step"] + 1, c["bits"] == 8, st["flat"]
        out = {n: None if f is None or n == "scales" else f.double() for n, f in flat.items()}
        at = 0
        for i, shape in enumerate(shapes_of(c)):
            n = math.prod(shape)
            here = slice(at, at + n)
            p, g, m, v = (st[x][i].double().flatten() for x in ("params", "grads", "m", "v"))
            if eight:
                a, b = (s.double().repeat_interleave(BLOCK)[:n] for s in st["scales"][i])
                m, v = m * a, (v * b) ** 2
            m = BETA1 * m + (1 - BETA1) * g
            v = BETA2 * v + (1 - BETA2) * g ** 2
            p = p - RATE * DECAY * p - RATE * (m / (1 - BETA1 ** t)) / ((v / (1 - BETA2 ** t)).sqrt() + EPS)
            out["m"][here], out["v"][here] = m, v
            out["weights" if len(shape) == 3 else "vectors"][here] = p
            if st["copies"][i] is not None:
                out["copies"][here] = p
            at += -(-n // BLOCK) * BLOCK
        if eight:  # a moment next to the border of two codes may have either: it has no value of its own
            out["m"] = out["v"] = None
        return out
    if op == "pack4":
        w = st["w"].double()
        K, G = c["d_in"], c["group"]
        n = -(-K // G)
        lines = torch.nn.functional.pad(w, (0, n * G - K)).unflatten(-1, (n, G))
        s = (lines.abs().max(-1).values / 7).to(st["w"].dtype).double()
        at = s.repeat_interleave(G, -1)[..., :K]
        q = torch.where(at == 0, 0.0, w / at).round().clamp(-8, 7)
        return {"scales": s, "w": q * at}
    if work(case)["flops"] > 6e12:  # 64-bit products at about 1 TFLOP/s
        return None
    x, r, K = st["x"], st["r"], c["d_in"]
    o = [0, x.shape[0]] if st["offsets"] is None else st["offsets"].tolist()
    n = x.shape[0] if st["rows"] is None else st["rows"].shape[0]
    y = torch.zeros(n, c["d_out"], dtype=torch.float64, device=x.device)
    for e in range(c["experts"]):
        a, b = o[e], o[e + 1]
        if b > a:
            q = torch.empty(c["d_out"], 2 * st["packed"].shape[-1], dtype=torch.float64, device=x.device)
            q[:, 0::2], q[:, 1::2] = st["packed"][e] % 16, st["packed"][e] // 16
            w = (q[:, :K] - 8) * st["scales"][e].double()[:, torch.arange(K, device=x.device) // c["group"]]
            src = x[a:b] if st["rows"] is None else x[st["rows"][a:b].long()]
            y[a:b] = exact_act(c["act"], src.double() @ w.t() + st["b"][e].double())
            if r is not None:
                y[a:b] += r[a:b].double()
    return y


# ------------------------------------------------------------------- its work

def work(case):
    """Bytes and operations of one pass: every input read once, every output written once."""
    c = full(case)
    T, E, k, op = c["tokens"], c["experts"], c["top_k"], c["op"]
    size = 4 if c["dtype"] == "fp32" else 2
    if op == "balance":
        return {"bytes": T * E * size + 4 * T * k + 8 * E + 8, "flops": 6 * T * E}
    if op == "balance_back":
        return {"bytes": T * E * size * (2 + c["residual"]) + 4 * T * k + 4 * E + 8, "flops": 10 * T * E}
    if op == "adamw":
        D, H, O, L = c["d_in"], c["hidden"], c["d_out"], c["layers"]
        big, small = L * E * H * (D + O), L * E * (D + 1 + H + O)
        state = 4 + 16 / BLOCK if c["bits"] == 8 else 16
        weight = (8 + 2 if c["masters"] else 4) + 2  # parameter read and written, the copy, the gradient
        return {"bytes": big * (weight + state) + small * (8 + 4 + state), "flops": 16 * (big + small)}
    N, K = c["d_out"], c["d_in"]
    if op == "pack4":
        return {"bytes": E * N * K * 2 * 2 + E * N * (K // 2 + 2 * -(-K // c["group"])), "flops": 6 * E * N * K}
    n = T * k
    live = n * (1 - c["padding"])
    hit = E * (1 - (1 - min(1.0, k / E)) ** (T * (1 - c["padding"])))  # experts that some token takes
    b = T * K * 2 + hit * N * (K / 2 + 2 * -(-K // c["group"]) + 4) + n * N * 2 * (1 + c["residual"])
    return {"bytes": b + (0 if E == 1 else 4 * n + 4 * (E + 1)), "flops": 2 * live * N * K}
