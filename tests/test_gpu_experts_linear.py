"""The experts' linear layers, their gradients and the blend against their plain 64-bit forms."""
import math

import pytest
import torch

import tests.experts_ref as R

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "fp16": torch.float16}


@pytest.fixture(scope="module")
def ntc():
    from paper_2608_27888_gb300 import ntc
    yield ntc
    ntc.ntc_linear_status(0)  # no kernel gave up a wait


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def normal(g, *shape, std=1.0, dtype=torch.float32):
    return (torch.randn(*shape, generator=g, device="cuda") * std).to(dtype)


def routed(g, T, E, k, drop=0.2):
    """Random ids with some dropped and some experts without rows, and their order."""
    ids = torch.rand(T, E, generator=g, device="cuda").topk(k, 1).indices.int()
    ids = torch.where(ids % 5 == 3, torch.full_like(ids, -1), ids)  # experts 3, 8, ... have no rows
    ids[torch.rand(T, generator=g, device="cuda") < drop] = -1
    return (ids,) + R.order(ids, E)


# tokens, in, out, experts, top_k: one token, one row per tile, tiles exactly full, sizes that fit nothing
SHAPES = [(1, 64, 64, 1, 1), (1, 8, 16, 4, 2), (2, 64, 128, 3, 1), (128, 64, 256, 1, 1), (129, 72, 130, 1, 1),
          (300, 200, 320, 4, 2), (77, 129, 61, 5, 3), (1, 1, 1, 1, 1), (260, 1000, 40, 7, 4), (64, 512, 2048, 32, 4),
          (1500, 96, 520, 2, 1), (40, 33, 700, 100, 8)]


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("T,K,N,E,k", SHAPES)
def test_linear_matches_the_definition(ntc, dtype, T, K, N, E, k):
    g = gen(T + K + N)
    dt = DT[dtype]
    x, w = normal(g, T, K, dtype=dt), normal(g, E, N, K, std=K ** -0.5, dtype=dt)
    b = normal(g, E, N)
    rows = offsets = None
    m = T
    if E > 1:
        _, rows, _, offsets = routed(g, T, E, k)
        m = T * k
    r = normal(g, m, N, dtype=dt)
    for act, bias, res, save in (("none", None, None, False), ("gelu", b, r, True), ("silu", b, None, True),
                                 ("relu", b, r, False), ("leaky", None, r, True)):
        y, z, yb, zb = R.linear(x, w, bias, rows, offsets, act, 0.05, res)
        got = ntc.linear(x, w, bias, rows=rows, offsets=offsets, activation=act, leaky_slope=0.05, residual=res, save=save)
        if save:
            R.assert_within(got[1], z, zb, "z " + act)
            got = got[0]
        if res is not None and offsets is not None:
            y[int(offsets[-1]):] = 0
        R.assert_within(got, y, yb, act)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("T,K,N,E,k", SHAPES)
@pytest.mark.parametrize("act", ["none", "gelu", "silu", "relu", "leaky"])
def test_linear_backward_matches_the_formula(ntc, dtype, T, K, N, E, k, act):
    g = gen(T + K * N)
    dt = DT[dtype]
    x, w = normal(g, T, K, dtype=dt), normal(g, E, N, K, std=K ** -0.5, dtype=dt)
    rows = offsets = None
    m = T
    if E > 1:
        _, rows, _, offsets = routed(g, T, E, k)
        m = T * k
    z = None if act == "none" else normal(g, m, N, dtype=dt)
    dy = normal(g, m, N, dtype=dt)
    want = R.linear_backward(dy, x, w, z, rows, offsets, act)
    got = ntc.linear_backward(dy, x, w, z=z, rows=rows, offsets=offsets, activation=act)
    for name, a, (ref, bound) in zip(("dx", "dw", "db"), got, want):
        R.assert_within(a, ref, bound, name)
    if E > 1:  # experts without rows and rows without an expert: exact zeros
        assert (got[1][3::5] == 0).all() and (got[2][3::5] == 0).all()
        assert (got[0][int(offsets[-1]):] == 0).all()
    again = ntc.linear_backward(dy, x, w, z=z, rows=rows, offsets=offsets, activation=act)
    for a, c in zip(got, again):
        assert torch.equal(a, c)
    only = ntc.linear_backward(dy, x, w, z=z, rows=rows, offsets=offsets, activation=act, need=("dw",))
    assert only[0] is None and only[2] is None and torch.equal(only[1], got[1])


def test_linear_backward_matches_differences(ntc):
    """dw and dx against central differences of a 64-bit forward pass at the same operands."""
    g = gen(5)
    T, K, N, E, k = 6, 8, 8, 2, 1
    x, w, b = normal(g, T, K, dtype=torch.bfloat16), normal(g, E, N, K, dtype=torch.bfloat16), normal(g, E, N)
    ids = torch.tensor([[0], [1], [1], [0], [1], [-1]], dtype=torch.int32, device="cuda")
    rows, _, offsets = R.order(ids, E)
    dy = normal(g, T, N, dtype=torch.bfloat16)
    for act in ("gelu", "silu"):
        _, z = ntc.linear(x, w, b, rows=rows, offsets=offsets, activation=act, save=True)
        dx, dw, db = ntc.linear_backward(dy, x, w, z=z, rows=rows, offsets=offsets, activation=act)

        def loss(x, w, b):
            return (R.linear(x, w, b, rows, offsets, act)[0] * dy.double()).sum().item()
        h = 1e-5
        xd, wd, bd = x.double(), w.double(), b.double()
        R.UNIT[torch.float64], R.TINY[torch.float64] = 2.0 ** -53, 0.0
        # z was stored in bf16: the slope is off by up to |act''| <= 0.8 times 2^-8 |z|; dz and the results are rounded
        zr = 2.0 ** -8 * z.double().abs() * 0.8 * dy.double().abs()
        dz = dy.double().abs() * 1.2
        for e in range(E):
            a, o = int(offsets[e]), int(offsets[e + 1])
            for n, c in ((0, 0), (3, 5), (7, 7)):
                up, down = wd.clone(), wd.clone()
                up[e, n, c] += h
                down[e, n, c] -= h
                diff = (loss(xd, up, bd) - loss(xd, down, bd)) / (2 * h)
                xs = xd[rows[a:o].long(), c].abs()
                bound = float(((zr[a:o, n] + 2.0 ** -8 * dz[a:o, n]) * xs).sum()) + 2.0 ** -8 * abs(diff) + 1e-5
                assert abs(float(dw[e, n, c]) - diff) <= bound
            for n in (0, 6):
                up, down = bd.clone(), bd.clone()
                up[e, n] += h
                down[e, n] -= h
                diff = (loss(xd, wd, up) - loss(xd, wd, down)) / (2 * h)
                assert abs(float(db[e, n]) - diff) <= float(zr[a:o, n].sum()) + 1e-5
        per_token = ntc.combine(dx, torch.argsort(rows.long())[:, None].int(), None, offsets)
        for t, c in ((0, 0), (2, 5), (5, 1)):
            up, down = xd.clone(), xd.clone()
            up[t, c] += h
            down[t, c] -= h
            diff = (loss(up, wd, bd) - loss(down, wd, bd)) / (2 * h)
            i = int((rows == t).nonzero()[0])
            e = max(0, int(ids[t, 0]))
            bound = float(((zr[i] + 2.0 ** -8 * dz[i]) * wd[e, :, c].abs()).sum()) + 2.0 ** -7 * abs(diff) + 1e-5
            assert abs(float(per_token[t, c]) - diff) <= bound


@pytest.mark.parametrize("skip,pad", [(0, 8), (1, 0), (0, 3), (4, 4), (8, 8)])
def test_linear_strides_and_alignment(ntc, skip, pad):
    """Every operand as a view at odd addresses and strides; what lies between the rows is neither read nor written."""
    g = gen(skip * 10 + pad)
    T, K, N, E = 150, 100, 90, 3

    def view(t):
        shape = list(t.shape)
        big = torch.full(shape[:-1] + [shape[-1] + skip + pad], math.nan, dtype=t.dtype, device="cuda")
        big[..., skip:skip + shape[-1]] = t
        return big[..., skip:skip + shape[-1]]
    x, w = normal(g, T, K, dtype=torch.bfloat16), normal(g, E, N, K, std=0.1, dtype=torch.bfloat16)
    _, rows, _, offsets = routed(g, T, E, 2)
    r, dy, z = (normal(g, 2 * T, N, dtype=torch.bfloat16) for _ in range(3))
    y, _, yb, _ = R.linear(x, w, None, rows, offsets, "gelu", residual=r)
    got = ntc.linear(view(x), view(w), rows=rows, offsets=offsets, activation="gelu", residual=view(r))
    R.assert_within(got, y, yb)
    want = R.linear_backward(dy, x, w, z, rows, offsets, "gelu")
    got = ntc.linear_backward(view(dy), view(x), view(w), z=view(z), rows=rows, offsets=offsets, activation="gelu")
    for a, (ref, bound) in zip(got, want):
        R.assert_within(a, ref, bound)
    want = R.linear_backward(dy, x, w, None, rows, offsets, "none")
    got = ntc.linear_backward(view(dy), view(x), view(w), rows=rows, offsets=offsets)
    for a, (ref, bound) in zip(got, want):
        R.assert_within(a, ref, bound)


def test_outputs_of_any_stride_leave_the_rest_alone(ntc):
    """Through the C entry: y and z with wide rows at an odd address, their surroundings untouched."""
    g = gen(3)
    M, K, N = 70, 64, 50
    x, w = normal(g, M, K, dtype=torch.float16), normal(g, N, K, std=0.1, dtype=torch.float16)
    for skip, ld in ((0, 56), (3, 61), (8, 64)):
        y, z = (torch.full((M, ld), 5.0, dtype=torch.float16, device="cuda") for _ in range(2))
        d = ntc.ntc_linear_desc(ntc.NTC_TYPE_FP16, K, N, 1, 4, 0.0, M, M, K, K, N * K, ld, ld, N)
        ntc.ntc_linear(d, x.data_ptr(), None, None, w.data_ptr(), None, None, y.data_ptr() + 2 * skip,
                       z.data_ptr() + 2 * skip if ld - skip >= N else z.data_ptr(), None, 0,
                       torch.cuda.current_stream().cuda_stream)
        want, wz, yb, zb = R.linear(x, w, activation="silu")
        flat = y.view(-1)
        inside = torch.zeros_like(flat, dtype=torch.bool)
        at = (torch.arange(M, device="cuda")[:, None] * ld + skip + torch.arange(N, device="cuda")).view(-1)
        inside[at] = True
        R.assert_within(flat[at].view(M, N), want, yb)
        assert (flat[~inside] == 5).all()


def test_neighbours_do_not_leak(ntc):
    """NaN and infinity in one expert's rows, weights, bias and gradient stay in that expert."""
    g = gen(8)
    E, K, N = 3, 96, 160
    counts = [70, 45, 100]
    offsets = torch.tensor([0, 70, 115, 215], dtype=torch.int32, device="cuda")
    M = sum(counts) + 9  # nine rows of no expert, NaN as well
    x, dy, z, r = (normal(g, M, c, dtype=torch.bfloat16) for c in (K, N, N, N))
    w, b = normal(g, E, N, K, std=0.1, dtype=torch.bfloat16), normal(g, E, N)
    for t in (x, dy, z, r):
        t[70:115] = math.nan
        t[90] = math.inf
        t[215:] = math.nan
    w[1], b[1] = math.nan, math.inf
    clean = [t.clone() for t in (x, dy, z, r, w, b)]
    for t in clean[:4]:
        t[70:115] = 0
        t[215:] = 0
    clean[4][1] = 0
    clean[5][1] = 0
    cx, cdy, cz, cr, cw, cb = clean
    keep = torch.cat([torch.arange(70), torch.arange(115, 215)]).cuda()
    for rows in (None, torch.arange(M, dtype=torch.int32, device="cuda")):
        y = ntc.linear(x, w, b, rows=rows, offsets=offsets, activation="gelu", residual=r)
        want, _, yb, _ = R.linear(cx, cw, cb, rows, offsets, "gelu", residual=cr)
        R.assert_within(y[keep], want[keep], yb[keep])
        assert torch.isnan(y[70:115]).any() and (y[215:] == 0).all()
        dx, dw, db = ntc.linear_backward(dy, x, w, z=z, rows=rows, offsets=offsets, activation="gelu")
        (wx, bx), (ww, bw), (wb, bb) = R.linear_backward(cdy, cx, cw, cz, rows, offsets, "gelu")
        R.assert_within(dx[keep], wx[keep], bx[keep])
        assert (dx[215:] == 0).all()
        for e in (0, 2):
            R.assert_within(dw[e], ww[e], bw[e])
            R.assert_within(db[e], wb[e], bb[e])


def test_indices_outside_are_rows_of_zeros_and_offsets_are_clamped(ntc):
    g = gen(4)
    x, w, b = normal(g, 20, 64, dtype=torch.bfloat16), normal(g, 2, 64, 64, std=0.1, dtype=torch.bfloat16), normal(g, 2, 64)
    rows = torch.tensor([0, -1, 20, 19, 2 ** 31 - 1, -2 ** 31, 5, 6], dtype=torch.int32, device="cuda")
    offsets = torch.tensor([0, 4, 8], dtype=torch.int32, device="cuda")
    y, _, yb, _ = R.linear(x, w, b, rows, offsets)
    R.assert_within(ntc.linear(x, w, b, rows=rows, offsets=offsets), y, yb)
    dy = normal(g, 8, 64, dtype=torch.bfloat16)
    for a, (ref, bound) in zip(ntc.linear_backward(dy, x, w, rows=rows, offsets=offsets),
                               R.linear_backward(dy, x, w, None, rows, offsets, "none")):
        R.assert_within(a, ref, bound)
    # offsets that lead outside are held inside 0..8
    wild = torch.tensor([-7, 4, 2 ** 31 - 1], dtype=torch.int32, device="cuda")
    R.assert_within(ntc.linear(x, w, b, rows=rows, offsets=wild), y, yb)
    back = torch.tensor([6, 2, 8], dtype=torch.int32, device="cuda")  # expert 0 ends before it begins: no rows
    got = ntc.linear(x, w, b, rows=rows, offsets=back)
    want, _, bound, _ = R.linear(x, w[1:], b[1:], rows, torch.tensor([2, 8]))
    R.assert_within(got[2:], want[2:], bound[2:])


def test_many_experts_and_long_segments(ntc):
    g = gen(6)
    T, E = 3000, 1024
    x, w = normal(g, T, 64, dtype=torch.bfloat16), normal(g, E, 64, 64, std=0.1, dtype=torch.bfloat16)
    ids = torch.randint(0, E, (T, 1), generator=g, device="cuda").int()
    ids[: 1500] = 1023
    rows, _, offsets = R.order(ids, E)
    y, _, yb, _ = R.linear(x, w, None, rows, offsets)
    R.assert_within(ntc.linear(x, w, rows=rows, offsets=offsets), y, yb)
    dy = normal(g, T, 64, dtype=torch.bfloat16)
    for a, (ref, bound) in zip(ntc.linear_backward(dy, x, w, rows=rows, offsets=offsets),
                               R.linear_backward(dy, x, w, None, rows, offsets, "none")):
        R.assert_within(a, ref, bound)


def test_empty_calls(ntc):
    w = torch.zeros(2, 8, 16, dtype=torch.bfloat16, device="cuda")
    x = torch.zeros(0, 16, dtype=torch.bfloat16, device="cuda")
    offsets = torch.zeros(3, dtype=torch.int32, device="cuda")
    assert ntc.linear(x, w, offsets=offsets).shape == (0, 8)
    dx, dw, db = ntc.linear_backward(torch.zeros(0, 8, dtype=torch.bfloat16, device="cuda"), x, w, offsets=offsets)
    assert dx.shape == (0, 16) and (dw == 0).all() and (db == 0).all()
    # rows, but none of any expert
    x = torch.full((5, 16), math.nan, dtype=torch.bfloat16, device="cuda")
    y, z = ntc.linear(x, w, offsets=offsets, activation="silu", save=True)
    assert (y == 0).all() and (z == 0).all()
    dy = torch.full((5, 8), math.nan, dtype=torch.bfloat16, device="cuda")
    for t in ntc.linear_backward(dy, x, w, z=dy, offsets=offsets, activation="silu"):
        assert (t == 0).all()


# ------------------------------------------------------------------ the blend

@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T,D,k,E", [(1, 1, 1, 1), (1, 64, 8, 16), (37, 100, 3, 5), (50, 512, 8, 64), (9, 1031, 32, 40),
                                     (300, 8, 2, 4)])
def test_combine_and_its_gradient(ntc, dtype, T, D, k, E):
    g = gen(T * D)
    ids, rows, place, offsets = routed(g, T, E, k)
    live = int(offsets[-1])
    y, r, dout = normal(g, T * k, D, dtype=dtype), normal(g, T, D, dtype=dtype), normal(g, T, D, dtype=dtype)
    y[live:] = math.nan  # rows of no expert: whatever they hold
    w = normal(g, T, k)
    w[place >= live] = math.nan
    p = place.long()
    in_ = p < live
    for weights in (w, None):
        ww = torch.where(in_, (w if weights is not None else torch.ones_like(w)).double(), torch.zeros((), dtype=torch.float64, device="cuda"))
        yy = torch.where(in_[:, :, None], y[p].double(), torch.zeros((), dtype=torch.float64, device="cuda"))
        for res in (r, None):
            want = (ww[:, :, None] * yy).sum(1) + (0 if res is None else res.double())
            mag = (ww.abs()[:, :, None] * yy.abs()).sum(1) + (0 if res is None else res.double().abs())
            got = ntc.combine(y, place, weights, offsets, residual=res)
            R.assert_within(got, want, (k + 4) * R.F32 * mag + R.UNIT[dtype] * want.abs() * 1.01 + R.TINY[dtype])
        dy, dw = ntc.combine_backward(dout, y, place, weights, offsets)
        want = (ww[:, :, None] * dout.double()[:, None, :])
        R.assert_within(dy[p], want, 2 * R.UNIT[dtype] * want.abs() + R.TINY[dtype])
        want = (yy * dout.double()[:, None, :]).sum(2)
        mag = (yy * dout.double()[:, None, :]).abs().sum(2)
        R.assert_within(dw, want, (D + 8) * R.F32 * mag + 1e-37)
    only = ntc.combine_backward(dout, y, place, w, offsets, need=("dweights",))
    assert only[0] is None and only[1].shape == (T, k)


def test_combine_strides_and_wild_places(ntc):
    g = gen(2)
    y = normal(g, 12, 40, dtype=torch.bfloat16)
    wide = torch.full((12, 47), math.nan, dtype=torch.bfloat16, device="cuda")
    wide[:, 3:43] = y
    place = torch.tensor([[0, 11], [12, -1], [2 ** 31 - 1, 3], [-2 ** 31, 5]], dtype=torch.int32, device="cuda")
    w = normal(g, 4, 2)
    rows = {0: [0, 11], 1: [], 2: [3], 3: [5]}
    want = torch.zeros(4, 40, dtype=torch.float64, device="cuda")
    for t, (a, b) in enumerate(place.tolist()):
        for j, p in ((0, a), (1, b)):
            if 0 <= p < 12:
                assert p in rows[t]
                want[t] += w[t, j].double() * y[p].double()
    got = ntc.combine(wide[:, 3:43], place, w)
    R.assert_within(got, want, 2.0 ** -8 * want.abs() + 1e-6)


# ------------------------------------------------------------------ together

def layer(ntc, logits, x, w1, b1, w2, b2, k):
    ids, wt = ntc.route(logits, k)
    rows, place, offsets = ntc.expert_order(ids, w1.shape[0])
    h, z = ntc.linear(x, w1, b1, rows=rows, offsets=offsets, activation="silu", save=True)
    y = ntc.linear(h, w2, b2, offsets=offsets)
    return ntc.combine(y, place, wt, offsets, residual=x)


def test_a_layer_on_its_own_stream_and_in_a_graph(ntc):
    g = gen(11)
    T, D, H, E, k = 200, 128, 256, 8, 2
    args = [normal(g, T, E), normal(g, T, D, dtype=torch.bfloat16), normal(g, E, H, D, std=0.1, dtype=torch.bfloat16),
            normal(g, E, H), normal(g, E, D, H, std=0.1, dtype=torch.bfloat16), normal(g, E, D), k]
    want = layer(ntc, *args)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        side = layer(ntc, *args)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(side, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = layer(ntc, *args)
    for _ in range(2):
        args[1].copy_(normal(g, T, D, dtype=torch.bfloat16))
        args[0].copy_(normal(g, T, E))
        graph.replay()
        assert torch.equal(out, layer(ntc, *args))
    # an explicit stream argument
    with torch.cuda.stream(s):
        s.synchronize()
    y = ntc.linear(args[1], args[2][0], stream=s)
    s.synchronize()
    assert torch.equal(y, ntc.linear(args[1], args[2][0]))


@pytest.mark.parametrize("rows_of", ["whole chunks", "any", "one long and many short"])
def test_dw_of_long_contractions(ntc, rows_of):
    """Many chunks per tile and many tiles per CTA: no wait of any warp runs out, whatever its pace."""
    g = gen(21)
    E, K, N = 16, 512, 1024
    counts = {"whole chunks": [2048] * E, "any": [2048 - 37 * e for e in range(E)],
              "one long and many short": [20000] + [e for e in range(1, E)]}[rows_of]
    offsets = torch.tensor([0] + counts, device="cuda").cumsum(0).int()
    M = sum(counts)
    x, dy = normal(g, M, K, dtype=torch.bfloat16), normal(g, M, N, dtype=torch.bfloat16)
    w = normal(g, E, N, K, std=0.05, dtype=torch.bfloat16)
    want = R.linear_backward(dy, x, w, None, None, offsets, "none")
    rows = torch.arange(M, dtype=torch.int32, device="cuda")
    for r in (None, rows):
        for _ in range(10):
            _, dw, _ = ntc.linear_backward(dy, x, w, rows=r, offsets=offsets, need=("dw",))
        ntc.ntc_linear_status(torch.cuda.current_stream().cuda_stream)
        R.assert_within(dw, *want[1])
    for _ in range(10):
        dx, _, _ = ntc.linear_backward(dy, x, w, offsets=offsets, need=("dx",))
        y = ntc.linear(x, w, rows=rows, offsets=offsets)
    ntc.ntc_linear_status(torch.cuda.current_stream().cuda_stream)
    R.assert_within(dx, *want[0])
    ref, _, bound, _ = R.linear(x, w, None, None, offsets)
    R.assert_within(y, ref, bound)


# rows of each expert, in, out: many rows per expert and enough tiles of 256 x 256 for pairs of CTAs, with rows, columns
# and contractions that end anywhere in them (in the second CTA's half, at its first row, before it)
@pytest.mark.parametrize("counts,K,N", [((2048, 2048), 64, 4096), ((1300, 1537, 1025, 3000), 200, 2600),
                                        ((0, 4097, 128, 300), 1000, 2568), ((5000,), 333, 2049)])
@pytest.mark.parametrize("gather", [False, True])
def test_large_products(ntc, counts, K, N, gather):
    g = gen(sum(counts) + K)
    E, M = len(counts), sum(counts) + 5
    offsets = torch.tensor([0] + list(counts), device="cuda").cumsum(0).int()
    T = M // 2 + 7
    rows = torch.randint(-1, T, (M,), generator=g, device="cuda").int() if gather else None
    x = normal(g, T if gather else M, K, dtype=torch.bfloat16)
    w, b = normal(g, E, N, K, std=K ** -0.5, dtype=torch.bfloat16), normal(g, E, N)
    r, z, dy = (normal(g, M, N, dtype=torch.bfloat16) for _ in range(3))
    y, wz, yb, zb = R.linear(x, w, b, rows, offsets, "gelu", residual=r)
    got, gz = ntc.linear(x, w, b, rows=rows, offsets=offsets, activation="gelu", residual=r, save=True)
    R.assert_within(got, y, yb, "y")
    R.assert_within(gz, wz, zb, "z")
    got = ntc.linear_backward(dy, x, w, z=z, rows=rows, offsets=offsets, activation="silu")
    for name, a, (ref, bound) in zip(("dx", "dw", "db"), got, R.linear_backward(dy, x, w, z, rows, offsets, "silu")):
        R.assert_within(a, ref, bound, name)
    ntc.ntc_linear_status(torch.cuda.current_stream().cuda_stream)


# the same where the contraction is long: what pairs of CTAs take, with pairs whose second CTA has all, some or no rows
@pytest.mark.parametrize("counts,K,N", [((1000, 1100, 900, 1000), 4104, 4104), ((0, 2300, 128, 1300, 129), 1100, 4100),
                                        ((4000,), 1096, 4098)])
@pytest.mark.parametrize("gather", [False, True])
def test_large_products_of_long_contractions(ntc, counts, K, N, gather):
    test_large_products(ntc, counts, K, N, gather)


# rows of each expert, in, out: few tiles of dw and many rows, whose contraction is split; experts with fewer chunks of
# rows than parts, with one row, with none; and experts without rows at any size of their gradient
@pytest.mark.parametrize("counts,K,N", [((5000,), 17, 47), ((7446,), 133, 278), ((3000, 1, 0, 65, 4000), 40, 72),
                                        ((0, 0, 9000), 129, 130), ((12000, 12000), 64, 64)])
@pytest.mark.parametrize("gather", [False, True])
def test_dw_of_few_tiles(ntc, counts, K, N, gather):
    test_large_products(ntc, counts, K, N, gather)


@pytest.mark.parametrize("K,N", [(1, 1), (3, 5), (28, 3462), (16, 300), (333, 77), (200, 640)])
def test_experts_without_rows(ntc, K, N):
    g = gen(K + N)
    E, M = 90, 41
    offsets = torch.zeros(E + 1, dtype=torch.int32, device="cuda")
    offsets[8:] = 17
    offsets[70:] = M
    x, dy = normal(g, M, K, dtype=torch.float16), normal(g, M, N, dtype=torch.float16)
    w = normal(g, E, N, K, std=K ** -0.5, dtype=torch.float16)
    empty = offsets[1:] == offsets[:-1]
    w[empty] = float("nan")  # not read
    y = ntc.linear(x, w, offsets=offsets)
    got = ntc.linear_backward(dy, x, w, offsets=offsets)
    w[empty] = 0
    ref, _, bound, _ = R.linear(x, w, None, None, offsets)
    R.assert_within(y, ref, bound)
    for name, a, (ref, bound) in zip(("dx", "dw", "db"), got, R.linear_backward(dy, x, w, None, None, offsets, "none")):
        R.assert_within(a, ref, bound, name)
    assert not got[1][empty].any() and not got[2][empty].any()
