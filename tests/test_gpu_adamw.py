"""The AdamW step of many tensors against a 64-bit reference: types, alignments, moments in 32 and in 8 bits."""
import math

import pytest
import torch

import tests.experts_ref as R
import tests.train_serve_ref as S

pytestmark = pytest.mark.gpu
F8 = torch.float8_e4m3fn
H, B, F = torch.float16, torch.bfloat16, torch.float32
HYPER = dict(lr=3e-3, beta1=0.85, beta2=0.98, eps=1e-8, weight_decay=0.1)


@pytest.fixture(scope="module")
def ntc():
    from paper_2608_27888_gb300 import ntc
    return ntc


def guarded(values, shift, fill):
    """values in a larger buffer, `shift` elements from its start, and the buffer."""
    n = values.numel()
    whole = torch.full((n + shift + 64,), fill, dtype=F, device="cuda").to(values.dtype)
    part = whole[shift:shift + n].view(values.shape)
    part.copy_(values)
    return part, whole


class Case:
    """Tensors of a step in buffers whose other elements must stay as they are."""

    def __init__(self, specs, eight, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.lists = {k: [] for k in ("p", "g", "m", "v", "c", "s")}
        self.guards = []
        for shape, pt, gt, ct, shift in specs:
            n = math.prod(shape)
            size = torch.exp(2 * torch.randn(n, generator=g, device="cuda")) * 1e-2
            normal = lambda: torch.randn(n, generator=g, device="cuda").view(shape)  # noqa: E731
            m, r = normal() * size.view(shape), (normal().abs() + 0.01) * size.view(shape)
            if eight:
                (m, a), (r, b) = encode(m), encode(r)
                s = torch.zeros(2, a.numel() + 3, device="cuda")
                s[0, :a.numel()], s[1, :a.numel()] = a, b
                self.lists["s"].append(s[:, :a.numel()])
            values = dict(p=normal().to(pt), g=(normal() * size.view(shape)).to(gt), m=m, v=r if eight else r * r,
                          c=None if ct is None else torch.zeros(shape, dtype=ct, device="cuda"))
            for k, x in values.items():
                if x is None:
                    self.lists[k].append(None)
                    continue
                part, whole = guarded(x, shift, 3.0)
                self.lists[k].append(part)
                self.guards.append((part, whole, shift))

    def intact(self):
        for part, whole, shift in self.guards:
            w, n = whole.float(), part.numel()
            if not (bool((w[:shift] == 3).all()) and bool((w[shift + n:] == 3).all())):
                return False
        return True

    def clone(self):
        return {k: [None if x is None else x.clone() for x in v] for k, v in self.lists.items()}


def encode(x):
    """e4m3 codes and the blocks' scales of x, to the nearest."""
    f = torch.zeros(-(-x.numel() // 256) * 256, device=x.device)
    f[:x.numel()] = x.flatten()
    f = f.view(-1, 256)
    s = f.abs().amax(1) / 448
    code = torch.where(s[:, None] > 0, f / s[:, None].clamp_min(1e-30), torch.zeros_like(f)).clamp(-448, 448).to(F8)
    return code.view(-1)[:x.numel()].view(x.shape), s


def decode(code, s):
    return code.double().flatten() * s.double().repeat_interleave(256)[:code.numel()]


def check_codes(code, s, want, bound, root):
    """Codes against the moments: a code is off by half of a step, 2^-4 of the value or half of the least code 2^-9 of
    the scale; the scale (largest / 448) by two roundings of fp32; with `root`, what is above 0 stays so."""
    n = want.numel()
    if n == 0:
        return
    pad = torch.zeros(s.numel() * 256, dtype=torch.float64, device=want.device)
    pad[:n] = want.abs().flatten()
    top = pad.view(-1, 256).amax(1)
    R.assert_within(s, top / 448, top / 448 * 2.0 ** -21 + 1e-30 + bound.max() / 448, "scales")
    least = s.double().repeat_interleave(256)[:n]
    got = decode(code, s)
    w = want.flatten()
    half = torch.maximum(w.abs() * 2.0 ** -4, least * 2.0 ** -10 * (2 if root else 1))  # a root below the least code takes it
    R.assert_within(got, w, half * (1 + 2.0 ** -18) + bound.flatten() + 1e-30, "codes")
    if root:
        assert bool((code.float().flatten()[(w > 1e-25) & (least > 0)] > 0).all())


def run_and_check(ntc, case, eight, step=7, grad_scale=1.0, **how):
    before = case.clone()
    l = case.lists
    ntc.adamw(l["p"], l["g"], l["m"], l["v"], scales=l["s"] if eight else None, copies=l["c"], **dict(HYPER, **how.pop("given", {})),
              step=how.pop("step_given", step), grad_scale=how.pop("scale_given", grad_scale), **how)
    for i, p0 in enumerate(before["p"]):
        m0, v0 = before["m"][i], before["v"][i]
        if eight:
            m0 = decode(m0, before["s"][i][0]).view(p0.shape)
            v0 = decode(v0, before["s"][i][1]).view(p0.shape) ** 2
        p, m, v, b_p, b_m, b_v = S.adamw(p0, before["g"][i], m0, v0, step, grad_scale=grad_scale, **HYPER)
        if eight:  # decoding: a product rounded once, the square of the root once more
            b_m = b_m + 2 * S.U32 * m0.abs()
            b_v = b_v + 6 * S.U32 * v0
            b_p = b_p + b_p * 8
        u = 0.0 if l["p"][i].dtype == F else R.UNIT[l["p"][i].dtype]
        R.assert_within(l["p"][i], p, b_p + u * (p.abs() + b_p) + (R.TINY[l["p"][i].dtype] if u else 0), ("p", i))
        if l["c"][i] is not None:
            u = R.UNIT[l["c"][i].dtype]
            R.assert_within(l["c"][i], p, b_p + u * (p.abs() + b_p) + R.TINY[l["c"][i].dtype], ("copy", i))
        if eight:
            check_codes(l["m"][i], l["s"][i][0], m, b_m, False)
            r = v.sqrt()
            b_r = torch.minimum(b_v / (2 * r).clamp_min(1e-300), b_v.sqrt()) + 2 * S.U32 * r
            check_codes(l["v"][i], l["s"][i][1], r, b_r, True)
        else:
            R.assert_within(l["m"][i], m, b_m, ("m", i))
            R.assert_within(l["v"][i], v, b_v, ("v", i))
        assert torch.equal(l["g"][i], before["g"][i])
    assert case.intact()


SPECS = [[((n,), pt, gt, ct, shift) for n, pt, gt, ct in
          [(1, F, F, None), (255, F, B, B), (256, F, H, H), (257, B, B, None), (1000, H, F, None), (4099, F, F, B), (31, B, F, F),
           (512, H, H, B), (70000, F, B, B)]] for shift in (0, 1, 4, 8)]


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("specs", SPECS, ids=["aligned", "by1", "by4", "by8"])
def test_types_sizes_and_alignments(ntc, specs, eight):
    run_and_check(ntc, Case(specs, eight), eight)
    run_and_check(ntc, Case(specs, eight, seed=1), eight, grad_scale=0.125)


@pytest.mark.parametrize("eight", [False, True])
def test_many_tensors_of_odd_shapes(ntc, eight):
    """More than a launch takes, an empty one among them."""
    specs = [((i % 5 + 1, (i * 37) % 211 + 1), F, B if i % 2 else F, B if i % 3 == 0 else None, i % 9) for i in range(530)]
    specs[17] = ((0, 8), F, F, None, 0)
    run_and_check(ntc, Case(specs, eight), eight)


@pytest.mark.parametrize("eight", [False, True])
def test_first_step_from_zero(ntc, eight):
    c = Case([((600,), F, F, None, 0)], eight)
    for k in ("m", "v"):
        c.lists[k][0].copy_(torch.zeros(600, device="cuda"))
    if eight:
        c.lists["s"][0].zero_()
    run_and_check(ntc, c, eight, step=1)


@pytest.mark.parametrize("eight", [False, True])
def test_device_scalars(ntc, eight):
    """step, lr and grad_scale on the device: the scalars come from the same formulas in 64 bits, so the bits are equal."""
    a, b = Case(SPECS[0], eight, seed=4), Case(SPECS[0], eight, seed=4)
    t = lambda x, dtype=F: torch.tensor([x], dtype=dtype, device="cuda")  # noqa: E731
    lr = float(t(HYPER["lr"]))
    run_and_check(ntc, a, eight, step=23, grad_scale=0.5, given=dict(lr=lr))
    run_and_check(ntc, b, eight, step=23, grad_scale=0.5, step_given=t(23, torch.int32), scale_given=t(0.5), given=dict(lr=t(lr)))
    for k in ("p", "m", "v", "c"):
        for x, y in zip(a.lists[k], b.lists[k]):
            assert x is None or torch.equal(x.float(), y.float()), k


@pytest.mark.parametrize("eight", [False, True])
def test_graph_counts_its_steps(ntc, eight):
    """Replays of a captured step are the steps that calls would take, with rates and gradients of their own."""
    from paper_2608_27888_gb300.optim import AdamW
    g = torch.Generator(device="cuda").manual_seed(2)
    start = [torch.randn(300, 7, generator=g, device="cuda").to(B), torch.randn(50, generator=g, device="cuda")]
    grads = [[torch.randn(p.shape, generator=g, device="cuda").to(p.dtype) for p in start] for _ in range(6)]
    one, two = [p.clone() for p in start], [p.clone() for p in start]
    calls = AdamW(one, lr=0.01, bits=8 if eight else 32)
    replays = AdamW(two, lr=0.01, bits=8 if eight else 32, captured=True)
    live = [x.clone() for x in grads[0]]
    calls.step(grads[0])
    replays.step(live)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        replays.step(live)
    for i in range(1, 6):
        lr = float(torch.tensor(0.01 / i))
        calls.set_lr(lr)
        replays.set_lr(lr)
        calls.step(grads[i])
        for x, y in zip(live, grads[i]):
            x.copy_(y)
        graph.replay()
    torch.cuda.synchronize()
    assert int(replays.steps) == calls.steps == 6
    for a, b in zip(one + calls.masters + calls.m + calls.v, two + replays.masters + replays.m + replays.v):
        assert torch.equal(a.float(), b.float())


def test_side_stream_and_equal_bits(ntc):
    runs = []
    for k in range(3):
        c = Case(SPECS[1], True, seed=9)
        l = c.lists
        s = torch.cuda.Stream() if k == 2 else None
        torch.cuda.synchronize()
        ntc.adamw(l["p"], l["g"], l["m"], l["v"], scales=l["s"], copies=l["c"], step=3, stream=s, **HYPER)
        torch.cuda.synchronize()
        runs.append([x.float().clone() for k in ("p", "m", "v", "c", "s") for x in l[k] if x is not None])
    for other in runs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(runs[0], other))


def test_not_a_number_stays_where_it_is(ntc):
    """In 32 bits an element; in 8 bits its block of 256, whose scale is no number."""
    for eight in (False, True):
        for bad in (math.nan, math.inf):
            c = Case([((1000,), F, F, None, 0)], eight)
            l = c.lists
            l["g"][0][300] = bad
            ntc.adamw(l["p"], l["g"], l["m"], l["v"], scales=l["s"] if eight else None, step=2, **HYPER)
            p = l["p"][0]
            assert not math.isfinite(float(p[300])) and int(torch.isfinite(p).sum()) == 999
            if not eight:
                assert int(torch.isfinite(l["m"][0]).sum()) == 999 and int(torch.isfinite(l["v"][0]).sum()) == 999
            else:
                for row in l["s"][0]:
                    assert torch.isnan(row).tolist() == [False, True, False, False]
                ntc.adamw(l["p"], l["g"], l["m"], l["v"], scales=l["s"], step=3, **HYPER)
                assert int(torch.isfinite(p).sum()) == 1000 - 256


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("scale", [0.0, 1e-25, 1e-12, 1e12])
def test_gradients_of_every_size(ntc, eight, scale):
    """A gradient of 1e-25 squared is below fp32's smallest number (v stays 0, eps holds the step), one of 1e12 is not
    above its largest; blocks of zeros have the scale 0."""
    p = torch.randn(700, device="cuda")
    g = torch.randn(700, device="cuda") * scale
    kind = F8 if eight else F
    m, v = (torch.zeros(700, device="cuda").to(kind) for _ in range(2))
    s = [torch.zeros(2, 3, device="cuda")] if eight else None
    want = p.double()
    gd = g.double()
    ntc.adamw([p], [g], [m], [v], scales=s, step=1, lr=0.1, weight_decay=0.0)
    v1 = 0.001 * gd * gd
    if scale == 1e-25:
        v1 = torch.zeros_like(v1)
    # at step 1 m / (1 - beta1) is g and v / (1 - beta2) its square
    want = want - 0.1 * gd / ((v1 / (1 - 0.999)).sqrt() + 1e-8)
    R.assert_within(p, want, 0.1 * 2.0 ** -19 + want.abs() * 2.0 ** -22, scale)
    if scale == 0.0:
        assert not m.float().any() and not v.float().any() and (not eight or not s[0].any())
    assert torch.isfinite(p).all() and torch.isfinite(m.float()).all() and torch.isfinite(v.float()).all()


def test_eight_bits_follow_thirty_two(ntc):
    """Twenty steps of one gradient with beta1 = beta2 = 1/2.  A code is off by 2^-4 of its value (all gradients are far
    above the least code's share of their block's largest), so m_k = m_{k-1} (1 + d) / 2 + g / 2 is off by at most
    2^-5 / (1 - 17 / 32) = 1/15 of g, v by ((17 / 16)^2 - 1) / 2 / (1 - (17 / 16)^2 / 2) = 0.148 of g^2, its root by 0.077
    of |g|; the two agree at the first step.  An update is off by (1/15 + 0.077) / (1 - 0.077) = 0.156 of itself."""
    g = torch.Generator(device="cuda").manual_seed(11)
    p0 = torch.randn(64 * 256, generator=g, device="cuda")
    grad = torch.randn(64 * 256, generator=g, device="cuda").sign() * (torch.rand(64 * 256, generator=g, device="cuda") + 0.01)
    runs = []
    for kind in (F, F8):
        p, m, v = p0.clone(), torch.zeros_like(p0).to(kind), torch.zeros_like(p0).to(kind)
        s = [torch.zeros(2, 64, device="cuda")] if kind == F8 else None
        for t in range(1, 21):
            ntc.adamw([p], [grad], [m], [v], scales=s, step=t, lr=0.01, beta1=0.5, beta2=0.5, weight_decay=0.0)
        runs.append((p - p0).double())
    R.assert_within(runs[1], runs[0], 0.157 * runs[0].abs() + 1e-6)


@pytest.mark.parametrize("scale", [1.0, 1e-9, 1e-14, 1e9])
def test_moments_are_rounded_as_they_are_defined(ntc, scale):
    """The same operations in torch, each rounded to nearest in fp32: the same moments, codes and scales, bit for bit.  A
    last digit that is off is a code that is off where codes are far apart."""
    n, b1, b2 = 256 * 4000, 0.85, 0.98
    g = torch.Generator(device="cuda").manual_seed(21)
    size = torch.exp(2 * torch.randn(n, generator=g, device="cuda")) * scale
    grad = torch.randn(n, generator=g, device="cuda") * size
    grad[: 256 * 3] = 0.0
    one = lambda x: torch.tensor(x, dtype=F, device="cuda")  # noqa: E731
    m32 = torch.randn(n, generator=g, device="cuda") * size
    (m, a), (r, b) = encode(m32), encode((torch.randn(n, generator=g, device="cuda").abs() + 0.01) * size)
    s = torch.stack([a, b])
    m0, r0 = m.float() * a.repeat_interleave(256), r.float() * b.repeat_interleave(256)
    p = torch.randn(n, generator=g, device="cuda")
    m1 = m0 * one(b1) + grad * one(1 - b1)
    v1 = (r0 * r0) * one(b2) + (grad * one(1 - b2)) * grad
    v32, m_old = r0 * r0, m0.clone()
    ntc.adamw([p.clone()], [grad], [m_old], [v32], step=5, lr=0.01, beta1=b1, beta2=b2)
    assert torch.equal(m_old, m1) and torch.equal(v32, v1)
    ntc.adamw([p], [grad], [m], [r], scales=[s], step=5, lr=0.01, beta1=b1, beta2=b2)
    for want, code, got_scale, root in ((m1, m, s[0], False), (torch.sqrt(v1), r, s[1], True)):
        f = want.view(-1, 256)
        top = f.abs().amax(1, keepdim=True)
        y = torch.where(top >= 2.0 ** -100, f * torch.div(torch.full_like(top, 448.0), top), torch.zeros_like(f))
        if root:
            y = torch.where(y > 0, y.clamp_min(2.0 ** -9), y)
        assert torch.equal(code.view(torch.uint8), y.to(F8).view(torch.uint8).view(-1))
        assert torch.equal(got_scale, torch.where(top >= 2.0 ** -100, top * one(1.0 / 448.0), torch.zeros_like(top)).view(-1))


def test_past_2_31_elements(ntc):
    """One tensor of 2^31 + 300 elements, most of them zero: offsets past 32 bits."""
    n = 2 ** 31 + 300
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("needs 24 GB")
    p, g = torch.zeros(n, dtype=B, device="cuda"), torch.zeros(n, dtype=B, device="cuda")
    m, v = (torch.zeros(n, dtype=torch.uint8, device="cuda").view(F8) for _ in range(2))
    s = torch.zeros(2, -(-n // 256), device="cuda")
    at = torch.tensor([0, 255, 256, 2 ** 31 - 1, 2 ** 31, 2 ** 31 + 256, n - 1], device="cuda")
    g[at] = 1.0
    ntc.adamw([p], [g], [m], [v], scales=[s], step=1, lr=0.5, weight_decay=0.0)
    assert torch.equal(p[at].float(), torch.full((7,), -0.5, device="cuda"))
    for lo, hi in ((0, 300), (2 ** 31 - 300, n)):
        other = torch.ones(hi - lo, dtype=torch.bool, device="cuda")
        other[at[(at >= lo) & (at < hi)] - lo] = False
        assert not p[lo:hi][other].any()
    assert torch.equal((s[0] > 0).nonzero().flatten(), torch.unique(at // 256))
    assert bool((m[-1:].float() == 448).all()) and bool((v[-1:].float() == 448).all())


def test_what_is_refused(ntc):
    z = lambda *s, dtype=F: torch.zeros(*s, dtype=dtype, device="cuda")  # noqa: E731
    one = lambda **k: dict(dict(params=[z(8)], grads=[z(8)], m=[z(8)], v=[z(8)], step=1, lr=0.1), **k)  # noqa: E731
    for how, word in [
            (one(grads=[]), "an entry for each"), (one(grads=[z(9)]), "shape"), (one(m=[z(8, dtype=H)]), "must be Float"),
            (one(v=[z(8, dtype=F8)]), "must be Float"), (one(m=[z(8, dtype=F8)], v=[z(8, dtype=F8)]), "need scales"),
            (one(scales=[z(2, 1)]), "float8"), (one(m=[z(8, dtype=F8)], v=[z(8, dtype=F8)], scales=[z(2, 2)]), "scales"),
            (one(params=[z(16)[::2]]), "contiguous"), (one(grads=[z(4, 2).t()], params=[z(2, 4)], m=[z(2, 4)], v=[z(2, 4)]), "contiguous"),
            (one(params=[z(8, dtype=torch.float64)]), "float32, float16 or bfloat16"), (one(params=[torch.zeros(8)]), "CUDA tensor"),
            (one(grads=[torch.zeros(8)]), "is on"), (one(copies=[z(7)]), "shape"), (one(step=0), "step"),
            (one(step=z(1)), "must be Int"), (one(lr=z(2)), "one element"), (one(grad_scale=z(1, dtype=H)), "must be Float")]:
        with pytest.raises(ValueError, match=word):
            ntc.adamw(**how)
    for how in (one(params=z(8).sum()), one(step="1"), one(lr=None)):
        with pytest.raises(TypeError):
            ntc.adamw(**how)
    p = z(8)
    for how, word in [(one(params=[p, p], grads=[z(8), z(8)], m=[z(8), z(8)], v=[z(8), z(8)]), "overlaps"), (one(params=[p], grads=[p]), "overlaps"),
                      (one(lr=-1.0), "negative"), (one(lr=math.nan), "finite"), (one(beta1=1.0), "beta1")]:
        with pytest.raises(ntc.NtcError, match=word):
            ntc.adamw(**how)
    ntc.adamw([], [], [], [], step=1, lr=0.1)
    leaf = torch.nn.Parameter(z(8))  # a step in place, as torch counts them
    before = leaf._version
    ntc.adamw([leaf], [z(8)], [z(8)], [z(8)], step=1, lr=0.1)
    assert leaf._version == before + 1


def test_state_of_the_optimizer():
    """A run from a saved state goes on with the same bits, and 16-bit parameters are their masters rounded."""
    from paper_2608_27888_gb300.optim import AdamW
    g = torch.Generator(device="cuda").manual_seed(5)
    for bits in (32, 8):
        w = dict(a=torch.randn(33, 17, generator=g, device="cuda").to(B), b=torch.randn(9, generator=g, device="cuda"))
        grads = [dict(a=torch.randn(33, 17, generator=g, device="cuda").to(B), b=torch.randn(9, generator=g, device="cuda")) for _ in range(4)]
        one = AdamW(w, lr=0.05, bits=bits)
        for x in grads[:2]:
            one.step(x)
        saved = {k: [t.clone() for t in x] if isinstance(x, list) else x for k, x in one.state().items()}
        w2 = {k: x.clone() for k, x in w.items()}
        two = AdamW(w2, lr=0.05, bits=bits)
        two.load(saved)
        for x in grads[2:]:
            one.step(x)
            two.step(x)
        assert all(torch.equal(w[k], w2[k]) for k in w) and two.steps == 4
        assert torch.equal(w["a"], one.masters[0].to(B))
        with pytest.raises(ValueError, match="bits"):
            AdamW(w, bits=40 - bits).load(saved)


@pytest.mark.parametrize("captured", [False, True])
def test_a_refused_step_is_none(captured):
    """Gradients that do not fit change nothing, and the next step is the first."""
    from paper_2608_27888_gb300.optim import AdamW
    w = [torch.ones(40, device="cuda"), torch.ones(3, device="cuda")]
    opt = AdamW(w, lr=0.1, captured=captured)
    with pytest.raises(ValueError, match="grads"):
        opt.step([torch.ones(40, device="cuda"), torch.ones(4, device="cuda")])
    assert int(opt.steps) == 0 and all(bool((p == 1).all()) for p in w)
    opt.step([torch.ones(40, device="cuda"), torch.ones(3, device="cuda")])
    assert int(opt.steps) == 1
    # the first step's change is the rate whatever the gradient, and the decay its hundredth
    assert all(bool(((p - (1 - 0.1 * 0.01 - 0.1)).abs() < 1e-6).all()) for p in w)
    AdamW([], captured=False).step([])
    with pytest.raises(ValueError, match="captured"):
        AdamW([], captured=True)
