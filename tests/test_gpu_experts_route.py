"""The router, its gradient, and the order by expert against their plain 64-bit forms."""
import math

import pytest
import torch

import tests.experts_ref as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ntc():
    from paper_2608_27888_gb300 import ntc
    return ntc


def apart(T, E, seed, spread=4.0):
    """Logits whose scores are well apart in every row (a shuffled grid), so that fp32 and 64 bits choose alike."""
    g = torch.Generator().manual_seed(seed)
    grid = torch.linspace(-spread, spread, E)
    return torch.stack([grid[torch.randperm(E, generator=g)] for _ in range(T)])


def check_weights(got, want, logits):
    # exp of a difference of up to 2 * range in fp32 (its argument's rounding), a sum of E terms, a division
    finite = logits[torch.isfinite(logits)].double().abs()
    rel = R.F32 * (4 * (float(finite.max()) if finite.numel() else 0.0) + logits.shape[1] + 64)
    R.assert_within(got.cpu(), want, rel * want.abs() + 1e-37, "weights")


@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (1, 8, 2), (3, 31, 5), (5, 33, 32), (17, 64, 6), (9, 100, 1), (7, 256, 8),
                                   (3, 257, 10), (2, 586, 9), (5, 1024, 32)])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_route_matches_the_definition(ntc, T, E, k, score):
    logits = apart(T, E, seed=E + k)
    bias = torch.linspace(-0.3, 0.3, E)[torch.randperm(E, generator=torch.Generator().manual_seed(2))] * (1e-3 / E)
    for b, renorm, scale in ((None, True, 1.0), (bias, False, 2.5)):
        want_ids, want = R.route(logits, k, b, score, renormalize=renorm, scale=scale)
        ids, w = ntc.route(logits.cuda(), k, bias=None if b is None else b.cuda(), score=score, renormalize=renorm,
                           scale=scale)
        assert torch.equal(ids.cpu(), want_ids)
        check_weights(w, want, logits)


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("E", [16, 40, 128, 1000])
def test_route_types_strides_and_alignment(ntc, dtype, E):
    """Every type, rows at odd strides and addresses, through views of a larger buffer."""
    logits = apart(6, E, seed=1, spread=E / 64).to(dtype)  # distinct after rounding or tied: ties go to the lower index
    want_ids, want = R.route(logits.float(), 4)
    for pad, skip in ((0, 0), (1, 0), (3, 1), (8, 8)):
        buf = torch.full((6, E + pad + skip), 7.0, dtype=dtype, device="cuda")
        view = buf[:, skip:skip + E]
        view.copy_(logits)
        ids, w = ntc.route(view, 4)
        assert torch.equal(ids.cpu(), want_ids), (pad, skip)
        check_weights(w, want, logits)


@pytest.mark.parametrize("E,groups,top", [(64, 8, 3), (64, 8, 8), (256, 8, 4), (60, 6, 2), (35, 7, 3), (32, 32, 5), (24, 2, 1),
                                          (160, 8, 4), (1024, 32, 3), (6, 6, 4)])
def test_route_groups(ntc, E, groups, top):
    k = min(4, E // groups * top)
    logits = apart(13, E, seed=groups)
    # a group's value is a sum of two: pull the groups apart
    logits += (torch.arange(E) // (E // groups)).float()[torch.randperm(E, generator=torch.Generator().manual_seed(3))] * 0.01
    bias = torch.linspace(0, 0.05, E)
    want_ids, want = R.route(logits, k, bias, "sigmoid", groups, top)
    ids, w = ntc.route(logits.cuda(), k, bias=bias.cuda(), score="sigmoid", groups=groups, top_groups=top)
    assert torch.equal(ids.cpu(), want_ids)
    check_weights(w, want, logits)


def test_route_ties_go_to_the_lower_index(ntc):
    for E in (5, 32, 70, 300):
        logits = torch.zeros(4, E)
        logits[1, E // 2:] = 1.0
        logits[2, ::3] = -0.0
        logits[3] = torch.arange(E) % 2
        for score in ("softmax", "sigmoid"):
            want, _ = R.route(logits, 5, None, score)
            ids, _ = ntc.route(logits.cuda(), 5, score=score)
            assert torch.equal(ids.cpu(), want), (E, score)
    # ties between groups: the lower group
    ids, _ = ntc.route(torch.zeros(1, 64).cuda(), 8, groups=8, top_groups=2)
    assert ids[0].tolist() == list(range(8))


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("groups", [1, 4])
def test_route_masks_and_infinities(ntc, score, groups):
    E, k, lowest = 40, 6, torch.finfo(torch.float32).min
    l = apart(8, E, seed=4)
    l[0, :] = -math.inf                  # an empty row
    l[1, 3:] = -math.inf                 # fewer left than top_k
    l[2, ::2] = math.nan
    l[3, 5] = math.inf
    l[4, :] = math.nan
    l[5, 1:] = lowest                    # masked by the type's lowest value: scores of 0, lowest index first
    l[6, 10:20] = -math.inf              # a whole group
    want_ids, want = R.route(l, k, None, score, groups, max(1, groups - 1))
    ids, w = ntc.route(l.cuda(), k, score=score, groups=groups, top_groups=max(1, groups - 1))
    assert torch.equal(ids.cpu(), want_ids)
    assert torch.isfinite(w).all()
    R.assert_within(w.cpu(), want, 1e-5 * want.abs() + 1e-37)
    assert (ids[0] == -1).all() and (w[0] == 0).all()
    g = ntc.route_backward(l.cuda(), ids, torch.randn(8, k, device="cuda"), score=score, renormalize=False)
    assert torch.isfinite(g).all()
    assert (g[0] == 0).all() and (g[4] == 0).all() and (g[2, ::2] == 0).all()


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [True, False])
@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (3, 8, 2), (5, 33, 4), (65, 64, 6), (4, 586, 10), (3, 1024, 32)])
def test_route_backward_matches_the_formula(ntc, score, renorm, T, E, k):
    g = torch.Generator().manual_seed(E * k)
    logits = torch.randn(T, E, generator=g)
    ids = torch.stack([torch.randperm(E, generator=g)[:k] for _ in range(T)]).int()
    dw = torch.randn(T, k, generator=g)
    l = logits.double().requires_grad_()
    w = R.route_weights(l, ids, score, renorm, 1.5)
    want, = torch.autograd.grad(w, l, dw.double())
    # every term is a product of scores and dw: bounded by the largest |dw| * 1.5 / (the chosen scores' sum)
    s = torch.sigmoid(l) if score == "sigmoid" else torch.softmax(l, 1)
    big = 1.5 * dw.abs().double().amax(1, keepdim=True) * (1 if not renorm or score == "softmax" else 1 / s.gather(1, ids.long()).sum(1, keepdim=True))
    for dtype in (torch.float32, torch.bfloat16, torch.float16):
        if dtype == torch.float32:
            x, ref = logits, want
        else:
            x = logits.to(dtype)
            l2 = x.double().requires_grad_()
            ref, = torch.autograd.grad(R.route_weights(l2, ids, score, renorm, 1.5), l2, dw.double())
        got = ntc.route_backward(x.cuda(), ids.cuda(), dw.cuda(), score=score, renormalize=renorm, scale=1.5)
        assert got.dtype == dtype
        bound = (E + k + 64) * R.F32 * big.detach() + 2 * R.UNIT[dtype] * ref.abs() + R.TINY[dtype]
        R.assert_within(got.cpu(), ref, bound, str(dtype))


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [True, False])
def test_route_backward_matches_differences(ntc, score, renorm):
    """The gradient against central differences of ntc.route's own weights."""
    T, E, k, h = 3, 12, 3, 2.0 ** -8
    logits = apart(T, E, seed=9, spread=2.0)
    dw = torch.randn(T, k, generator=torch.Generator().manual_seed(1))
    ids, _ = ntc.route(logits.cuda(), k, score=score, renormalize=renorm)
    got = ntc.route_backward(logits.cuda(), ids, dw.cuda(), score=score, renormalize=renorm).cpu()
    for e in range(E):
        up, down = logits.clone(), logits.clone()
        up[:, e] += h
        down[:, e] -= h
        (i1, a), (i0, b) = (ntc.route(v.cuda(), k, score=score, renormalize=renorm) for v in (up, down))
        assert torch.equal(i1, ids) and torch.equal(i0, ids)
        diff = ((a.double() - b.double()).cpu() * dw.double()).sum(1) / (2 * h)
        # third derivatives are at most 1 per weight: h^2 / 6; fp32 weights: 2^-22 / (2 h) each
        bound = dw.abs().double().sum(1) * (h * h / 6 + 2.0 ** -22 / h)
        R.assert_within(got[:, e], diff, bound)


def test_route_backward_ids_outside_and_repeated(ntc):
    l = torch.randn(2, 10, generator=torch.Generator().manual_seed(0)).cuda()
    ids = torch.tensor([[3, -1, 99], [4, 4, 7]], dtype=torch.int32, device="cuda")
    dw = torch.tensor([[1.0, 5.0, 7.0], [0.5, 0.25, -1.0]], device="cuda")
    got = ntc.route_backward(l, ids, dw, score="sigmoid", renormalize=False).cpu().double()
    s = torch.sigmoid(l.cpu().double())
    want = torch.zeros(2, 10, dtype=torch.float64)
    want[0, 3] = s[0, 3] * (1 - s[0, 3])
    want[1, 4] = 0.75 * s[1, 4] * (1 - s[1, 4])
    want[1, 7] = -s[1, 7] * (1 - s[1, 7])
    R.assert_within(got, want, torch.full_like(want, 16 * R.F32))


@pytest.mark.parametrize("n,k,E", [(0, 1, 4), (1, 1, 1), (1, 8, 64), (33, 1, 7), (512, 8, 64), (513, 8, 1024), (4096, 2, 16),
                                   (4097, 1, 16), (5000, 8, 586), (70000, 6, 64), (3000, 32, 1024)])
def test_expert_order_is_the_stable_sort(ntc, n, k, E):
    g = torch.Generator().manual_seed(n + E)
    ids = torch.randint(-2, E + 3, (n, k), generator=g).int()
    ids[n // 2:n // 2 + 5] = -2 ** 31
    ids[n // 3:n // 3 + 50] = E - 1  # a run of one expert
    want = R.order(ids, E)
    for _ in range(2):
        got = ntc.expert_order(ids.cuda(), E)
        for a, b in zip(got, want):
            assert torch.equal(a.cpu(), b)


def test_empty_route(ntc):
    l = torch.empty(0, 16, device="cuda")
    ids, w = ntc.route(l, 2)
    assert ids.shape == (0, 2) and w.shape == (0, 2)
    assert ntc.route_backward(l, ids, w).shape == (0, 16)


@pytest.mark.parametrize("E", [16, 100, 300])
def test_a_bias_of_minus_infinity_or_nan_masks_an_expert(ntc, E):
    l = apart(5, E, seed=3)
    bias = torch.zeros(E)
    bias[::3] = -math.inf
    bias[1::3] = math.nan
    ids, w = ntc.route(l.cuda(), 5, bias=bias.cuda(), score="sigmoid")
    masked = l.clone()
    masked[:, ::3] = -math.inf
    masked[:, 1::3] = -math.inf
    want_ids, want = R.route(masked, 5, None, "sigmoid")
    assert torch.equal(ids.cpu(), want_ids)
    check_weights(w, want, l)


def test_equal_values_of_one_lane_in_any_number(ntc):
    """Runs of equal values inside and across the lanes' shares of a row, with more choices than a share holds."""
    g = torch.Generator().manual_seed(5)
    for E in (8, 24, 64, 128, 200, 256):
        for k in (4, 8, 9, 20):
            if k > E:
                continue
            l = torch.randint(0, 3, (50, E), generator=g).float()
            want, _ = R.route(l, k, None, "sigmoid")
            ids, _ = ntc.route(l.cuda(), k, score="sigmoid")
            assert torch.equal(ids.cpu(), want), (E, k)
