"""Training and serving a routed layer past 2^31 elements: offsets past 32 bits in the balance loss and the 4-bit weights."""
import pytest
import torch

import tests.experts_ref as R
import tests.train_serve_ref as S

pytestmark = pytest.mark.gpu
B = torch.bfloat16


@pytest.fixture(scope="module")
def ntc():
    from paper_2608_27888_gb300 import ntc
    return ntc


def room(gb):
    if torch.cuda.mem_get_info()[0] < gb << 30:
        pytest.skip(f"needs {gb} GB")


def test_packing_past_2_31_weights(ntc):
    room(32)
    E, N, K, group = 3, 65536, 12288, 64  # 2.4e9 weights
    w = torch.empty(E, N, K, dtype=B, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    some = [(e, n) for e in range(E) for n in (0, 1, 40000, N - 1)]
    for e in range(E):
        w[e].normal_(generator=g)
    packed, scales = ntc.pack4(w, group=group)
    back = ntc.unpack4(packed, scales, K, group=group)
    for e, n in some:
        q, s = S.pack4(w[e, n][None], group, B)
        assert torch.equal(scales[e, n], s[0]) and torch.equal(S.nibbles(packed[e, n], K), q[0]), (e, n)
        assert torch.equal(back[e, n], S.values(packed[e, n], scales[e, n], K, group).to(B)), (e, n)
    # a number off by one anywhere, or rows that are another's, would be off by a scale or more
    for e in range(E):
        for n in range(0, N, 8192):
            part = slice(n, n + 8192)
            off = (back[e, part].float() - w[e, part].float()).abs()
            assert bool((off <= 0.52 * scales[e, part].float().repeat_interleave(group, -1) + 2.0 ** -8 * w[e, part].float().abs()).all()), (e, n)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_a_balance_loss_of_2_31_logits(ntc, score):
    """Sums over 8.4 million tokens: a lane adds n / (304 CTAs of 8 teams) = 3,450 terms in a chain, then its warps and the
    CTAs their sums, below 4,100 in all, which are off by as many roundings of 2^-24 at worst."""
    room(60)
    n, E, k = (1 << 23) + 5, 257, 2
    g = torch.Generator(device="cuda").manual_seed(3)
    l = torch.empty(n, E, dtype=B, device="cuda").normal_(generator=g)
    ids = torch.randint(0, E, (n, k), generator=g, device="cuda", dtype=torch.int32)
    ids[::5] = -1
    loss, counts, mean = ntc.balance_loss(l, ids, score=score)
    c, live = S.counts(ids, E)
    assert torch.equal(counts[:E].long(), c) and int(counts[E]) == int(live.sum())
    total = torch.zeros(E, dtype=torch.float64, device="cuda")
    step = 1 << 19
    for a in range(0, n, step):
        p, _ = S.probabilities(l[a:a + step], score)
        total += p[live[a:a + step]].sum(0)
    want = total / int(live.sum())
    R.assert_within(mean, want, want * (R.SPECIAL + 4100 * S.U32), "mean")
    exact = float(E * (c.double() * want).sum() / c.sum())
    assert abs(float(loss) - exact) <= exact * (R.SPECIAL + 4700 * S.U32)
    dloss = torch.tensor(float(n), device="cuda")
    d = ntc.balance_loss_backward(l, ids, counts, dloss=dloss, score=score)
    a_all = float(n) * E / (int(live.sum()) * int(c.sum()))
    for a in (0, 4177920, n - 300):  # 4177920 * 257 is below 2^30, the last rows are past 2^31
        part = slice(a, a + 300)
        p, _ = S.probabilities(l[part], score)
        diff = c.double() - c.double().mean()
        centred = diff - (p * diff).sum(1, keepdim=True)
        slope = torch.sigmoid(-l[part].double()) if score == "sigmoid" else torch.ones_like(p)
        w = torch.where(live[part][:, None], a_all * p * centred * slope, torch.zeros_like(p))
        off = a_all * p * slope * (centred.abs() * 3 * R.SPECIAL + (p * diff.abs()).sum(1, keepdim=True) * (2 * R.SPECIAL + (E + 8) * S.U32))
        R.assert_within(d[part], w, off + R.UNIT[B] * (w.abs() + off) + R.TINY[B], a)
