"""The balance loss, its counts and its gradient against 64-bit references."""
import math

import pytest
import torch

import tests.experts_ref as R
import tests.train_serve_ref as S

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ntc():
    from paper_2608_27888_gb300 import ntc
    return ntc


def batch(n, E, k, dtype, seed=0, ld=None, spread=1.0):
    """Logits with masked and padded tokens, and ids some of which are no expert or repeat."""
    g = torch.Generator(device="cuda").manual_seed(seed + 1000 * n + E)
    l = torch.randn(n, ld or E, generator=g, device="cuda") * spread
    ids = torch.randint(0, E, (n, k), generator=g, device="cuda", dtype=torch.int32)
    if n > 8:
        l[1::7] = torch.where(torch.rand(l[1::7].shape, generator=g, device="cuda") < 0.3, -math.inf, l[1::7])
        l[2::11, ::2] = math.nan
        l[5::13] = -math.inf  # a token with choices and no logit
        ids[3::5] = -1        # padding
        ids[4::17, 0] = E
        ids[6::19, 0] = -2 ** 31
        ids[7::23] = 2 ** 31 - 1
        l[8::29, 0] = math.inf
    return l.to(dtype)[:, :E], ids


SIZES = [(1, 1, 1), (3, 2, 1), (33, 7, 3), (200, 8, 2), (129, 16, 4), (700, 60, 6), (1000, 64, 8), (511, 100, 9), (300, 128, 8),
         (77, 200, 32), (2000, 256, 8), (150, 300, 5), (90, 512, 10), (33, 771, 4), (1200, 1024, 8), (20000, 33, 2)]


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("n,E,k", SIZES)
def test_loss_counts_mean_and_gradient(ntc, n, E, k, dtype, score):
    l, ids = batch(n, E, k, dtype)
    loss, counts, mean = ntc.balance_loss(l, ids, score=score, scale=0.75)
    want, c, m, b_loss, b_mean = S.balance_loss(l, ids, score, 0.75)
    assert torch.equal(counts, c)
    R.assert_within(mean, m, b_mean, "mean")
    assert loss.shape == () and abs(float(loss) - want) <= b_loss
    dloss = torch.tensor(float(n), device="cuda")
    got = ntc.balance_loss_backward(l, ids, counts, dloss=dloss, score=score, scale=0.75)
    g, bound = S.balance_loss_backward(l, ids, score, 0.75, float(n))
    assert got.dtype == dtype and got.shape == (n, E)
    R.assert_within(got, g, bound, "dlogits")
    res = torch.randn(n, E, device="cuda").to(dtype)
    got = ntc.balance_loss_backward(l, ids, counts, dloss=dloss, score=score, scale=0.75, residual=res)
    g, bound = S.balance_loss_backward(l, ids, score, 0.75, float(n), res)
    R.assert_within(got, g, bound, "with residual")


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("shift", [-3000.0, -95.0, -40.0, 40.0, 3000.0])
def test_rows_far_from_zero(ntc, score, shift):
    """p is a ratio: it has its digits wherever the row lies (a sigmoid's there: all 1, or exp(l) of one another)."""
    l, ids = batch(300, 24, 3, torch.float32, seed=5, spread=4.0)
    l = torch.where(torch.isfinite(l), l + shift, l)
    loss, counts, mean = ntc.balance_loss(l, ids, score=score)
    want, _, m, b_loss, b_mean = S.balance_loss(l, ids, score)
    R.assert_within(mean, m, b_mean, "mean")
    assert abs(float(loss) - want) <= b_loss
    R.assert_within(ntc.balance_loss_backward(l, ids, counts, score=score), *S.balance_loss_backward(l, ids, score), "dlogits")


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
def test_strides_and_alignments(ntc, dtype):
    for E, ld, at in [(64, 72, 0), (64, 65, 0), (64, 80, 1), (100, 104, 4), (256, 264, 3), (16, 17, 1)]:
        l, ids = batch(400, E, 4, dtype, ld=ld + at)
        big = torch.full((400, ld + at), math.nan, dtype=dtype, device="cuda")
        big[:, at:at + E] = l
        l = big[:, at:at + E]
        res = torch.randn(400, ld + at, device="cuda").to(dtype)[:, at:at + E]
        loss, counts, mean = ntc.balance_loss(l, ids)
        want, c, m, b_loss, b_mean = S.balance_loss(l, ids)
        assert torch.equal(counts, c) and abs(float(loss) - want) <= b_loss
        R.assert_within(mean, m, b_mean, (E, ld, at))
        R.assert_within(ntc.balance_loss_backward(l, ids, counts, residual=res), *S.balance_loss_backward(l, ids, residual=res), (E, ld, at))


def test_nothing_to_count(ntc):
    for n in (0, 1, 100, 5000):
        l = torch.randn(n, 40, device="cuda")
        ids = torch.full((n, 2), -1, dtype=torch.int32, device="cuda")
        loss, counts, mean = ntc.balance_loss(l, ids)
        assert float(loss) == 0 and not counts.any() and not mean.any()
        res = torch.randn(n, 40, device="cuda")
        assert not ntc.balance_loss_backward(l, ids, counts).any()
        assert torch.equal(ntc.balance_loss_backward(l, ids, counts, residual=res), res)


def test_an_even_load_has_no_gradient(ntc):
    l = torch.randn(64, 16, device="cuda") * 9
    ids = (torch.arange(128, device="cuda", dtype=torch.int32) % 16).view(64, 2)
    loss, counts, _ = ntc.balance_loss(l, ids, scale=3.0)
    assert abs(float(loss) - 3.0) < 1e-4 and not ntc.balance_loss_backward(l, ids, counts).any()
    one = torch.randn(50, 1, device="cuda")
    assert not ntc.balance_loss_backward(one, torch.zeros(50, 1, dtype=torch.int32, device="cuda"),
                                         torch.tensor([50, 50], dtype=torch.int32, device="cuda")).any()


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_gradient_against_differences(ntc, score):
    """Central differences of the loss itself, h = 2^-5.  n' = 4 and E = 8 with c / C <= 1: the third derivative of the
    loss along one logit is at most E / n' times that of a probability, which is below 1: 2 h^2 / 6 = 3.3e-4; the two losses
    (below 8) are off by 2^-19 of themselves at most, which is the same for both but for the changed token's share:
    2 * 8 * 2^-20 / (2 h) = 2.4e-4."""
    h, g = 2.0 ** -5, torch.Generator(device="cuda").manual_seed(3)
    l = torch.randn(4, 8, generator=g, device="cuda")
    ids = torch.tensor([[0, 1], [0, 2], [0, 5], [1, 0]], dtype=torch.int32, device="cuda")
    counts = ntc.balance_loss(l, ids, score=score)[1]
    got = ntc.balance_loss_backward(l, ids, counts, score=score)
    for t in range(4):
        for e in range(8):
            up, down = l.clone(), l.clone()
            up[t, e] += h
            down[t, e] -= h
            d = (float(ntc.balance_loss(up, ids, score=score)[0]) - float(ntc.balance_loss(down, ids, score=score)[0])) / (2 * h)
            assert abs(d - float(got[t, e])) <= 6e-4


def test_streams_graphs_and_equal_bits(ntc):
    l, ids = batch(9000, 96, 6, torch.bfloat16)
    first = ntc.balance_loss(l, ids)
    back = ntc.balance_loss_backward(l, ids, first[1])
    for _ in range(3):
        again = ntc.balance_loss(l, ids)
        assert all(torch.equal(a, b) for a, b in zip(first, again))
        assert torch.equal(back, ntc.balance_loss_backward(l, ids, first[1]))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = ntc.balance_loss(l, ids, stream=side)
    d = ntc.balance_loss_backward(l, ids, other[1], stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, other)) and torch.equal(back, d)
    # two graphs at once, replayed on new inputs
    pair = [(l.clone(), ids.clone()), (l.flip(0).contiguous(), ids.flip(0).contiguous())]
    graphs, outs = [], []
    for x, i in pair:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            r = ntc.balance_loss(x, i, score="sigmoid")
            outs.append(r + (ntc.balance_loss_backward(x, i, r[1], score="sigmoid"),))
        graphs.append(g)
    for x, i in pair:
        x.copy_(x.flip(1).clone())
        i.copy_((i + 1) % 96)
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for s, g in zip((a, b), graphs):
        with torch.cuda.stream(s):
            g.replay()
    torch.cuda.synchronize()
    for (x, i), got in zip(pair, outs):
        want = ntc.balance_loss(x, i, score="sigmoid")
        assert all(torch.equal(p, q) for p, q in zip(got, want + (ntc.balance_loss_backward(x, i, want[1], score="sigmoid"),)))


def test_what_is_refused(ntc):
    z = lambda *s, dtype=torch.float32: torch.zeros(*s, dtype=dtype, device="cuda")  # noqa: E731
    I = torch.int32
    for call, word in [
            (lambda: ntc.balance_loss(z(4), z(4, 1, dtype=I)), "two dimensions"),
            (lambda: ntc.balance_loss(z(4, 8), z(4, 1)), "must be Int"),
            (lambda: ntc.balance_loss(z(4, 8), z(3, 1, dtype=I)), "shape"),
            (lambda: ntc.balance_loss(z(4, 8), z(4, 4, dtype=I)[:, ::2]), "contiguous"),
            (lambda: ntc.balance_loss(z(8, 4).t(), z(4, 1, dtype=I)), "last dimension"),
            (lambda: ntc.balance_loss(z(4, 8, dtype=torch.float64), z(4, 1, dtype=I)), "float32, float16 or bfloat16"),
            (lambda: ntc.balance_loss(z(4, 8), z(4, 1, dtype=I), score="tanh"), "score must be"),
            (lambda: ntc.balance_loss(torch.zeros(4, 8), z(4, 1, dtype=I)), "CUDA tensor"),
            (lambda: ntc.balance_loss_backward(z(4, 8), z(4, 1, dtype=I), z(8, dtype=I)), "shape"),
            (lambda: ntc.balance_loss_backward(z(4, 8), z(4, 1, dtype=I), z(9, dtype=I), dloss=z(2)), "one element"),
            (lambda: ntc.balance_loss_backward(z(4, 8), z(4, 1, dtype=I), z(9, dtype=I), residual=z(4, 9)), "shape")]:
        with pytest.raises(ValueError, match=word):
            call()
    for call, word in [(lambda: ntc.balance_loss(z(4, 8), z(4, 33, dtype=I)), "top_k"),
                       (lambda: ntc.balance_loss(z(4, 1025), z(4, 1, dtype=I)), "num_experts"),
                       (lambda: ntc.balance_loss(z(4, 8), z(4, 1, dtype=I), scale=math.nan), "scale")]:
        with pytest.raises(ntc.NtcError, match=word):
            call()
