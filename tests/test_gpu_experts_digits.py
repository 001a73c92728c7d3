"""The router's fp32 results to a relative bound, where a formula's plain evaluation loses its digits."""
import pytest
import torch

import tests.experts_ref as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ntc():
    from paper_2608_27888_gb300 import ntc
    return ntc


@pytest.mark.parametrize("k", [2, 9])
def test_sigmoid_gradient_of_large_logits(ntc, k):
    """s (1 - s) dw to a relative bound where s is near 1: exp's argument is off by 2^-24 |l|, each of its few
    operations by 2^-22 at most."""
    l = torch.linspace(-40, 40, 161)[:, None].repeat(1, 12)
    ids = torch.arange(k, dtype=torch.int32).repeat(161, 1)
    dw = torch.randn(161, k, generator=torch.Generator().manual_seed(3))
    got = ntc.route_backward(l.cuda(), ids.cuda(), dw.cuda(), score="sigmoid", renormalize=False).cpu()
    d = l.double()[:, :k]
    want = 1 / (1 + torch.exp(-d)) / (1 + torch.exp(d)) * dw.double()
    R.assert_within(got[:, :k], want, want.abs() * (2.0 ** -23 * d.abs() * 2 + 2.0 ** -19))
    assert (got[:, k:] == 0).all()


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_one_choice_alone_has_no_gradient(ntc, score):
    """Renormalized over one chosen expert a weight is the scale whatever the logits are: exact zeros."""
    g = torch.Generator(device="cuda").manual_seed(4)
    l = torch.randn(4096, 16, generator=g, device="cuda") * 3
    ids, _ = ntc.route(l, 1, score=score)
    dw = torch.randn(4096, 1, generator=g, device="cuda")
    assert not ntc.route_backward(l, ids, dw, score=score).any()
    # the only one left of several: the others masked, or none
    for k in (2, 9):
        some = torch.cat([torch.full((4096, k - 1), -1, dtype=torch.int32, device="cuda"), ids], 1)
        dw = torch.randn(4096, k, generator=g, device="cuda")
        assert not ntc.route_backward(l, some, dw, score=score).any()


# Relative bounds of scores: 2^t to 2 ulp, log 2 to 2^-29 of itself times |x|, sums, quotients and products of a few
# roundings of 2^-24 each, E of them in a softmax's sum; what the logits' own difference is rounded by does not arise
# (they are whole multiples of 2^-10).
def relative(x, E):
    return 2.0 ** -22 * 3 + 2.0 ** -29 * x + E * 2.0 ** -24


@pytest.mark.parametrize("E,k", [(8, 8), (40, 12), (300, 32)])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [False, True])
def test_weights_far_from_the_largest(ntc, E, k, score, renorm):
    g = torch.Generator().manual_seed(E + k)
    l = -torch.arange(E) * (80.0 / E)
    l = (torch.round(l * 1024) / 1024)[torch.stack([torch.randperm(E, generator=g) for _ in range(50)])]
    ids, w = ntc.route(l.cuda(), k, score=score, renormalize=renorm)
    d = l.double()
    s = torch.exp(d - torch.logsumexp(d, 1, keepdim=True)) if score == "softmax" else 1 / (1 + torch.exp(-d))
    s = s.gather(1, ids.cpu().long())
    want = s / s.sum(1, keepdim=True) if renorm else s
    R.assert_within(w.cpu(), want, want * relative(80, E))


@pytest.mark.parametrize("E", [8, 40, 300])
def test_gradient_far_from_the_largest(ntc, E):
    """Softmax without renormalization: the logits that were not chosen have -s_e times one sum."""
    l = torch.round(-torch.arange(E) * (80.0 / E) * 1024).repeat(5, 1) / 1024
    ids = torch.zeros(5, 1, dtype=torch.int32)
    dw = torch.arange(1, 6)[:, None].float()
    got = ntc.route_backward(l.cuda(), ids.cuda(), dw.cuda(), renormalize=False).cpu()
    d = l.double()
    s = torch.exp(d - torch.logsumexp(d, 1, keepdim=True))
    want = -s * s[:, :1] * dw.double()
    R.assert_within(got[:, 1:], want[:, 1:], want[:, 1:].abs() * 2 * relative(80, E))
