"""A layer of routed experts as a whole: its gradients against 64-bit autograd, and the example that trains one."""
import importlib.util
import os

import pytest
import torch

import tests.experts_ref as R

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("T,D,H,O,E,k,score", [(1, 16, 128, 8, 4, 2, "softmax"), (300, 64, 96, 40, 6, 3, "sigmoid"),
                                               (1000, 33, 70, 9, 16, 2, "softmax")])
def test_gradients_of_the_layer(T, D, H, O, E, k, score):
    """Forward and backward against 64-bit autograd through the same choice.

    Between the calls bf16 tensors are rounded four times (h, y; dy, dh or dlogits), each relative 2^-8 per element; a
    norm over many elements sees at most their sum, 2^-6, plus the results' own rounding: 2^-5 is allowed."""
    from paper_2608_27888_gb300.routed import RoutedExperts
    g = torch.Generator(device="cuda").manual_seed(T)
    layer = RoutedExperts(D, H, O, E, k, score=score, generator=g)
    layer.b1.normal_(generator=g)
    layer.b2.normal_(generator=g)
    layer.router_bias.normal_(generator=g)
    x = torch.randn(T, D, generator=g, device="cuda").bfloat16()
    res = torch.randn(T, O, generator=g, device="cuda").bfloat16()
    dout = torch.randn(T, O, generator=g, device="cuda").bfloat16()
    out, kept = layer.forward(x, res, keep=True)
    grads, dx = layer.backward(dout, kept)
    ids = kept[2].long()

    p = {n: getattr(layer, n).double().requires_grad_() for n in layer.NAMES}
    xd = x.double().requires_grad_()
    logits = xd @ p["router"].t() + p["router_bias"]
    # the logits that the choice and its weights saw were rounded to bf16: straight through
    logits = logits + (kept[1].double() - logits).detach()
    w = R.route_weights(logits, ids, score, True, 1.0)
    want = res.double()
    for j in range(k):
        e = ids[:, j]
        z = torch.einsum("td,thd->th", xd, p["w1"][e]) + p["b1"][e]
        h = z * torch.sigmoid(z)
        want = want + w[:, j, None] * (torch.einsum("th,toh->to", h, p["w2"][e]) + p["b2"][e])
    want.backward(dout.double())

    def close(a, b, what):
        assert float((a.double() - b).norm()) <= 2.0 ** -5 * float(b.norm()), what
    close(out, want.detach(), "out")
    close(dx, xd.grad, "dx")
    for n in layer.NAMES:
        assert grads[n].shape == getattr(layer, n).shape, n
        close(grads[n], p[n].grad, n)


def test_the_example_learns():
    spec = importlib.util.spec_from_file_location("routed_decoders", os.path.join(ROOT, "examples", "routed_decoders.py"))
    ex = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(ex)
    layer, first, last, x, target = ex.train(steps=60, log=None)
    assert last < 0.5 * first
    load = torch.zeros(layer.num_experts)
    _, kept = layer.forward(x[:4096], keep=True)
    offsets = kept[6].cpu()
    load = offsets[1:] - offsets[:-1]
    assert int(load.sum()) == 4096 * layer.top_k
