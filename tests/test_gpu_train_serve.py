"""A routed layer trained and served: the balance loss in its gradients, its optimizer, its weights in 4 bits, together."""
import importlib.util
import os

import pytest
import torch

import tests.experts_ref as R
import tests.train_serve_ref as S

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def layer_of(T, D, H, O, E, k, score="softmax"):
    from paper_2608_27888_gb300.routed import RoutedExperts
    g = torch.Generator(device="cuda").manual_seed(T)
    layer = RoutedExperts(D, H, O, E, k, score=score, generator=g)
    for b in (layer.b1, layer.b2, layer.router_bias):
        b.normal_(generator=g)
    return layer, torch.randn(T, D, generator=g, device="cuda").bfloat16(), g


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_the_layer_adds_the_balance_losss_gradient(score):
    """The logits' gradient with the balance loss, through the router: the router bias' gradient is its column sum."""
    from paper_2608_27888_gb300 import ntc
    layer, x, g = layer_of(700, 48, 64, 24, 8, 2, score)
    out, kept = layer.forward(x, keep=True)
    dout = torch.randn(out.shape, generator=g, device="cuda").bfloat16()
    plain, _ = layer.backward(dout, kept)
    both, _ = layer.backward(dout, kept, balance=200.0)
    loss, counts, mean = layer.balance_loss(kept)
    want, c, _, b_loss, _ = S.balance_loss(kept[1], kept[2], score)
    assert abs(float(loss) - want) <= b_loss and torch.equal(counts, c)
    d, _ = S.balance_loss_backward(kept[1], kept[2], score, 200.0)
    # a logit's gradient is rounded to bf16 twice at most, in either call: 2^-7 of its parts' magnitudes
    dy, dweights = ntc.combine_backward(dout, kept[9], kept[5], kept[3], kept[6])
    first = ntc.route_backward(kept[1], kept[2], dweights, score=score).double()
    bound = (2.0 ** -7 * (first.abs() + d.abs())).sum(0) + 1e-6
    R.assert_within(both["router_bias"], plain["router_bias"].double() + d.sum(0), bound)
    assert torch.equal(both["w1"], plain["w1"]) and torch.equal(both["b2"], plain["b2"])


@pytest.mark.parametrize("T,D,H,O,E,k", [(1, 16, 128, 9, 4, 2), (60, 100, 70, 33, 8, 2), (900, 64, 96, 40, 6, 3)])
def test_a_packed_layer_is_the_layer_of_its_weights(T, D, H, O, E, k):
    """Against the same layer with the unpacked weights: h and y are rounded to bf16 at other last digits (2^-8 each), the
    unpacked weights once (2^-9 each on average, 2^-8 at most): as norms 2^-6 is above their sum."""
    from paper_2608_27888_gb300 import ntc
    layer, x, g = layer_of(T, D, H, O, E, k)
    served = layer.pack4(group=32)
    res = torch.randn(T, O, generator=g, device="cuda").bfloat16()
    out = served.forward(x, res)
    layer.w1 = ntc.unpack4(served.w1, served.s1, D, group=32)
    layer.w2 = ntc.unpack4(served.w2, served.s2, H, group=32)
    want = layer.forward(x, res)
    assert float((out.double() - want.double()).norm()) <= 2.0 ** -6 * float(want.double().norm())


@pytest.mark.parametrize("bits", [32, 8])
def test_steps_of_a_layer_in_a_graph(bits):
    """Forward, backward with the balance loss and the optimizer's step as one graph: its replays are the steps of calls."""
    from paper_2608_27888_gb300.optim import AdamW
    runs = []
    for captured in (False, True):
        layer, x, g = layer_of(300, 24, 48, 12, 6, 2)
        target = torch.randn(300, 12, generator=g, device="cuda")
        adam = AdamW(layer.parameters(), lr=0.01, bits=bits, captured=captured)

        def step():
            out, kept = layer.forward(x, keep=True)
            grads, _ = layer.backward(((out.float() - target) / out.numel()).to(out.dtype), kept, balance=0.01)
            adam.step(grads)
        step()
        if captured:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                step()
            for _ in range(5):
                graph.replay()
        else:
            for _ in range(5):
                step()
        torch.cuda.synchronize()
        runs.append([p.clone() for p in layer.parameters().values()])
    assert all(torch.equal(a, b) for a, b in zip(*runs))


def test_the_example_runs_in_8_bits_and_packs():
    spec = importlib.util.spec_from_file_location("routed_decoders", os.path.join(ROOT, "examples", "routed_decoders.py"))
    ex = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(ex)
    layer, first, last, x, target = ex.train(steps=6, log=None, bits=8, batch=1024)
    out = layer.pack4(group=32).forward(x[:500])
    assert out.shape == (500, target.shape[1]) and bool(torch.isfinite(out).all())
