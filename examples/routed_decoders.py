"""Many decoders distilled into a few routed experts.

The teacher is the framework's own decode: a G-buffer's queries, each through the
decoder of its texture set.  The student sees the same latent features and no set id:
a layer of routed experts learns which expert decodes what.  After the training steps
the student decodes a batch through a CUDA graph, as a renderer would replay it.

    python examples/routed_decoders.py [--steps 200] [--experts 8] [--top-k 2]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2608_27888_gb300 import ntc, workloads as W  # noqa: E402
from paper_2608_27888_gb300.routed import RoutedExperts  # noqa: E402


def teacher(name="gbuffer-1080p"):
    """Features [n, in] and channels [n, out] of the workload's queries."""
    w = W.named(name, "small")
    dec = ntc.Decoder(w.assets, "fp16")
    q = ntc.queries_to_device(w.queries)
    x, y = dec.features(q), dec.decode(q)
    dec.close()
    return x.to(torch.bfloat16), y


def train(steps=200, experts=8, top_k=2, hidden=128, batch=8192, rate=0.02, seed=0, log=print):
    """The trained layer and the mean squared error before and after."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    x, target = teacher()
    layer = RoutedExperts(x.shape[1], hidden, target.shape[1], experts, top_k, generator=g)
    master = {n: getattr(layer, n).float() for n in layer.NAMES}  # fp32 copies that the steps add up in
    moment = {n: (torch.zeros_like(p), torch.zeros_like(p)) for n, p in master.items()}
    errors = []
    for step in range(1, steps + 1):
        at = torch.randint(0, x.shape[0], (batch,), generator=g, device="cuda")
        out, kept = layer.forward(x[at], keep=True)
        diff = out.float() - target[at]
        grads, _ = layer.backward((diff * (2.0 / diff.numel())).to(out.dtype), kept)
        for n, p in master.items():  # Adam
            m, v = moment[n]
            d = grads[n].float()
            m.mul_(0.9).add_(d, alpha=0.1)
            v.mul_(0.99).addcmul_(d, d, value=0.01)
            p.sub_(rate * (m / (1 - 0.9 ** step)) / ((v / (1 - 0.99 ** step)).sqrt() + 1e-8))
            getattr(layer, n).copy_(p)
        layer.balance(kept[6])
        errors.append(diff.square().mean())
        if log and step % 50 == 1:
            log(f"step {step:4d}  mean squared error {float(errors[-1]):.5f}")
    ntc.ntc_linear_status(torch.cuda.current_stream().cuda_stream)
    return layer, float(errors[0]), float(torch.stack(errors[-10:]).mean()), x, target


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--experts", type=int, default=8)
    ap.add_argument("--top-k", type=int, default=2)
    a = ap.parse_args()
    layer, first, last, x, target = train(a.steps, a.experts, a.top_k)
    print(f"mean squared error {first:.5f} -> {last:.5f} after {a.steps} steps")

    batch = x[:4096].clone()
    layer.forward(batch)  # first use of every kernel, outside the capture
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = layer.forward(batch)
    start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    start.record()
    for _ in range(100):
        graph.replay()
    end.record()
    torch.cuda.synchronize()
    print(f"{batch.shape[0]} texels decoded in {start.elapsed_time(end) * 10:.1f} us a pass, "
          f"error {float((out.float() - target[:4096]).square().mean()):.5f}")


if __name__ == "__main__":
    main()
