"""The optimizer's arguments: what needs no tensor."""
import warnings

import pytest
import torch

from paper_2608_27888_gb300 import build as B

B.build()
from paper_2608_27888_gb300.optim import AdamW  # noqa: E402


def test_a_decay_that_8_bits_do_not_follow_draws_a_warning():
    for beta2 in (0.0, 0.98, 0.99):
        with pytest.warns(UserWarning, match="8 bits"):
            AdamW([], bits=8, beta2=beta2)
    with warnings.catch_warnings():
        warnings.simplefilter("error")
        AdamW([], bits=8)
        AdamW([], bits=8, beta2=0.995)
        AdamW([], bits=32, beta2=0.9)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("spoil", ["shape", "masters", "steps", "missing", "type"])
def test_a_state_that_does_not_fit_changes_nothing(bits, spoil):
    def made(fill):
        w = [torch.full((300,), fill).bfloat16(), torch.full((5,), fill)]
        opt = AdamW(w, bits=bits)
        for t in opt.m + opt.v + opt.masters + (opt.scales or []):
            t.copy_(torch.full(t.shape, fill).to(t.dtype))
        return w, opt

    w, mine = made(1.0)
    state = made(2.0)[1].state()
    if spoil == "shape":
        state["v"] = [state["v"][0], state["v"][1][:4]]
    elif spoil == "masters":
        state["masters"] = []
    elif spoil == "steps":
        state["steps"] = -1
    elif spoil == "missing":
        del state["steps"]
    else:
        state["v"] = [t.float() if bits == 8 else t.to(torch.float8_e4m3fn) for t in state["v"]]
    with pytest.raises((ValueError, KeyError)):
        mine.load(state)
    assert mine.steps == 0
    for t in w + mine.m + mine.v + mine.masters + (mine.scales or []):
        assert bool((t.float() == 1).all())
    good = made(2.0)[1].state()
    good["steps"] = 3
    mine.load(good)
    assert mine.steps == 3 and bool((w[0] == 2).all()) and bool((mine.m[1].float() == 2).all())
