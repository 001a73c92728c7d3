"""Linear layers whose rows are shorter than a 16-byte piece, at every address: the copies that their products read."""
import pytest
import torch

import tests.experts_ref as R

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("K", [1, 2, 3, 5, 6, 7])
@pytest.mark.parametrize("skip,gap", [(0, 0), (1, 0), (4, 1), (3, 3)])
@pytest.mark.parametrize("gather", [False, True])
def test_narrow_inputs(K, skip, gap, gather):
    from paper_2608_27888_gb300 import ntc
    g = torch.Generator(device="cuda").manual_seed(K * 100 + skip * 10 + gap)
    T, N, E = 150, 24, 3

    def view(t):  # its rows `gap` apart, `skip` elements past 16 bytes, NaN around and between them
        n = t.numel() // K
        flat = torch.full((skip + n * (K + gap) + 16,), float("nan"), dtype=t.dtype, device="cuda")
        out = flat[skip:skip + n * (K + gap)].view(*t.shape[:-1], K + gap)[..., :K]
        out.copy_(t)
        return out
    x = torch.randn(T, K, generator=g, device="cuda").bfloat16()
    w = torch.randn(E, N, K, generator=g, device="cuda").bfloat16()
    rows = torch.randint(-1, T + 1, (T,), generator=g, device="cuda").int() if gather else None
    dy = torch.randn(T, N, generator=g, device="cuda").bfloat16()
    offsets = torch.tensor([0, 60, 60, 140], dtype=torch.int32, device="cuda")
    y, _, bound, _ = R.linear(x, w, None, rows, offsets)
    R.assert_within(ntc.linear(view(x), view(w), rows=rows, offsets=offsets), y, bound, "y")
    got = ntc.linear_backward(dy, view(x), view(w), rows=rows, offsets=offsets)
    for name, a, (ref, bound) in zip(("dx", "dw", "db"), got, R.linear_backward(dy, x, w, None, rows, offsets, "none")):
        R.assert_within(a, ref, bound, name)
    ntc.ntc_linear_status(0)
