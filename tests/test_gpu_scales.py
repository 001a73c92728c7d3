"""Scales as the header defines them, where a formula that looks the same has another last digit."""
import pytest
import torch

pytestmark = pytest.mark.gpu
B, F, F8 = torch.bfloat16, torch.float32, torch.float8_e4m3fn


def test_a_packed_groups_scale_is_a_product():
    """13.91796875 is 7 * 1.98828125, half way between two bf16 numbers; the fp32 product with fl(1 / 7) is above the half."""
    from paper_2608_27888_gb300 import ntc
    top = 13.91796875
    w = torch.zeros(1, 64, device="cuda")
    w[0, 3], w[0, 40] = top, -7.0
    packed, scales = ntc.pack4(w, group=32, dtype=B)
    assert scales.tolist() == [[1.9921875, 1.0]]
    assert packed.view(-1)[1] >> 4 == 15 and packed.view(-1)[20] & 15 == 1


def test_a_blocks_scale_and_codes_are_products():
    """Every power of two and a spread of significands: scale = top * fl(1 / 448), the largest's code 448."""
    from paper_2608_27888_gb300 import ntc
    g = torch.Generator(device="cuda").manual_seed(2)
    grad = torch.randn(4096, 256, generator=g, device="cuda") * torch.exp2(torch.randint(-30, 30, (4096, 1), generator=g, device="cuda").float())
    p = torch.zeros_like(grad)
    m, v = (torch.zeros_like(grad).to(F8) for _ in range(2))
    s = torch.zeros(2, 4096, device="cuda")
    ntc.adamw([p], [grad], [m], [v], scales=[s], step=1, lr=0.0, beta1=0.0, beta2=0.0)
    top = grad.abs().amax(1)  # beta 0: the moments are the gradient and its square
    by = torch.tensor(1.0 / 448.0, dtype=F, device="cuda")
    assert torch.equal(s[0], top * by)
    assert torch.equal(m.view(torch.uint8), (grad * (448.0 / top)[:, None]).to(F8).view(torch.uint8))
    largest = (m.float() * s[0][:, None]).abs().amax(1)
    assert bool(((largest - top).abs() <= 3 * 2.0 ** -24 * top).all())
    assert bool((m.float().abs().amax(1) == 448).all()) and bool((v.float().amax(1) == 448).all())
