"""The activations and their slopes far from 0, to bounds that see an error in their tails.

z comes through the bias, exactly (the product is 0); the slope through db, which is fp32: dy is 1 and a column has one row.
"""
import math

import pytest
import torch

import tests.experts_ref as R

pytestmark = pytest.mark.gpu

PHI = 7.5e-8  # half of what the formula for erf is off by


def z_of(n):
    return torch.cat([torch.linspace(-14, 10, n), torch.tensor([0.0, -0.0, -40.0, -80.0, 60.0])]).cuda()


def phi(z):
    return 0.5 * torch.special.erfc(-z * math.sqrt(0.5))


@pytest.fixture(scope="module")
def ntc():
    from paper_2608_27888_gb300 import ntc
    return ntc


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows", [3, 40])
def test_activations(ntc, dtype, rows):
    z = z_of(4003)
    x, w = torch.zeros(rows, 8, dtype=dtype, device="cuda"), torch.zeros(z.numel(), 8, dtype=dtype, device="cuda")
    d, u, tiny = z.double(), R.UNIT[dtype], R.TINY[dtype]
    # Phi: the formula's error and its value's roundings, eight of them
    want = d * phi(d)
    y = ntc.linear(x, w, z, activation="gelu")
    R.assert_within(y, want.expand(rows, -1), (d.abs() * (PHI + 8 * R.F32 * phi(d)) + u * want.abs() * 1.01 + tiny).expand(rows, -1))
    # exp's argument is rounded, relative 2^-24 |z| of the result, besides a few roundings
    want = d / (1 + torch.exp(-d))
    y = ntc.linear(x, w, z, activation="silu")
    off = want.abs() * (2.0 ** -23 * d.abs() + 8 * R.F32)
    R.assert_within(y, want.expand(rows, -1), (off + u * want.abs() * 1.01 + tiny).expand(rows, -1))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_slopes(ntc, dtype):
    z = z_of(4003).to(dtype)
    n = z.numel()
    x, w = torch.zeros(1, 8, dtype=dtype, device="cuda"), torch.zeros(n, 8, dtype=dtype, device="cuda")
    dy = torch.ones(1, n, dtype=dtype, device="cuda")
    d = z.double()
    density = torch.exp(-d * d / 2) / math.sqrt(2 * math.pi)
    want = phi(d) + d * density
    got = ntc.linear_backward(dy, x, w, z=z[None], activation="gelu", need=("db",))[2]
    # the density's exponent is rounded twice, relative 2^-23 z^2 / 2 of it
    R.assert_within(got, want, PHI + R.F32 * (8 * phi(d) + d.abs() * density * (8 + d * d)) + 1e-37)
    s = 1 / (1 + torch.exp(-d))
    want = s * (1 + d * (1 - s))
    got = ntc.linear_backward(dy, x, w, z=z[None], activation="silu", need=("db",))[2]
    # s is off by 2^-23 |z| of itself; 1 - s by 2^-23, times z
    R.assert_within(got, want, R.F32 * (s * (1 + d.abs()) * (8 + 2 * d.abs())) + 1e-37)
