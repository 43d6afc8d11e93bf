"""GELU and its slope where they are small: relative to their values, z from -13 to -1/2.

bf16: the distribution's tail is off by 1e-4 of itself (its polynomial 9e-5, the rest float arithmetic: exponent z^2 / 2 * 2^-22, reciprocal, products and
sums 2^-19); the slope z e^(-z^2/2) / sqrt(2 pi) + tail loses at most a factor of 1.25 for z <= -3 (tail <= e^.. / (sqrt(2 pi) |z|)); then a rounding to
the type.  Float: erfcf's argument is off by 2 units of 2^-24 of itself, which is z^2 + 2 times that of the tail, erfcf by 4 units in the last place, the
exponential by z^2 / 2 * 2^-23 and 2 units, products and sums by 2^-24 each: (2 z^2 + 20) 2^-24, times 1.25."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.bfloat16]


@pytest.fixture(scope="module")
def B():
    from paper_2501_17086_b200 import binding
    return binding


def gelu_of(z):
    z = z.double()
    tail = 0.5 * torch.special.erfc(-z / math.sqrt(2))
    return z * tail, tail + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)


def relative(z, dtype):
    z = z.double()
    return torch.full_like(z, 2e-4) if dtype == torch.bfloat16 else 1.25 * (2 * z * z + 20) * 2.0 ** -24


def within(got, want, rel, dtype):
    half = torch.finfo(dtype).eps / 2
    over = (got.double() - want).abs() / want.abs() - (rel + half * (1 + rel))
    assert float(over.max()) <= 0, (float(over.max()), int(over.argmax()))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("lo,hi", [(-6.0, -3.0), (-13.0, -6.0), (-3.0, -0.5)])
def test_gelu_of_values_far_below_zero(B, dtype, lo, hi):
    z = torch.linspace(lo, hi, 64 * 512, device="cuda").view(64, 512).to(dtype)
    act, _, _ = B.checkpoint_gelu(z)
    within(act, gelu_of(z)[0], relative(z, dtype), dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("lo,hi", [(-6.0, -3.0), (-13.0, -6.0)])
def test_slope_and_gelu_of_what_was_kept(B, dtype, lo, hi):
    z = torch.linspace(lo, hi, 64 * 512, device="cuda").view(64, 512).to(dtype)
    codes, scales = B.checkpoint_store(z)
    z8 = B.checkpoint_load(codes, scales, torch.float32)
    g = torch.exp2(torch.arange(64 * 512, device="cuda").view(64, 512) % 5 - 2.0).to(dtype)  # (exact products)
    dz, act = B.checkpoint_gelu_backward(g, codes, scales, with_act=True)
    want, slope = gelu_of(z8)
    rel = relative(z8, dtype)
    within(act, want, rel, dtype)
    within(dz, g.double() * slope, rel, dtype)


@pytest.mark.parametrize("dtype", TYPES)
def test_ends_of_the_range(B, dtype):
    z = torch.zeros(1, 32, device="cuda")
    z[0, :12] = torch.tensor([0.0, -0.0, 40.0, -40.0, 1e30, -1e30, 2.0 ** -100, -2.0 ** -100, 14.0, -14.0, -13.5, 1.0])
    act, _, _ = B.checkpoint_gelu(z.to(dtype))
    z = z.to(dtype).double()
    want = z * torch.special.ndtr(z)
    half = torch.finfo(dtype).eps / 2
    assert bool(((act.double() - want).abs() <= (half + 1e-6) * want.abs() + 2e-38).all())
