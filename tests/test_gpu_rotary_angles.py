"""Angles of rotary positions, far out and near half a turn, against decimal arithmetic of 60 digits.

A coefficient is off by: sincospif 2 units in the last place (2^-23 near 1), what the fraction's float lost put right (a fused product and sum, 2^-25), the
amplitude's product (2^-25); two products and a sum of values below |a| + |b| add 2^-23; together below 3.1e-7 (|a| + |b|).  The angle is off by
|position| * 2^-62 + 2^-32 turns (on the ramp of the scaling by parts times fast / (fast - slow), here below 1.1)."""
import math
from decimal import Decimal, getcontext

import pytest
import torch

pytestmark = pytest.mark.gpu

getcontext().prec = 60
TWO_PI = 2 * Decimal("3.14159265358979323846264338327950288419716939937510582097494459")


@pytest.fixture(scope="module")
def B():
    from paper_2501_17086_b200 import binding
    return binding


def turns_of(r, base, scaling="none", factor=1.0, trained_length=0.0, fast=32.0, slow=1.0):
    out = []
    for i in range(r // 2):
        f = (Decimal(base).ln() * (Decimal(-2 * i) / r)).exp()
        if scaling == "linear":
            f /= Decimal(factor)
        if scaling == "by_parts":
            w = (Decimal(trained_length) * f / TWO_PI - Decimal(slow)) / (Decimal(fast) - Decimal(slow))
            w = min(Decimal(1), max(Decimal(0), w))
            f *= w + (1 - w) / Decimal(factor)
        out.append(f / TWO_PI)
    return out


def angles(positions, turns):
    """Radians from -pi to pi [positions, pairs], as doubles."""
    out = []
    for p in positions:
        out.append([float(((p * t) % 1 - (0 if (p * t) % 1 < Decimal("0.5") else (1 if p * t > 0 else -1))) * TWO_PI) for t in turns])
    return torch.tensor(out, dtype=torch.float64)


@pytest.mark.parametrize("r,base,scaling", [(64, 10000.0, {}), (80, 10000.0, {}), (128, 500000.0, {}), (256, 1.5, {}), (2, 10000.0, {}),
                                            (64, 10000.0, dict(scaling="linear", factor=8.0)),
                                            (96, 10000.0, dict(scaling="by_parts", factor=16.0, trained_length=4096.0))])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_far_positions(B, r, base, scaling, layout):
    """Up to 2^36: a frequency of 53 digits would be off by 4e-6 radians there."""
    g = torch.Generator().manual_seed(r)
    pos = [0, 1, -1, (1 << 36) - 1, -(1 << 36) + 5, 1 << 35, 123456789012 % (1 << 36)]
    pos += torch.randint(0, 1 << 36, (20,), generator=g).tolist() + torch.randint(0, 1 << 20, (20,), generator=g).tolist()
    x = torch.randn(len(pos), 3, max(r, 4), generator=g)  # (no head is narrower than 4)
    got, _ = B.rotary(x.cuda(), positions=torch.tensor(pos, dtype=torch.int64).cuda(), base=base, layout=layout, rotary_dim=r, **scaling)
    a = angles(pos, turns_of(r, base, **scaling))[:, None]
    first, second = (slice(0, r // 2), slice(r // 2, r)) if layout == "half" else (slice(0, r, 2), slice(1, r, 2))
    u, v = x.double()[..., first], x.double()[..., second]
    off = 3.1e-7 + 2 * math.pi * 1.1 * (torch.tensor(pos, dtype=torch.float64).abs()[:, None, None] * 2.0 ** -62 + 2.0 ** -32)
    bound = off * (u.abs() + v.abs())
    got = got.double().cpu()
    for y, want in ((got[..., first], u * a.cos() - v * a.sin()), (got[..., second], v * a.cos() + u * a.sin())):
        over = (y - want).abs() - bound
        assert float(over.max()) <= 0, float(over.max())


def test_sines_of_angles_near_half_a_turn(B):
    """(1, 0) turned by nearly pi: the sine is small, and what it is off by is small too: 2 units in its last place, the fraction's 2^-32 turns and the
    products' share (|sine| 2^-22, and 2^-25 of what the float had lost)."""
    pos = [p for p in range(1, 1 << 16) if abs(p % (2 * math.pi) - math.pi) < 0.01][:400]
    a = angles(pos, turns_of(2, 10000.0))[:, 0]
    x = torch.zeros(len(pos), 1, 8)
    x[..., 0] = 1
    got, _ = B.rotary(x.cuda(), positions=torch.tensor(pos, dtype=torch.int32).cuda(), rotary_dim=2)
    off = (got[:, 0, 1].double().cpu() - a.sin()).abs()
    assert float((off - a.sin().abs() * 2.0 ** -22 - 2 * math.pi * 2.0 ** -32 - 2.0 ** -50).max()) <= 0, float(off.max())
