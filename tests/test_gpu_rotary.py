"""Rotary positions against the rotation in 64 bits.  Bounds: the fraction of a turn is rounded to float (2^-26 turns, 9.4e-8
radians), sine and cosine are off by 2 units in the last place (2.4e-7 together with the amplitude's product), and the two products
and their sum by 2^-24 each: below 6e-7 * amplitude * (|a| + |b|); then one rounding to the type.  The angle itself is a double:
its frequency (here exp of up to 10 in magnitude, there pow and a division) and its product are off by at most 16 * 2^-53 of it on both sides
together, which counts from positions of some 2^30 on (2^40 radians: 2e-3)."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2501_17086_b200 import binding
    return binding


HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def reference(x, pos, r, layout="half", base=10000.0, scaling="none", factor=1.0, trained_length=0.0, fast=32.0, slow=1.0, amplitude=1.0,
              inverse=False):
    """(the turned tensor, what bounds the float part of its error) in 64 bits."""
    x = x.double()
    i = torch.arange(r // 2, dtype=torch.float64, device=x.device)
    f = torch.exp(-2 * i / r * math.log(base))
    if scaling == "linear":
        f = f / factor
    if scaling == "by_parts":
        w = ((trained_length * f / (2 * math.pi) - slow) / (fast - slow)).clamp(0, 1)
        f = f * (w + (1 - w) / factor)
    # float parameters reach the library as float
    angle = pos.double()[:, None] * f
    c, s = (amplitude * angle.cos())[:, None], (amplitude * angle.sin())[:, None] * (-1 if inverse else 1)
    y, bound = x.clone(), torch.zeros_like(x)
    first, second = (slice(0, r // 2), slice(r // 2, r)) if layout == "half" else (slice(0, r, 2), slice(1, r, 2))
    a, b = x[..., first], x[..., second]
    y[..., first], y[..., second] = a * c - b * s, b * c + a * s
    bound[..., first] = bound[..., second] = (6e-7 + 2.0 ** -49 * angle.abs()[:, None]) * amplitude * (a.abs() + b.abs())
    return y, bound


def check(got, x, pos, r, **kw):
    y, bound = reference(x, pos, r, **kw)
    off = (got.double() - y).abs()
    # the value that is rounded is itself off by the bound
    over = float((off - bound - HALF[x.dtype] * (y.abs() + bound)).max())
    assert over <= 0, over


def make(rows, heads, hd, dtype, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(rows, heads, hd, generator=g, device="cuda").to(dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("rows,qh,kh,hd,r", [(1, 1, 1, 64, 64), (7, 3, 1, 64, 32), (133, 8, 2, 128, 128), (65, 5, 5, 80, 24), (31, 2, 1, 8, 2),
                                             (1000, 12, 12, 64, 64), (17, 33, 3, 256, 256), (3, 4, 4, 136, 40), (64, 1, 1, 16, 6)])
def test_rotation(B, dtype, layout, rows, qh, kh, hd, r):
    q, k = make(rows, qh, hd, dtype, 1), make(rows, kh, hd, dtype, 2)
    pos = torch.randint(-1000, 300000, (rows,), device="cuda", dtype=torch.int64)
    for inverse in (False, True):
        qo, ko = B.rotary(q, k, positions=pos, rotary_dim=r, layout=layout, inverse=inverse)
        check(qo, q, pos, r, layout=layout, inverse=inverse)
        check(ko, k, pos, r, layout=layout, inverse=inverse)
        assert torch.equal(qo[..., r:], q[..., r:]) and torch.equal(ko[..., r:], k[..., r:])


@pytest.mark.parametrize("scaling", [dict(scaling="linear", factor=8.0),
                                     dict(scaling="by_parts", factor=16.0, trained_length=4096.0, amplitude=1.25),
                                     dict(scaling="by_parts", factor=4.0, trained_length=512.0, fast=16.0, slow=2.0)])
def test_scaled_positions(B, scaling):
    q = make(129, 3, 96, torch.float32)
    pos = torch.arange(129, device="cuda", dtype=torch.int32) * 8191
    got, none = B.rotary(q, positions=pos, base=500000.0, **scaling)
    assert none is None
    check(got, q, pos, 96, base=500000.0, **scaling)


def test_positions_counted_and_positions_far_away(B):
    q = make(50, 2, 64, torch.float32)
    at = torch.arange(50, device="cuda")
    check(B.rotary(q)[0], q, at, 64)
    check(B.rotary(q, first=1 << 40)[0], q, (1 << 40) + at, 64)
    check(B.rotary(q, first=5, period=7)[0], q, 5 + at % 7, 64)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_parts_of_one_buffer_in_place(B, dtype):
    """Queries and keys of a [rows][3 d] buffer, turned in place; the values beside them and the rows behind stay as they were."""
    rows, heads, hd = 77, 4, 64
    buf = make(rows + 3, 3 * heads, hd, dtype)
    was = buf.clone()
    q, k = buf[:rows, :heads], buf[:rows, heads:2 * heads]
    B.rotary(q, k, period=32, q_out=q, k_out=k)
    pos = torch.arange(rows, device="cuda") % 32
    check(q, was[:rows, :heads], pos, hd)
    check(k, was[:rows, heads:2 * heads], pos, hd)
    assert torch.equal(buf[rows:], was[rows:]) and torch.equal(buf[:, 2 * heads:], was[:, 2 * heads:])
    part = make(rows, heads, hd, dtype, 3)  # part of the channels, in place: nothing is copied
    kept = part.clone()
    B.rotary(part, rotary_dim=16, q_out=part)
    check(part, kept, torch.arange(rows, device="cuda"), 16)


def test_heads_before_rows(B):
    """[heads, rows, head_dim] seen as [rows, heads, head_dim], and an output laid out otherwise."""
    x = make(6, 90, 64, torch.bfloat16).transpose(0, 1)
    pos = torch.arange(90, device="cuda")
    out = torch.empty(90, 6, 64, device="cuda", dtype=torch.bfloat16)
    B.rotary(x, q_out=out)
    check(out, x, pos, 64)


def test_the_inverse_is_the_gradient(B):
    q = make(40, 2, 64, torch.float32, 1)
    w = make(40, 2, 64, torch.float32, 2)
    kw = dict(rotary_dim=48, amplitude=1.5, layout="interleaved")
    grad, _ = B.rotary(w, inverse=True, **kw)
    x = q.double().requires_grad_()
    y, _ = reference(x, torch.arange(40, device="cuda"), r=48, amplitude=1.5, layout="interleaved")
    (y * w.double()).sum().backward()
    assert float((grad.double() - x.grad).abs().max()) <= 6e-7 * 1.5 * 2 * float(w.abs().max()) + 2.0 ** -24 * float(x.grad.abs().max())
    # and by differences: the map is linear, so any step is exact but for rounding
    d = make(40, 2, 64, torch.float32, 3)
    lhs = ((B.rotary(q + d, **kw)[0].double() - B.rotary(q, **kw)[0].double()) * w.double()).sum()
    rhs = (grad.double() * ((q + d).double() - q.double())).sum()
    scale = float((w.double().abs() * 6).sum())
    assert abs(float(lhs - rhs)) <= 4e-6 * scale


def test_rows_beyond_32_bits(B):
    """Elements more than 2^31 behind the first: rows 2^20 elements apart, 2100 of them (4.4 GB)."""
    buf = torch.empty(2100 * (1 << 20), device="cuda", dtype=torch.bfloat16)
    x = buf.as_strided((2100, 2, 64), (1 << 20, 64, 1))
    x.copy_(make(2100, 2, 64, torch.bfloat16))
    got, _ = B.rotary(x)
    check(got, x, torch.arange(2100, device="cuda"), 64)
    kept = x.clone()
    B.rotary(x, q_out=x)
    assert torch.equal(x, got) and not torch.equal(x, kept)


def test_captured_and_replayed_on_another_stream(B):
    q, k = make(300, 4, 64, torch.bfloat16, 1), make(300, 2, 64, torch.bfloat16, 2)
    pos = torch.arange(300, device="cuda", dtype=torch.int32)
    qo, ko = torch.zeros_like(q), torch.zeros_like(k)
    B.rotary(q, k, positions=pos)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        B.rotary(q, k, positions=pos, q_out=qo, k_out=ko)
    for step in (0, 1000):
        pos.copy_(torch.arange(300, device="cuda", dtype=torch.int32) + step)
        graph.replay()
        check(qo, q, pos, 64)
        check(ko, k, pos, 64)


def test_refusals_of_the_binding(B):
    q = make(4, 2, 64, torch.float32)
    for bad in (dict(k=make(5, 2, 64, torch.float32)), dict(k=make(4, 2, 64, torch.bfloat16)), dict(positions=torch.zeros(4, device="cuda")),
                dict(positions=torch.zeros(3, device="cuda", dtype=torch.int32)), dict(q_out=make(4, 2, 32, torch.float32)),
                dict(rotary_dim=66), dict(rotary_dim=7)):
        with pytest.raises(B.HbpError) as e:
            B.rotary(q, **bad)
        assert e.value.code == 2
    for bad in (dict(positions=torch.zeros(4, dtype=torch.int32)), dict(k=torch.zeros(4, 2, 64))):  # on the host
        with pytest.raises(B.HbpError) as e:
            B.rotary(q, **bad)
        assert e.value.code == 1
    assert B.rotary(q[:0], q[:0])[0].shape == (0, 2, 64)
