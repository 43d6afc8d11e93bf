"""Activations in 8 bits: codes and scales bit for bit, GELU and its backward pass from them against 64 bits.  Bounds: one
rounding to the type, and for gelu and gelu' themselves: float, erff to 2 units in the last place of 1 (2.4e-7), times z; bf16,
1.5e-7 for the formula's half of erfc, 4e-7 for its float arithmetic, times z."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
TYPES = [torch.float32, torch.bfloat16]


@pytest.fixture(scope="module")
def B():
    from paper_2501_17086_b200 import binding
    return binding


def reference(x):
    """codes and scales of finite x by the definition, through whole-number comparisons only."""
    rows, d = x.shape
    g = torch.nn.functional.pad(x.double(), (0, -d % 32)).view(rows, -1, 32)
    most = g.abs().amax(-1, keepdim=True)
    e = torch.full_like(most, -126.0)
    for k in range(-126, 123):
        e = torch.where(most > 127.0 * 2.0 ** k, torch.full_like(e, k + 1.0), e)
    codes = torch.round(g / torch.exp2(e))
    codes = torch.where(e == 122, codes.clamp(-63, 63), codes)  # 64 * 2^122 is no float
    return codes.flatten(1)[:, :d].to(torch.int8), (e[..., 0] + 127).to(torch.uint8), (codes * torch.exp2(e)).flatten(1)[:, :d]


def make(rows, d, dtype, seed=0, scale=True):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(rows, d, generator=g, device="cuda")
    if scale:
        x = x * torch.exp2(torch.randint(-12, 5, (rows, 1), generator=g, device="cuda").float())
    return x.to(dtype)


SIZES = [(1, 8), (1, 32), (3, 40), (77, 1492 // 8 * 8), (33, 4096), (4097, 24), (129, 1000), (2, 65536)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,d", SIZES)
def test_codes_scales_and_values(B, dtype, rows, d):
    x = make(rows, d, dtype)
    codes, scales = B.checkpoint_store(x)
    c, s, v = reference(x)
    assert torch.equal(codes, c) and torch.equal(scales, s)
    for t in TYPES:  # the stored values are bf16 numbers
        assert torch.equal(B.checkpoint_load(codes, scales, t).double(), v)
    step = torch.exp2(scales.double() - 127).repeat_interleave(32, 1)[:, :d]
    assert bool(((x.double() - v).abs() <= step / 2).all())


def test_float_rows_that_are_no_multiple_of_eight(B):
    x = make(37, 1492, torch.float32)
    codes, scales = B.checkpoint_store(x)
    c, s, v = reference(x)
    assert torch.equal(codes, c) and torch.equal(scales, s) and torch.equal(B.checkpoint_load(codes, scales, torch.float32).double(), v)


@pytest.mark.parametrize("dtype", TYPES)
def test_borders_of_a_scale(B, dtype):
    """127 * 2^e is kept with scale e, the next number up is not; ties go to the even code; zeros, the smallest and the largest numbers."""
    up = torch.finfo(dtype).eps
    rows = []
    for top in (127.0, 127.0 * (1 + up), 126.0, 128.0, 64.0, 63.5):
        r = torch.zeros(32)
        r[:8] = torch.tensor([top, 0.5, 1.5, 2.5, -0.5, -1.5, -2.5, 63.5])
        rows += [r, r * 2.0 ** -20, r * 2.0 ** 40]
    rows.append(torch.zeros(32))
    rows.append(torch.full((32,), torch.finfo(dtype).max))
    rows.append(torch.full((32,), torch.finfo(dtype).tiny))
    rows.append(torch.full((32,), torch.finfo(dtype).tiny * 2.0 ** -5))
    x = torch.stack(rows).to(dtype).cuda()
    codes, scales = B.checkpoint_store(x)
    c, s, v = reference(x)
    assert torch.equal(codes, c) and torch.equal(scales, s)
    back = B.checkpoint_load(codes, scales, dtype).double()
    assert bool(torch.isfinite(back).all()) and float((back - v).abs().max()) == 0


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_groups_that_are_not_finite_read_back_as_nan(B, dtype, bad):
    x = make(5, 104, dtype)
    x[1, 40] = bad
    x[4, 103] = bad
    codes, scales = B.checkpoint_store(x)
    back = B.checkpoint_load(codes, scales, dtype)
    nan = torch.zeros_like(x, dtype=torch.bool)
    nan[1, 32:64] = nan[4, 96:] = True
    assert torch.equal(back.isnan(), nan) and int((scales == 255).sum()) == 2
    assert torch.equal(B.checkpoint_gelu_backward(torch.ones_like(x), codes, scales).isnan(), nan)


def bounds(z, dtype):
    z = z.double()
    phi = torch.special.ndtr(z)
    dens = torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    e = 2.4e-7 + 2.0 ** -24 if dtype == torch.float32 else 5.5e-7
    # (z * z * constant is rounded before the exponential: relative error of z^2 / 2 * 2^-22 there)
    dens_e = z.abs() * dens * (4e-7 + z * z * 2.0 ** -23)
    return z * phi, z.abs() * e + 1e-38, phi + z * dens, e + dens_e


def within(got, want, e, dtype):
    over = float(((got.double() - want).abs() - e - HALF[dtype] * (want.abs() + e) - 1e-38).max())
    assert over <= 0, over


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,d", SIZES)
def test_gelu_and_its_backward_pass(B, dtype, rows, d):
    z = make(rows, d, dtype, 1)
    g = make(rows, d, dtype, 2)
    act, codes, scales = B.checkpoint_gelu(z)
    c, s, z8 = reference(z)
    assert torch.equal(codes, c) and torch.equal(scales, s)
    want, e, _, _ = bounds(z, dtype)
    within(act, want, e, dtype)
    dz, act8 = B.checkpoint_gelu_backward(g, codes, scales, with_act=True)
    want, e, slope, es = bounds(z8, dtype)
    within(act8, want, e, dtype)
    want, e = g.double() * slope, g.double().abs() * es
    within(dz, want, e, dtype)
    assert torch.equal(B.checkpoint_gelu_backward(g, codes, scales), dz)  # without the activation


@pytest.mark.parametrize("dtype", TYPES)
def test_slope_by_differences(B, dtype):
    """gelu'(z8) against differences of gelu(z8) in 64 bits, and against automatic differentiation."""
    z = make(64, 256, dtype, 1, scale=False) * 3
    codes, scales = B.checkpoint_store(z)
    z8 = B.checkpoint_load(codes, scales, torch.float32).double()
    got = B.checkpoint_gelu_backward(torch.ones_like(z), codes, scales).double()
    x = z8.clone().requires_grad_()
    torch.nn.functional.gelu(x).sum().backward()
    tol = 1e-6 + HALF[dtype] * 1.2
    assert float((got - x.grad).abs().max()) <= tol
    h = 1e-4
    f = torch.nn.functional.gelu
    assert float((got - (f(z8 + h) - f(z8 - h)) / (2 * h)).abs().max()) <= tol + h * h  # |gelu'''| / 6 < 1


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [96, 104])
def test_in_place_and_rows_apart(B, dtype, d):
    """Outputs over their inputs; rows of wider buffers, whose other channels and rows stay as they were."""
    wide = make(20, 3 * 128, dtype, 1)
    z = wide[:13, 128:128 + d]
    was, kept = wide.clone(), z.clone()
    want, c, s = B.checkpoint_gelu(kept)
    act, codes, scales = B.checkpoint_gelu(z, act=z)
    assert torch.equal(act, want) and torch.equal(codes, c) and torch.equal(scales, s)
    assert torch.equal(B.checkpoint_store(was[:13, 128:128 + d])[0], c)
    wide[:13, 128:128 + d] = was[:13, 128:128 + d]
    assert torch.equal(wide, was)
    g = wide[3:16, 256:256 + d]
    want, want8 = B.checkpoint_gelu_backward(g.clone(), c, s, with_act=True)
    other = torch.full((13, 256), 7.0, device="cuda", dtype=dtype)
    B.checkpoint_gelu_backward(g, c, s, dz=g, act=other[:, :d])
    assert torch.equal(g, want) and torch.equal(other[:, :d], want8) and bool((other[:, d:] == 7).all())
    wide[3:16, 256:256 + d] = was[3:16, 256:256 + d]
    assert torch.equal(wide, was)
    out = torch.full((13, 256), 7.0, device="cuda", dtype=dtype)
    B.checkpoint_load(c, s, out=out[:, :d])
    assert torch.equal(out[:, :d], B.checkpoint_load(c, s, dtype)) and bool((out[:, d:] == 7).all())


def test_more_than_32_bits_of_elements(B):
    """2^31 and some values (4.3 GB of bf16): the last rows are what they are on their own."""
    rows, d = (1 << 20) + 3, 2048
    x = torch.zeros(rows, d, device="cuda", dtype=torch.bfloat16)
    x[-5:] = make(5, d, torch.bfloat16)
    act, codes, scales = B.checkpoint_gelu(x)
    a, c, s = B.checkpoint_gelu(x[-5:].clone())
    assert torch.equal(codes[-5:], c) and torch.equal(scales[-5:], s) and torch.equal(act[-5:], a)
    assert int(codes[:-5].max()) == 0 and int(scales[:-5].max()) == 1
    back = B.checkpoint_load(codes, scales, out=x)
    assert torch.equal(back[-5:], B.checkpoint_load(c, s))


def test_captured_and_replayed(B):
    z, g = make(100, 512, torch.bfloat16, 1), make(100, 512, torch.bfloat16, 2)
    B.checkpoint_gelu(z)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        act, codes, scales = B.checkpoint_gelu(z)
        dz = B.checkpoint_gelu_backward(g, codes, scales)
    for seed in (3, 4):
        z.copy_(make(100, 512, torch.bfloat16, seed))
        graph.replay()
        want, c, s = B.checkpoint_gelu(z)
        assert torch.equal(act, want) and torch.equal(codes, c) and torch.equal(dz, B.checkpoint_gelu_backward(g, c, s))


def test_refusals_of_the_binding(B):
    z = make(4, 64, torch.float32)
    codes, scales = B.checkpoint_store(z)
    for call in (lambda: B.checkpoint_store(make(4, 66, torch.float32)), lambda: B.checkpoint_store(z.t()),
                 lambda: B.checkpoint_store(z, codes=codes[:3]), lambda: B.checkpoint_store(z, scales=scales[:, :1]),
                 lambda: B.checkpoint_gelu(z, act=z.bfloat16()), lambda: B.checkpoint_gelu_backward(z[:3], codes, scales),
                 lambda: B.checkpoint_load(codes, scales, out=z[:3])):
        with pytest.raises(B.HbpError) as e:
            call()
        assert e.value.code == 2
    with pytest.raises(B.HbpError) as e:
        B.checkpoint_store(z.half())
    assert e.value.code == 3
    with pytest.raises(B.HbpError) as e:
        B.checkpoint_store(z.cpu())
    assert e.value.code == 1
    assert B.checkpoint_store(z[:0])[0].shape == (0, 64)
