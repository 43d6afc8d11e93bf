"""The residual update between two norms, and its gradients, against the formulas in 64 bits.

Bounds, with e = 2^-24.  A row's sum is formed by adding at most 32 values a thread, 5 exchanges in a warp and 16 warps: 53 additions deep, so a
mean is off by 53 e mean|v|, a sum of squares by 57 e of itself, and 1 / sqrt of it by half of that and 3 roundings: xhat by
C e (|xhat| + r mean|v|) with C = 64.  What follows adds a few roundings of each term (C' = 2 C is taken for gradients, which use two
such sums).  Sums over rows: each term's error, and (rows + 64) e of the magnitudes."""
import pytest
import torch

pytestmark = pytest.mark.gpu
E, C = 2.0 ** -24, 64
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


@pytest.fixture(scope="module")
def B():
    from paper_2501_17086_b200 import binding
    return binding


def rows_of(n, d, dtype, seed, std=1.0, mean=0.0, stride=None):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(n, stride or d, generator=g, device="cuda") * std + mean).to(dtype)[:, :d]


def vector(d, dtype, seed, mean):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(d, generator=g, device="cuda") * 0.2 + mean).to(dtype)


def norm(v, kind, eps):
    """(xhat, 1 / sqrt, bound of xhat's error)"""
    m = v.mean(1, keepdim=True) if kind == "layer" else 0.0
    r = 1.0 / torch.sqrt(((v - m) ** 2).mean(1, keepdim=True) + eps)
    xhat = (v - m) * r
    mean = v.abs().mean(1, keepdim=True) if kind == "layer" else 0.0
    return xhat, r, C * E * (xhat.abs() + r * mean)


def near(got, want, bound, dtype=torch.float32, what=""):
    half = HALF[dtype]
    over = float(((got.double() - want).abs() - bound - half * (want.abs() + bound) - 1e-37).max())
    assert over <= 0, (what, over)


class Inputs:
    def __init__(self, n, d, dtype, post, gate, weights, seed=0, pad=0):
        self.x = rows_of(n, d, dtype, seed + 1, 2.0, 0.5, d + pad)
        self.f = rows_of(n, d, dtype, seed + 2, 0.3, 0.1, d + pad)
        self.w_pre = vector(d, dtype, seed + 3, 1.0) if weights else None
        self.w_post = vector(d, dtype, seed + 4, 1.0) if weights and post else None
        self.gate = vector(d, dtype, seed + 5, 0.9) if gate else None
        self.post = post
        self.d_y = rows_of(n, d, dtype, seed + 6, 2.0 ** -8, 0.0, d + pad)
        self.d_new = rows_of(n, d, dtype, seed + 7, 2.0 ** -8, 0.0, d + pad)

    def kw(self, **more):
        return dict(post=self.post, w_post=self.w_post, gate=self.gate, w_pre=self.w_pre, **more)


def wide(w, like):
    return torch.ones_like(like[0]).double() if w is None else w.double()


def check_forward(s, x_new, y, kind, scale, eps):
    dtype, x, f = s.x.dtype, s.x.double(), s.f.double()
    h, err = f, torch.zeros_like(f)
    if s.post:
        h, _, err = norm(f, kind, eps)
        w = wide(s.w_post, x)
        h, err = h * w, err * w.abs() + 2 * E * (h * w).abs()
    g = wide(s.gate, x)
    near(x_new, g * x + scale * h, abs(scale) * err + 3 * E * ((g * x).abs() + (scale * h).abs()), dtype, "x_new")
    if y is not None:
        xhat, _, err = norm(x_new.double(), kind, eps)
        w = wide(s.w_pre, x)
        near(y, xhat * w, err * w.abs() + 2 * E * (xhat * w).abs(), dtype, "y")


def check_backward(s, x_new, got, kind, scale, eps, with_y=True, with_new=True):
    dtype, n = s.x.dtype, s.x.shape[0]
    x, f, v = s.x.double(), s.f.double(), x_new.double()
    dx, df, dw_pre, dw_post, da = got
    layer = kind == "layer"

    def back(a, a_err, xhat, r, err):
        along, flat = (a * xhat).mean(1, keepdim=True), a.mean(1, keepdim=True) if layer else 0.0
        size = a.abs() + (a.abs().mean(1, keepdim=True) if layer else 0.0) + xhat.abs() * (a.abs() * xhat.abs()).mean(1, keepdim=True)
        e = 2 * C * E * size + err * along.abs() + xhat.abs() * (a.abs() * err).mean(1, keepdim=True)
        e = e + a_err + (a_err.mean(1, keepdim=True) if layer else 0.0) + xhat.abs() * (a_err * xhat.abs()).mean(1, keepdim=True)
        return r * (a - flat - xhat * along), r * e

    t, t_err = torch.zeros_like(x), torch.zeros_like(x)
    if with_new:
        t = s.d_new.double()
    if with_y:
        xhat, r, err = norm(v, kind, eps)
        dy, w = s.d_y.double(), wide(s.w_pre, x)
        u, t_err = back(dy * w, E * (dy * w).abs(), xhat, r, err)
        t = t + u
        t_err = t_err + 2 * E * (u.abs() + t.abs())
        if dw_pre is not None:
            near(dw_pre, (dy * xhat).sum(0), (dy.abs() * err).sum(0) + (n + 64) * E * (dy * xhat).abs().sum(0), what="dw_pre")
    g = wide(s.gate, x)
    if dx is not None:
        near(dx, g * t, g.abs() * t_err + E * (g * t).abs(), dtype, "dx")
    if da is not None:
        near(da, (t * x).sum(0), (t_err * x.abs()).sum(0) + (n + 64) * E * (t * x).abs().sum(0), what="da")
    u, u_err = scale * t, abs(scale) * t_err + E * (scale * t).abs()
    if s.post:
        fhat, r, err = norm(f, kind, eps)
        if dw_post is not None:
            near(dw_post, (u * fhat).sum(0), (u_err * fhat.abs() + u.abs() * err).sum(0) + (n + 64) * E * (u * fhat).abs().sum(0), what="dw_post")
        w = wide(s.w_post, x)
        u, u_err = back(u * w, u_err * w.abs() + E * (u * w).abs(), fhat, r, err)
    if df is not None:
        near(df, u, u_err, dtype, "df")


SIZES = [(1, 8), (3, 64), (17, 256), (5, 264), (9, 512), (301, 768), (33, 1032), (1237, 1496), (65, 2048), (7, 2056), (12, 4096), (4, 8192)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("post,gate,weights", [(False, False, False), (True, True, True), (True, False, True), (False, True, False)])
@pytest.mark.parametrize("n,d", SIZES)
def test_both_passes(B, dtype, kind, post, gate, weights, n, d):
    s = Inputs(n, d, dtype, post, gate, weights, n + d, 16)
    kw = s.kw(kind=kind, eps=1e-5, scale=0.625)
    x_new, y = B.norm_residual(s.x, s.f, **kw)
    check_forward(s, x_new, y, kind, 0.625, 1e-5)
    got = B.norm_residual_backward(s.d_y, x_new, s.f, s.x, d_new=s.d_new, **kw)
    assert [t is None for t in got] == [False, False, not weights, not (weights and post), not gate]
    check_backward(s, x_new, got, kind, 0.625, 1e-5)
    again = B.norm_residual_backward(s.d_y, x_new, s.f, s.x, d_new=s.d_new, **kw)
    assert all(a is None or torch.equal(a, b) for a, b in zip(got, again))  # the same bits


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows", [5000, 20001])
def test_many_rows(B, dtype, rows):
    """More rows than groups of threads."""
    s = Inputs(rows, 320, dtype, True, True, True)
    kw = s.kw(kind="layer", scale=1.0)
    x_new, y = B.norm_residual(s.x, s.f, **kw)
    check_forward(s, x_new, y, "layer", 1.0, 1e-5)
    check_backward(s, x_new, B.norm_residual_backward(s.d_y, x_new, s.f, s.x, d_new=s.d_new, **kw), "layer", 1.0, 1e-5)


@pytest.mark.parametrize("kind", ["layer", "rms"])
def test_parts_alone(B, kind):
    s = Inputs(77, 384, torch.bfloat16, True, True, True)
    kw = s.kw(kind=kind, scale=0.5)
    # the norm of a stream: a final norm
    x, y = B.norm_residual(s.x, kind=kind, w_pre=s.w_pre)
    assert x.data_ptr() == s.x.data_ptr()
    xhat, _, err = norm(s.x.double(), kind, 1e-5)
    near(y, xhat * s.w_pre.double(), err * s.w_pre.double().abs() + 2 * E * xhat.abs() * s.w_pre.double().abs(), s.x.dtype)
    plain = Inputs(77, 384, torch.bfloat16, False, False, True)
    plain.x, plain.d_y = s.x, s.d_y
    got = B.norm_residual_backward(s.d_y, s.x, kind=kind, w_pre=plain.w_pre, with_df=False)
    assert got[1] is None and got[3] is None and got[4] is None
    check_backward(plain, s.x, got, kind, 1.0, 1e-5, with_new=False)
    # the update alone
    x_new, y = B.norm_residual(s.x, s.f, with_y=False, **kw)
    assert y is None
    check_forward(s, x_new, None, kind, 0.5, 1e-5)
    got = B.norm_residual_backward(None, None, s.f, s.x, d_new=s.d_new, **kw)
    assert got[2] is None
    check_backward(s, x_new, got, kind, 0.5, 1e-5, with_y=False)
    # gradients of some
    full = B.norm_residual_backward(s.d_y, x_new, s.f, s.x, d_new=s.d_new, **kw)
    some = B.norm_residual_backward(s.d_y, x_new, s.f, None, d_new=s.d_new, with_weights=False, with_dx=False, **kw)
    assert torch.equal(some[1], full[1]) and [t is None for t in some] == [True, False, True, True, True]
    some = B.norm_residual_backward(s.d_y, x_new, s.f, s.x, d_new=s.d_new, with_df=False, with_dx=False, **kw)
    assert all(torch.equal(some[i], full[i]) for i in (2, 3, 4))


def test_gradients_against_differences(B):
    """Central differences of the formula in 64 bits along one direction of all inputs."""
    s = Inputs(6, 72, torch.float32, True, True, True)
    w = {k: getattr(s, k).double() for k in ("x", "f", "w_pre", "w_post", "gate")}
    g = torch.Generator(device="cuda").manual_seed(9)
    step = {k: torch.randn(t.shape, generator=g, device="cuda", dtype=torch.float64) for k, t in w.items()}
    d_y, d_new = s.d_y.double(), s.d_new.double()

    def value(h):
        p = {k: t + h * step[k] for k, t in w.items()}
        new = p["gate"] * p["x"] + 0.5 * norm(p["f"], "layer", 1e-5)[0] * p["w_post"]
        return float((d_new * new).sum() + (d_y * norm(new, "layer", 1e-5)[0] * p["w_pre"]).sum())

    h = 1e-5
    slope = (value(h) - value(-h)) / (2 * h)
    kw = s.kw(kind="layer", scale=0.5)
    x_new, _ = B.norm_residual(s.x, s.f, **kw)
    got = dict(zip(("x", "f", "w_pre", "w_post", "gate"), B.norm_residual_backward(s.d_y, x_new, s.f, s.x, d_new=s.d_new, **kw)))
    along = {k: float((got[k].double() * step[k]).sum()) for k in got}
    # x_new is rounded to float (2^-24 of each value, which the norm's gradient passes on), differences have h^2 of third derivatives: 1e-6 of the terms
    assert abs(sum(along.values()) - slope) <= 2e-6 * sum(float((got[k].double() * step[k]).abs().sum()) for k in got)


def test_in_place_broadcast_and_strides(B):
    s = Inputs(130, 768, torch.bfloat16, True, True, True)
    kw = s.kw(kind="rms", scale=0.5)
    x_new, y = B.norm_residual(s.x, s.f, **kw)
    x, f = s.x.clone(), s.f.clone()
    a, b = B.norm_residual(x, f, x_new=x, y=f, **kw)
    assert a.data_ptr() == x.data_ptr() and torch.equal(x, x_new) and torch.equal(f, y)
    want = B.norm_residual_backward(s.d_y, x_new, s.f, s.x, d_new=s.d_new, **kw)
    d_y, d_new = s.d_y.clone(), s.d_new.clone()
    B.norm_residual_backward(d_y, x_new, s.f, s.x, d_new=d_new, dx=d_new, df=d_y, **kw)
    assert torch.equal(d_new, want[0]) and torch.equal(d_y, want[1])
    row = s.d_y[:1].expand(130, 768)
    got = B.norm_residual_backward(row, x_new, s.f, s.x, d_new=s.d_new, **kw)
    want = B.norm_residual_backward(row.contiguous(), x_new, s.f, s.x, d_new=s.d_new, **kw)
    assert all(torch.equal(p, q) for p, q in zip(got, want))
    out = torch.full((130, 800), 3.0, device="cuda", dtype=torch.bfloat16)
    B.norm_residual(s.x, s.f, y=out[:, 8:776], **kw)
    assert torch.equal(out[:, 8:776], y) and bool((out[:, :8] == 3.0).all()) and bool((out[:, 776:] == 3.0).all())


@pytest.mark.parametrize("kind", ["layer", "rms"])
def test_rows_of_zeros_large_rows_and_rows_that_are_not_finite(B, kind):
    s = Inputs(40, 256, torch.float32, True, False, True)
    x = s.x.clone()
    x[3] = 0.0
    s.f[3] = 0.0
    x[4] = 1000.0 + 0.001 * torch.randn(256, device="cuda")  # far from zero: its variance is no difference of squares
    x[7, 5] = float("nan")
    x[8, 9] = float("inf")
    s.x = x
    kw = s.kw(kind=kind, scale=0.5)
    x_new, y = B.norm_residual(s.x, s.f, **kw)
    fine = torch.ones(40, dtype=torch.bool, device="cuda")
    fine[7] = fine[8] = False
    assert bool(y[fine].isfinite().all()) and bool(y[7].isnan().all()) and bool(y[8].isnan().any())
    assert not y[3].any()
    got = B.norm_residual_backward(s.d_y, x_new, s.f, s.x, d_new=s.d_new, **kw)
    assert bool(got[0][fine].isfinite().all())
    sub = Inputs(38, 256, torch.float32, True, False, True)
    for k in ("x", "f", "d_y", "d_new"):
        setattr(sub, k, getattr(s, k)[fine].contiguous())
    sub.w_pre, sub.w_post = s.w_pre, s.w_post
    check_forward(sub, x_new[fine], y[fine], kind, 0.5, 1e-5)
    check_backward(sub, x_new[fine], (got[0][fine], got[1][fine], None, None, None), kind, 0.5, 1e-5)


def test_no_rows(B):
    e = torch.empty(0, 64, device="cuda")
    w = torch.ones(64, device="cuda")
    assert B.norm_residual(e, e, w_pre=w)[1].shape == (0, 64)
    got = B.norm_residual_backward(e, e, e, e, d_new=e, gate=w, w_pre=w)
    assert got[0].shape == (0, 64) and not got[2].any() and not got[4].any()
