"""Cross entropy of a large vocabulary and its gradients against the formulas in 64 bits.

Bounds.  A logit is a float sum on the tensor core: exact products, a truncation of at most 2^-23 of the magnitudes A = sum |x w| an instruction of 16
of K, and inside one: off by z_err = (d / 16 + 8) 2^-23 A (float data: per 32 of K, and as much again for the parts left out).
The terms exp(z - r) are then off by 2 z_err (z and r) and |z - r| 2^-23 and the functions' few units, below 2e-5 together for |z - r| <= 100;
their sum S' by as much of itself, and the loss, log1p(S'), by that times S' / S = 1 - exp(-loss) <= 1 (by expm1: losses go down to 1e-20).
Gradients (bf16 data): a rounding of each numerator, 2^-8, and in all but the target's the row's share of the rounding of that, as much again; for dw a third one, of
x times its factor.  Float data has none of these.  Then the sums' truncations, and the output's rounding."""
import pytest
import torch

pytestmark = pytest.mark.gpu
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


@pytest.fixture(scope="module")
def B():
    from paper_2501_17086_b200 import binding
    return binding


class Case:
    def __init__(self, n, d, vocab, dtype, seed=0, lead=0.0, std=0.02, pad=0, ignored=0.1, target_type=torch.int64):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.w = (torch.randn(vocab, d + pad, generator=g, device="cuda") * std).to(dtype)[:, :d]
        t = torch.randint(0, vocab, (n,), generator=g, device="cuda")
        wt = self.w[t].float()
        x = torch.randn(n, d, generator=g, device="cuda") + lead * wt / wt.norm(dim=1, keepdim=True).clamp_min(1e-6)
        self.x = torch.zeros(n, d + pad, device="cuda", dtype=dtype)[:, :d].copy_(x)
        self.t = torch.where(torch.rand(n, generator=g, device="cuda") < ignored, -1, t).to(target_type)
        self.d_loss = torch.rand(n, generator=g, device="cuda") / n

    def reference(self):
        x, w, t = self.x.double(), self.w.double(), self.t.long()
        there = t >= 0
        x = torch.where(there[:, None], x, 0.0)
        z = x @ w.T
        loss = torch.logsumexp(z, 1) - z.gather(1, t.clamp_min(0)[:, None])[:, 0]
        # (small losses without cancellation)
        at = torch.zeros_like(z, dtype=torch.bool).scatter_(1, t.clamp_min(0)[:, None], True)
        rest = torch.logsumexp(z.masked_fill(at, -torch.inf), 1) - z.gather(1, t.clamp_min(0)[:, None])[:, 0]
        loss = torch.where(rest < -10, torch.log1p(rest.exp()), loss)
        d = x.shape[1]
        k = (d / 16 + 8) if self.x.dtype == torch.bfloat16 else 2 * (d / 32 + 8)
        z_err = k * 2.0 ** -23 * (x.abs() @ w.abs().T).max(1).values
        rel = 2 * z_err + 2e-5
        return there, z, at, torch.where(there, loss, 0.0), torch.where(there, rel * -torch.expm1(-loss) + 2.0 ** -22 * loss, 0.0), rel


def check(c, loss, dx=None, dw=None, d_loss=None):
    there, z, at, want, bound, rel = c.reference()
    # terms below 2^-126, the smallest normal number, are taken for zero: up to `vocab` of them, 2^-100 of a loss
    over = float(((loss.double() - want).abs() - bound - 2.0 ** -100).max())
    assert over <= 0, over
    assert not loss[~there].any()
    if dx is None and dw is None:
        return
    g = torch.where(there, 1.0 if d_loss is None else d_loss.double(), 0.0)
    p = torch.softmax(z, 1)
    rest = p.masked_fill(at, 0.0).sum(1)
    dz = torch.where(at, -rest[:, None], p) * g[:, None]
    bf = c.x.dtype == torch.bfloat16
    half = HALF[c.x.dtype]
    x, w = torch.where(there[:, None], c.x.double(), 0.0), c.w.double()
    each = (rel + (2 * half if bf else 2.0 ** -22))[:, None] * dz.abs()
    (n, vocab) = z.shape
    if dx is not None:
        exact = dz @ w
        b = each @ w.abs() + (vocab / 16 + 16) * 2.0 ** -23 * (dz.abs() @ w.abs())
        over = float(((dx.double() - exact).abs() - b - half * (exact.abs() + b) - 1e-37).max())
        assert over <= 0, ("dx", over)
        assert not dx[~there].any()
    if dw is not None:
        exact = dz.T @ x
        b = (1 + half) * (each.T @ x.abs()) + ((n / 16 + 24) * 2.0 ** -23 + (half if bf else 0.0)) * (dz.abs().T @ x.abs())
        # factors and terms below the smallest normal numbers are taken for zero: gradients of 2^-100 and less
        over = float(((dw.double() - exact).abs() - b - HALF[dw.dtype] * (exact.abs() + b) - n * 2.0 ** -100).max())
        assert over <= 0, ("dw", over)


SIZES = [(1, 64, 50), (1, 8, 1), (5, 72, 7), (16, 512, 1003), (64, 128, 64), (100, 256, 129), (128, 264, 4099), (129, 64, 300), (300, 520, 1111), (513, 768, 2049), (1000, 1024, 5003),
         (77, 4096, 513)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("lead", [0.0, 20.0])
@pytest.mark.parametrize("n,d,vocab", SIZES)
def test_loss_and_gradients(B, dtype, lead, n, d, vocab):
    c = Case(n, d, vocab, dtype, n + d, lead, pad=8, target_type=torch.int32 if n % 2 else torch.int64)
    c.t[0] = c.t[0].clamp_min(0)
    check(c, B.cross_entropy(c.x, c.w, c.t))
    loss, dx, dw = B.cross_entropy_gradients(c.x, c.w, c.t, d_loss=c.d_loss)
    assert dw.dtype == torch.float32 and dx.dtype == dtype
    check(c, loss, dx, dw, c.d_loss)
    again = B.cross_entropy_gradients(c.x, c.w, c.t, d_loss=c.d_loss)
    assert torch.equal(again[0], loss) and torch.equal(again[1], dx) and torch.equal(again[2], dw)
    if dtype == torch.bfloat16:
        dw16 = B.cross_entropy_gradients(c.x, c.w, c.t, d_loss=c.d_loss, dw_dtype=dtype)[2]
        assert torch.equal(dw16, dw.to(dtype))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_pieces(B, dtype):
    """Scratch for fewer rows at a time."""
    c = Case(1500, 128, 3001, dtype, 3)
    whole = B.cross_entropy_scratch_bytes(dtype, 1500, 3001, 128)
    least = B.cross_entropy_scratch_bytes(dtype, 256, 3001, 128) + (4 * 3001 * 128 + 256)
    want = B.cross_entropy_gradients(c.x, c.w, c.t, d_loss=c.d_loss)
    for size in (whole, whole - 256, whole // 2, least):
        scratch = torch.empty(size, dtype=torch.uint8, device="cuda")
        for dw_dtype in {torch.float32, dtype}:
            loss, dx, dw = B.cross_entropy_gradients(c.x, c.w, c.t, d_loss=c.d_loss, dw_dtype=dw_dtype, scratch=scratch)
            check(c, loss, dx, dw, c.d_loss)
            assert torch.equal(loss, want[0])
    small = torch.empty(B.cross_entropy_scratch_bytes(dtype, 256, 3001, 128, False), dtype=torch.uint8, device="cuda")
    # (the loss alone is summed in another order, around each tile's largest logit, than with gradients: by itself it is the same in any pieces)
    alone = B.cross_entropy(c.x, c.w, c.t, scratch=small)
    check(c, alone)
    assert torch.equal(alone, B.cross_entropy(c.x, c.w, c.t))
    with pytest.raises(B.HbpError) as e:
        B.cross_entropy_gradients(c.x, c.w, c.t, scratch=small[: 64 << 10])
    assert e.value.code == 5


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n", [40, 300])
def test_targets_far_below_the_largest_logit(B, dtype, n):
    """Losses of hundreds, in some rows or in all, beside ordinary ones; and logits of hundreds with the target on top."""
    c = Case(n, 256, 777, dtype, 5, std=0.02)
    c.x[: n // 2] *= 200.0
    loss, dx, dw = B.cross_entropy_gradients(c.x, c.w, c.t, d_loss=c.d_loss)
    assert float(loss.max()) > 100
    check(c, loss, dx, dw, c.d_loss)
    check(c, B.cross_entropy(c.x, c.w, c.t))
    top = (c.x.double() @ c.w.double().T).argmax(1)
    c.t = torch.where(torch.arange(n, device="cuda") % 3 == 0, top, c.t)
    loss, dx, dw = B.cross_entropy_gradients(c.x, c.w, c.t, d_loss=c.d_loss)
    check(c, loss, dx, dw, c.d_loss)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_small_losses_keep_their_digits(B, dtype):
    """A target far above the others: losses down to 1e-12, where 1 - p is a difference of like numbers, and gradients of that size."""
    c = Case(90, 512, 400, dtype, 7, lead=60.0, ignored=0.0)
    loss, dx, dw = B.cross_entropy_gradients(c.x, c.w, c.t)
    assert float(loss.min()) < 1e-6
    check(c, loss, dx, dw)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_without_a_target_may_hold_anything(B, dtype):
    c = Case(200, 128, 500, dtype, 11)
    want = B.cross_entropy_gradients(c.x, c.w, c.t, d_loss=c.d_loss)
    out = c.t < 0
    assert out.any()
    x, d_loss = c.x.clone(), c.d_loss.clone()
    x[out] = float("nan")
    d_loss[out] = float("nan")
    got = B.cross_entropy_gradients(x, c.w, c.t, d_loss=d_loss)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert torch.equal(B.cross_entropy(x, c.w, c.t), B.cross_entropy(c.x, c.w, c.t))
    none = torch.full_like(c.t, -1)
    loss, dx, dw = B.cross_entropy_gradients(x, c.w, none)
    assert not loss.any() and not dx.any() and not dw.any()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_one_row_that_is_not_finite(B, dtype):
    c = Case(200, 128, 500, dtype, 12, ignored=0.0)
    want = B.cross_entropy_gradients(c.x, c.w, c.t)
    x = c.x.clone()
    x[17, 3] = float("nan")
    loss, dx, _ = B.cross_entropy_gradients(x, c.w, c.t)
    others = torch.arange(200, device="cuda") != 17
    assert loss[17].isnan() and bool(dx[17].isnan().all())
    assert torch.equal(loss[others], want[0][others]) and torch.equal(dx[others], want[1][others])


def test_targets_beyond_the_vocabulary_are_none_and_reported(B):
    for dtype in (torch.float32, torch.bfloat16):
        c = Case(50, 64, 90, dtype, 13)
        want = B.cross_entropy_gradients(c.x, c.w, c.t)
        t = torch.where(c.t < 0, 90 + torch.arange(50, device="cuda") * 2 ** 33, c.t)
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        got = B.cross_entropy_gradients(c.x, c.w, t, status=status)
        assert status.item() == 1 and all(torch.equal(a, b) for a, b in zip(got, want))
        status.zero_()
        assert torch.equal(B.cross_entropy(c.x, c.w, t, status=status), B.cross_entropy(c.x, c.w, c.t)) and status.item() == 1
        status.zero_()
        B.cross_entropy(c.x, c.w, c.t, status=status)
        assert status.item() == 0


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_parts_strides_and_no_rows(B, dtype):
    c = Case(140, 128, 333, dtype, 14)
    loss, dx, dw = B.cross_entropy_gradients(c.x, c.w, c.t, d_loss=c.d_loss)
    a = B.cross_entropy_gradients(c.x, c.w, c.t, d_loss=c.d_loss, with_dw=False)
    b = B.cross_entropy_gradients(c.x, c.w, c.t, d_loss=c.d_loss, with_dx=False)
    assert a[2] is None and b[1] is None and torch.equal(a[1], dx) and torch.equal(b[2], dw)
    out = torch.full((140, 160), 5.0, device="cuda", dtype=dtype)
    wide = torch.full((333, 136), 5.0, device="cuda")
    B.cross_entropy_gradients(c.x, c.w, c.t, d_loss=c.d_loss, dx=out[:, 16:144], dw=wide[:, :128])
    assert torch.equal(out[:, 16:144], dx) and torch.equal(wide[:, :128], dw)
    assert bool((out[:, :16] == 5).all() and (out[:, 144:] == 5).all() and (wide[:, 128:] == 5).all())
    one = torch.full((1,), 0.25, device="cuda").expand(140)
    got = B.cross_entropy_gradients(c.x, c.w, c.t, d_loss=one)
    want = B.cross_entropy_gradients(c.x, c.w, c.t, d_loss=one.contiguous())
    assert all(torch.equal(p, q) for p, q in zip(got, want))
    none = c.x[:0]
    wide.fill_(5.0)
    loss, dx, dw = B.cross_entropy_gradients(none, c.w, c.t[:0], dw=wide[:, :128])
    assert loss.shape == (0,) and dx.shape == (0, 128) and not dw.any() and bool((wide[:, 128:] == 5).all())
    assert B.cross_entropy(none, c.w, c.t[:0]).shape == (0,)


def test_gradients_against_differences(B):
    """Central differences of the loss in 64 bits along one direction of x and of w."""
    c = Case(30, 64, 200, torch.float32, 15, std=0.3)
    g = torch.Generator(device="cuda").manual_seed(1)
    sx, sw = (torch.randn(t.shape, generator=g, device="cuda", dtype=torch.float64) for t in (c.x, c.w))
    there, t = c.t >= 0, c.t.clamp_min(0)

    def value(h):
        z = (c.x.double() + h * sx) @ (c.w.double() + h * sw).T
        return float((torch.where(there, torch.logsumexp(z, 1) - z.gather(1, t[:, None])[:, 0], 0.0) * c.d_loss.double()).sum())

    h = 1e-5
    slope = (value(h) - value(-h)) / (2 * h)
    _, dx, dw = B.cross_entropy_gradients(c.x, c.w, c.t, d_loss=c.d_loss)
    a, b = dx.double() * sx, dw.double() * sw
    # 1e-6 of the terms: the gradients' bound above; h^2 of third derivatives (1e-10 times some hundreds) and the difference's 2^-52 / h are less
    assert abs(float(a.sum() + b.sum()) - slope) <= 2e-6 * float(a.abs().sum() + b.abs().sum())


# Few rows of float data: sums of 32 channels, 16 multiplications each, joined one by one, are within the bound of a logit above; a gradient's sums, of the stretches of
# a block's threads, the threads and the blocks, have vocab / 16 steps at most; dw's 16.
@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 32, 33])
@pytest.mark.parametrize("d,vocab", [(4, 3), (4, 20011), (68, 2100), (260, 64), (1100, 4097), (2052, 20011)])
def test_few_rows_of_float_data(B, n, d, vocab):
    c = Case(n, d, vocab, torch.float32, n + d, 5.0, pad=4, ignored=0.2)
    c.t[-1] = c.t[-1].clamp_min(0)
    if n > 2:
        c.t[1] = -1
        c.x[1] = float("nan")
    check(c, B.cross_entropy(c.x, c.w, c.t))
    loss, dx, dw = B.cross_entropy_gradients(c.x, c.w, c.t, d_loss=c.d_loss)
    check(c, loss, dx, dw, c.d_loss)
    again = B.cross_entropy_gradients(c.x, c.w, c.t, d_loss=c.d_loss)
    assert torch.equal(again[0], loss) and torch.equal(again[1], dx) and torch.equal(again[2], dw)


@pytest.mark.parametrize("n", [1, 7, 30])
def test_few_rows_far_below_the_largest_logit(B, n):
    """A row's columns lie with several blocks, which agree on another reference."""
    c = Case(n, 128, 20011, torch.float32, 11, ignored=0.0)
    c.x[: (n + 1) // 2] *= 300.0
    check(c, B.cross_entropy(c.x, c.w, c.t))
    loss, dx, dw = B.cross_entropy_gradients(c.x, c.w, c.t, d_loss=c.d_loss)
    assert float(loss.max()) > 40
    check(c, loss, dx, dw, c.d_loss)


@pytest.mark.parametrize("n", [6, 16])
def test_few_rows_of_strided_outputs_parts_and_bad_rows(B, n):
    c = Case(n, 132, 4500, torch.float32, 21, pad=12, ignored=0.0)
    loss, dx, dw = B.cross_entropy_gradients(c.x, c.w, c.t, d_loss=c.d_loss)
    a = B.cross_entropy_gradients(c.x, c.w, c.t, d_loss=c.d_loss, with_dw=False)
    b = B.cross_entropy_gradients(c.x, c.w, c.t, d_loss=c.d_loss, with_dx=False)
    assert a[2] is None and b[1] is None and torch.equal(a[1], dx) and torch.equal(b[2], dw)
    out, wide = torch.full((n, 140), 5.0, device="cuda"), torch.full((4500, 140), 5.0, device="cuda")
    B.cross_entropy_gradients(c.x, c.w, c.t, d_loss=c.d_loss, dx=out[:, 4:136], dw=wide[:, 4:136])
    assert torch.equal(out[:, 4:136], dx) and torch.equal(wide[:, 4:136], dw)
    assert all(bool((t[:, :4] == 5).all() and (t[:, 136:] == 5).all()) for t in (out, wide))
    x = c.x.clone()
    x[2, 7] = float("nan")
    others = torch.arange(n, device="cuda") != 2
    bad = B.cross_entropy_gradients(x, c.w, c.t, d_loss=c.d_loss)
    assert bool(bad[0][2].isnan()) and bool(bad[1][2].isnan().all()) and bool(bad[2].isnan().all())
    assert torch.equal(bad[0][others], loss[others]) and torch.equal(bad[1][others], dx[others])
    # a target beyond the vocabulary is none, and reported
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    c.t[2] = 4500
    beyond = B.cross_entropy_gradients(x, c.w, c.t, d_loss=c.d_loss, status=status)
    c.t[2] = -1
    none = B.cross_entropy_gradients(x, c.w, c.t, d_loss=c.d_loss)
    assert int(status) != 0 and all(torch.equal(p, q) for p, q in zip(beyond, none))
    check(c, *none, c.d_loss)


def test_few_rows_captured_and_replayed(B):
    """Replays read what the tensors hold then."""
    c, other = Case(9, 260, 20011, torch.float32, 31), Case(9, 260, 20011, torch.float32, 32)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        B.cross_entropy_gradients(c.x, c.w, c.t, d_loss=c.d_loss)
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = B.cross_entropy_gradients(c.x, c.w, c.t, d_loss=c.d_loss)
    for source in (c, other):
        c.x.copy_(source.x)
        c.w.copy_(source.w)
        c.t.copy_(source.t)
        graph.replay()
        check(c, *got, c.d_loss)
