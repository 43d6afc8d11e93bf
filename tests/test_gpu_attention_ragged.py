"""Attention over ragged batches and its backward pass against the formulas in 64 bits.

Bounds, element by element, u = half a step of the type (bf16 2^-8, float 2^-24), f = 2^-24:
  a score is off by (head_dim + 4) f scale |q| . |k|, so that a probability is off by r = that + 2^-19 (exponential, log-sum-exp) relatively;
  bf16 probabilities and ds are rounded once more (u) before they are multiplied;
  a sum of n products adds n f times the sum of their magnitudes (2 n f on the tensor cores, which truncate);
  the result is rounded once (u).  D takes over what o is off by."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
U = {F32: 2.0 ** -24, BF16: 2.0 ** -8}


@pytest.fixture(scope="module")
def B():
    from paper_2501_17086_b200 import binding
    return binding


def reference(q, k, v, d_o, ql, kl, causal, scale, o_given=None, q_at=0, k_at=0):
    """{name: (value, bound)} in 64 bits for the sequences of lengths ql, kl one after the other from rows q_at, k_at on."""
    t = q.dtype
    u, f = U[t], 2.0 ** -24
    pu = u if t == BF16 else 0.0
    q, k, v, d_o = (x.double() for x in (q, k, v, d_o))
    group, hd = q.shape[1] // k.shape[1], q.shape[2]
    z = lambda x: (torch.zeros_like(x), torch.zeros_like(x))  # noqa: E731
    out = {"o": z(q), "dq": z(q), "dk": z(k), "dv": z(v),
           "lse": (torch.full(q.shape[:2], -math.inf, dtype=torch.float64, device=q.device), torch.zeros(q.shape[:2], dtype=torch.float64, device=q.device))}
    for nq, nk in zip(ql, kl):
        a, b = slice(q_at, q_at + nq), slice(k_at, k_at + nk)
        q_at, k_at = q_at + nq, k_at + nk
        if nq == 0 or nk == 0:
            continue
        seen = torch.ones(nq, nk, dtype=torch.bool, device=q.device)
        if causal:
            seen = seen.tril(nk - nq)
        some = seen.any(1)
        for h in range(q.shape[1]):
            g = h // group
            Q, K, V, G = q[a, h], k[b, g], v[b, g], d_o[a, h]
            s = (Q @ K.T * scale).masked_fill(~seen, -math.inf)
            lse = torch.logsumexp(s, 1)
            p = torch.exp(s - torch.where(some, lse, 0.0)[:, None])
            es = (hd + 4) * f * abs(scale) * (Q.abs() @ K.abs().T)
            r = torch.where(seen, es + (es * p).sum(1, keepdim=True) + 2.0 ** -19 + 2 * nk * f, 0.0)
            pe = p * (r + pu)  # what a probability is off by when it is multiplied
            o = p @ V
            oe = pe @ V.abs() + 2 * nk * f * (p @ V.abs())
            oe = oe + u * (o.abs() + oe)
            out["o"][0][a, h], out["o"][1][a, h] = o, oe
            out["lse"][0][a, h] = lse
            out["lse"][1][a, h] = torch.where(some, es.amax(1) + 2.0 ** -19 + 2 * nk * f + 2.0 ** -23 * lse.abs(), 0.0)
            dp = G @ V.T
            D = (G * o).sum(1, keepdim=True)
            De = (G.abs() * oe).sum(1, keepdim=True) + 2 * hd * f * (G.abs() * o.abs()).sum(1, keepdim=True)
            ds = p * (dp - D)
            dse = p * (r * (dp - D).abs() + De + 2 * hd * f * (G.abs() @ V.abs().T))
            dse = dse + pu * (ds.abs() + dse)
            out["dv"][0][b, g] += p.T @ G
            out["dv"][1][b, g] += pe.T @ G.abs() + 2 * nq * f * (p.T @ G.abs())
            out["dk"][0][b, g] += scale * (ds.T @ Q)
            out["dk"][1][b, g] += abs(scale) * (dse.T @ Q.abs() + 2 * nq * f * (ds.abs().T @ Q.abs()))
            dq = scale * (ds @ K)
            dqe = abs(scale) * (dse @ K.abs() + 2 * nk * f * (ds.abs() @ K.abs()))
            out["dq"][0][a, h], out["dq"][1][a, h] = dq, dqe + u * (dq.abs() + dqe)
    for n in ("dk", "dv"):
        y, e = out[n]
        e += group * 2 * f * y.abs() + u * (y.abs() + e)
    out["lse"] = tuple(x.T for x in out["lse"])
    return out


def check(got, want, name):
    y, e = want
    got = got.double()
    fin = torch.isfinite(y)
    assert torch.equal(got[~fin], y[~fin]), name
    over = (got - y).abs()[fin] - e[fin] - 1e-30
    assert bool((over <= 0).all()), (name, float(over.max()), float((got - y)[fin].norm() / y[fin].norm()))


def make(rows, heads, hd, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(rows, heads, hd, generator=g, device="cuda").to(dtype)


def offsets(lengths, at=0):
    out = [at]
    for n in lengths:
        out.append(out[-1] + n)
    return torch.tensor(out, device="cuda", dtype=torch.int32)


def case(B, dtype, ql, kl, qh, kh, hd, causal, ragged=True, scale=None, seed=0):
    q, d_o = make(sum(ql), qh, hd, dtype, seed), make(sum(ql), qh, hd, dtype, seed + 1)
    k, v = make(sum(kl), kh, hd, dtype, seed + 2), make(sum(kl), kh, hd, dtype, seed + 3)
    kw = dict(q_offsets=offsets(ql), kv_offsets=offsets(kl), q_len=max(ql), kv_len=max(kl)) if ragged else dict(sequences=len(ql))
    kw.update(causal=causal, scale=scale, status=torch.zeros(1, dtype=torch.int32, device="cuda"))
    o, lse = B.attention_forward(q, k, v, **kw)
    dq, dk, dv = B.attention_backward(d_o, q, k, v, o, lse, **kw)
    assert int(kw["status"]) == 0
    want = reference(q, k, v, d_o, ql, kl, causal, hd ** -0.5 if scale is None else scale)
    for name, got in (("o", o), ("lse", lse), ("dq", dq), ("dk", dk), ("dv", dv)):
        check(got, want[name], name)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("n", [1, 2, 17, 63, 64, 65, 127, 128, 129, 200, 256, 385])
def test_lengths(B, dtype, causal, n):
    case(B, dtype, [n], [n], 2, 2, 64, causal, ragged=False)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("nq,nk", [(1, 300), (300, 1), (1, 1000), (65, 130), (130, 65), (128, 129), (129, 128), (200, 72), (5, 64), (192, 320)])
def test_unequal_lengths(B, dtype, causal, nq, nk):
    """More queries than keys leave the first queries of a causal sequence without any."""
    case(B, dtype, [nq, nq], [nk, nk], 2, 1, 64, causal, ragged=False)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("hd", [8, 16, 24, 56, 64, 72, 80, 96, 120, 128])
def test_head_widths(B, dtype, hd):
    case(B, dtype, [150, 33], [150, 33], 2, 2, hd, True)
    case(B, dtype, [70], [140], 2, 1, hd, False)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("qh,kh", [(1, 1), (4, 1), (6, 2), (8, 4), (5, 5)])
@pytest.mark.parametrize("hd", [64, 128])
def test_grouped_heads(B, dtype, qh, kh, hd):
    case(B, dtype, [130, 64, 7], [130, 64, 7], qh, kh, hd, True)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("ql,kl", [([0, 5, 0, 130, 1, 0], [0, 5, 3, 130, 1, 0]), ([3, 0, 64], [0, 7, 128]), ([100, 200, 300], [300, 200, 100]),
                                   ([1] * 20, [7] * 20), ([0, 0], [4, 2]), ([9], [9])])
@pytest.mark.parametrize("hd", [64, 128])
def test_ragged(B, dtype, causal, ql, kl, hd):
    case(B, dtype, ql, kl, 4, 2, hd, causal)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_large_scores(B, dtype):
    """Scores of some hundreds: the maximum moves by more than float's exponent range allows without one."""
    case(B, dtype, [200], [200], 2, 2, 64, True, scale=6.0)
    case(B, dtype, [130], [300], 1, 1, 128, False, scale=-3.0)
    case(B, dtype, [130], [130], 1, 1, 64, True, scale=0.0)


def test_long(B):
    case(B, BF16, [2100], [2100], 2, 1, 128, True)
    case(B, BF16, [1500], [2300], 2, 2, 64, False)
    case(B, F32, [1100], [1100], 2, 1, 64, True)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("hd", [64, 128, 40])
@pytest.mark.parametrize("causal", [True, False])
def test_what_is_in_no_sequence_is_neither_read_nor_written(B, dtype, hd, causal):
    """NaN before the first sequence and behind the last in every input; sequences end inside tiles next to each other."""
    ql, kl, at = [70, 3, 130], [70, 90, 131], 11
    rows = [at + sum(ql) + 19, at + sum(kl) + 23]
    q, d_o = make(rows[0], 4, hd, dtype, 0), make(rows[0], 4, hd, dtype, 1)
    k, v = make(rows[1], 2, hd, dtype, 2), make(rows[1], 2, hd, dtype, 3)
    want = reference(q, k, v, d_o, ql, kl, causal, hd ** -0.5, q_at=at, k_at=at)
    for t, n in ((q, ql), (d_o, ql), (k, kl), (v, kl)):
        t[:at] = math.nan
        t[at + sum(n):] = math.nan
    kw = dict(q_offsets=offsets(ql, at), kv_offsets=offsets(kl, at), q_len=140, kv_len=300, causal=causal)
    full = lambda t: torch.full_like(t, 7.0)  # noqa: E731
    o, lse = full(q), torch.full((4, rows[0]), 7.0, device="cuda")
    B.attention_forward(q, k, v, o=o, lse=lse, **kw)
    dq, dk, dv = full(q), full(k), full(v)
    o[:at] = math.nan
    B.attention_backward(d_o, q, k, v, o, lse, dq=dq, dk=dk, dv=dv, **kw)
    for name, got, n in (("o", o, ql), ("dq", dq, ql), ("dk", dk, kl), ("dv", dv, kl)):
        inside = slice(at, at + sum(n))
        check(got[inside], tuple(x[inside] for x in want[name]), name)
        outside = torch.cat([got[:at], got[at + sum(n):]])
        assert bool(((outside == 7) | ((name == "o") & outside.isnan())).all()), name
    check(lse[:, at:at + sum(ql)], tuple(x[:, at:at + sum(ql)] for x in want["lse"]), "lse")
    assert bool((lse[:, :at] == 7).all()) and bool((lse[:, at + sum(ql):] == 7).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_another_sequence_that_is_not_finite_stays_by_itself(B, dtype, bad):
    """A sequence between two others, within their last tiles, holds values that are not finite."""
    ql = kl = [67, 40, 66]
    ts = [make(173, 2, 64, dtype, s) for s in range(4)]
    want = reference(*(ts[i] for i in (0, 1, 2, 3)), ql, kl, True, 0.125)
    for t in ts:
        t[67:107] = bad
    q, k, v, d_o = ts
    kw = dict(q_offsets=offsets(ql), kv_offsets=offsets(kl), q_len=67, kv_len=67)
    o, lse = B.attention_forward(q, k, v, **kw)
    grads = B.attention_backward(d_o, q, k, v, o, lse, **kw)
    for part in (slice(0, 67), slice(107, 173)):
        for name, got in zip(("o", "dq", "dk", "dv"), (o, *grads)):
            check(got[part], tuple(x[part] for x in want[name]), name)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("hd", [64, 128])
def test_parts_of_one_buffer(B, dtype, hd):
    """q, k and v as column blocks of one [rows][3 heads] buffer, their gradients likewise; heads before rows for the output."""
    rows, heads = 150, 3
    buf, d_o = make(rows, 3 * heads, hd, dtype, 0), make(heads, rows, hd, dtype, 1).transpose(0, 1)
    q, k, v = buf.split(heads, 1)
    grad = torch.full_like(buf, 7.0)
    o = torch.empty(heads, rows, hd, dtype=dtype, device="cuda").transpose(0, 1)
    _, lse = B.attention_forward(q, k, v, o=o)
    dq, dk, dv = grad.split(heads, 1)
    B.attention_backward(d_o, q, k, v, o, lse, dq=dq, dk=dk, dv=dv)
    want = reference(q, k, v, d_o, [rows], [rows], True, hd ** -0.5)
    for name, got in (("o", o), ("lse", lse), ("dq", dq), ("dk", dk), ("dv", dv)):
        check(got, want[name], name)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_broadcast_inputs(B, dtype):
    """One key head seen as four (stride 0), one row of d_o seen as all: the gradients are those of the copies, every head's own."""
    n, hd = 140, 64
    q, k, v, d_o = make(n, 4, hd, dtype, 0), make(n, 1, hd, dtype, 1).expand(n, 4, hd), make(n, 1, hd, dtype, 2).expand(n, 4, hd), make(1, 4, hd, dtype, 3).expand(n, 4, hd)
    o, lse = B.attention_forward(q, k, v)
    grads = B.attention_backward(d_o, q, k, v, o, lse)
    want = reference(q, k, v, d_o, [n], [n], True, hd ** -0.5)
    for name, got in zip(("o", "lse", "dq", "dk", "dv"), (o, lse, *grads)):
        check(got, want[name], name)
    with pytest.raises(B.HbpError) as e:
        B.attention_backward(d_o, q, k, v, o, lse, dk=make(n, 1, hd, dtype, 4).expand(n, 4, hd))
    assert e.value.code == 2


def test_narrowest_heads(B):
    case(B, F32, [70], [70], 3, 3, 4, True)
    case(B, F32, [70], [130], 2, 1, 12, False)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_beyond_32_bits(B, dtype):
    """Rows 2^23 elements apart, 300 of them: elements beyond 2^31 from the first."""
    n, hd = 300, 64
    buf = torch.empty((n << 23) + 256, device="cuda", dtype=dtype)
    far = buf.as_strided((n, 2, hd), (1 << 23, hd, 1))
    far.copy_(make(n, 2, hd, dtype, 0))
    k, v, d_o = (make(n, 2, hd, dtype, s) for s in (1, 2, 3))
    want = reference(far.clone(), k, v, d_o, [n], [n], True, 0.125)
    o, lse = B.attention_forward(far, k, v)
    check(o, want["o"], "o")
    dq, dk, dv = B.attention_backward(d_o, far, k, v, o, lse)
    for name, got in (("dq", dq), ("dk", dk), ("dv", dv)):
        check(got, want[name], name)
    want = reference(k, far.clone(), v, d_o, [n], [n], True, 0.125)  # as keys
    o, lse = B.attention_forward(k, far, v)
    check(o, want["o"], "o")
    B.attention_backward(d_o, k, far.clone(), v, o, lse, dk=far)
    check(far, want["dk"], "dk")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("off", [[0, 40, 30, 90], [0, 40, 80, 101], [-3, 40, 80, 90], [0, 70, 80, 90]])
def test_bad_offsets_are_reported_and_skipped(B, dtype, off):
    """Offsets that decrease, leave the tensor, begin before it or span more than q_len rows: that sequence is an empty one."""
    q, k, v, d_o = (make(100, 2, 64, dtype, s) for s in range(4))
    kw = dict(q_offsets=torch.tensor(off, device="cuda", dtype=torch.int32), kv_offsets=torch.tensor([0, 30, 60, 90], device="cuda", dtype=torch.int32),
              q_len=50, kv_len=50, status=torch.zeros(1, dtype=torch.int32, device="cuda"))
    o, lse = torch.full_like(q, 7.0), torch.full((2, 100), 7.0, device="cuda")
    B.attention_forward(q, k, v, o=o, lse=lse, **kw)
    assert int(kw["status"]) == 1
    kw["status"].zero_()
    grads = [torch.full_like(q, 7.0) for _ in range(3)]
    B.attention_backward(d_o, q, k, v, o, lse, dq=grads[0], dk=grads[1], dv=grads[2], **kw)
    assert int(kw["status"]) == 1
    bad = [i for i in range(3) if off[i] < 0 or off[i + 1] < off[i] or off[i + 1] > 100 or off[i + 1] - off[i] > 50]
    assert bad
    for i in range(3):
        assert bool((grads[1][30 * i:30 * i + 30] == 7).all()) == (i in bad)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_runs_agree_bit_for_bit_and_calls_on_two_streams_do_not_meet(B, dtype):
    q, k, v, d_o = (make(500, 4, 64, dtype, s) for s in range(4))
    kw = dict(q_offsets=offsets([200, 0, 300]), kv_offsets=offsets([150, 50, 300]), q_len=300, kv_len=300)

    def call():
        o, lse = B.attention_forward(q, k, v, **kw)
        return (o, lse, *B.attention_backward(d_o, q, k, v, o, lse, **kw))

    first = call()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(5):
        with torch.cuda.stream(side):
            there = call()
        here = call()
        torch.cuda.synchronize()
        for a, b, c in zip(first, here, there):
            assert torch.equal(a, b) and torch.equal(a, c)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_captured_and_replayed_with_other_offsets(B, dtype):
    q, k, v, d_o = (make(260, 2, 64, dtype, s) for s in range(4))
    off = offsets([100, 160])
    kw = dict(q_offsets=off, kv_offsets=off, q_len=260, kv_len=260)
    o, lse = B.attention_forward(q, k, v, **kw)
    B.attention_backward(d_o, q, k, v, o, lse, **kw)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o, lse = B.attention_forward(q, k, v, **kw)
        dq, dk, dv = B.attention_backward(d_o, q, k, v, o, lse, **kw)
    for lens in ([100, 160], [259, 1], [0, 260]):
        off.copy_(offsets(lens))
        graph.replay()
        want = reference(q, k, v, d_o, lens, lens, True, 0.125)
        for name, got in (("o", o), ("lse", lse), ("dq", dq), ("dk", dk), ("dv", dv)):
            check(got, want[name], name)


def test_gradients_by_differences(B):
    """sum(o * w) in float, moved along random directions: the gradient's product with them, to the difference's own order."""
    q, k, v, w = (make(90, 2, 64, F32, s) for s in range(4))
    o, lse = B.attention_forward(q, k, v)
    grads = B.attention_backward(w, q, k, v, o, lse)
    h = 2.0 ** -7
    for i, g in enumerate(grads):
        d = make(90, 2, 64, F32, 10 + i)
        at = lambda s: [t + s * h * d if j == i else t for j, t in enumerate((q, k, v))]  # noqa: E731
        diff = sum(((B.attention_forward(*at(s))[0].double() * w.double()).sum() * s for s in (1, -1))) / (2 * h)
        dot = (g.double() * d.double()).sum()
        # third derivatives of a softmax of scores with |score| < 5 along a step of h: h^2 / 6 * |d score|^3 stays below 0.05 of |o| |w|
        scale = float((o.double().abs() * w.double().abs()).sum())
        assert abs(float(diff - dot)) <= 0.05 * h * scale


def test_empty_tensors(B):
    q, k = make(0, 2, 64, BF16, 0), make(5, 2, 64, BF16, 1)
    o, lse = B.attention_forward(q, k, k)
    assert o.shape == (0, 2, 64) and lse.shape == (2, 0)
    dq, dk, dv = B.attention_backward(q, q, k, k, o, lse)
    assert bool((dk == 0).all()) and bool((dv == 0).all())
    o, lse = B.attention_forward(k, q, q, causal=False)
    assert bool((o == 0).all()) and bool((lse == -math.inf).all())
    dq, dk, dv = B.attention_backward(k, k, q, q, o, lse, causal=False)
    assert bool((dq == 0).all()) and dk.shape == (0, 2, 64)


def test_refusals_of_the_binding(B):
    q, k = make(6, 4, 64, F32, 0), make(6, 2, 64, F32, 1)
    o, lse = B.attention_forward(q, k, k)
    off = offsets([2, 4])
    for call in (lambda: B.attention_forward(q, k[:, :, :32], k), lambda: B.attention_forward(q, k.bfloat16(), k.bfloat16()),
                 lambda: B.attention_forward(q, k, k, q_offsets=off), lambda: B.attention_forward(q, k, k, q_offsets=off.long(), q_len=6),
                 lambda: B.attention_forward(q, k, k, sequences=3, q_offsets=off, q_len=6), lambda: B.attention_forward(q, k, k, lse=lse.T),
                 lambda: B.attention_forward(q, k, k, sequences=2, q_len=4), lambda: B.attention_backward(q[:5], q, k, k, o, lse),
                 lambda: B.attention_forward(q[:, :3], k, k)):
        with pytest.raises(B.HbpError) as e:
            call()
        assert e.value.code == 2
    with pytest.raises(B.HbpError) as e:
        B.attention_backward(q, q, k, k, o, lse, scratch=torch.empty(16, device="cuda"))
    assert e.value.code == 5
    with pytest.raises(B.HbpError) as e:
        B.attention_forward(q.half(), k.half(), k.half())
    assert e.value.code == 3


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_an_attention_step_with_rotary_positions(B, dtype):
    """Turn, attend, and back: the run of them as a decoder's step uses it, against the same in 64 bits by automatic differentiation."""
    rows, qh, kh, hd = 140, 4, 2, 64
    q, k, v, w = make(rows, qh, hd, dtype, 0), make(rows, kh, hd, dtype, 1), make(rows, kh, hd, dtype, 2), make(rows, qh, hd, dtype, 3)
    off = offsets([60, 80])
    pos = torch.cat([torch.arange(60), torch.arange(80)]).cuda()
    kw = dict(q_offsets=off, kv_offsets=off, q_len=80, kv_len=80)
    qr, kr = B.rotary(q, k, positions=pos)
    o, lse = B.attention_forward(qr, kr, v, **kw)
    dq, dk, dv = B.attention_backward(w, qr, kr, v, o, lse, **kw)
    dq, dk = B.rotary(dq, dk, positions=pos, inverse=True, q_out=dq, k_out=dk)

    a, b, c = (t.double().requires_grad_() for t in (q, k, v))
    angle = pos.double()[:, None] * 10000.0 ** (-torch.arange(0, hd, 2, device="cuda", dtype=torch.float64) / hd)

    def turn(x):
        x0, x1 = x.chunk(2, -1)
        cs, sn = angle.cos()[:, None], angle.sin()[:, None]
        return torch.cat([x0 * cs - x1 * sn, x1 * cs + x0 * sn], -1)

    out = []
    for lo, hi in ((0, 60), (60, 140)):
        Q, K, V = turn(a)[lo:hi].transpose(0, 1), turn(b)[lo:hi].transpose(0, 1).repeat_interleave(2, 0), c[lo:hi].transpose(0, 1).repeat_interleave(2, 0)
        s = (Q @ K.transpose(1, 2)) * hd ** -0.5
        s = s.masked_fill(~torch.ones(hi - lo, hi - lo, dtype=torch.bool, device="cuda").tril(), -math.inf)
        out.append((torch.softmax(s, -1) @ V).transpose(0, 1))
    y = torch.cat(out)
    y.backward(w.double())
    # roundings to the type on the way of each result, of relative size u each and at random: q, k turned (entering scores of size up to 5),
    # p, o, ds, the gradient and its turn; in the norm at most 5 * 2 + 5 of them
    tol = 15 * U[dtype] if dtype == BF16 else 15 * 64 * U[dtype]
    for got, want in ((o, y), (dq, a.grad), (dk, b.grad), (dv, c.grad)):
        assert float((got.double() - want).norm() / want.norm()) <= tol


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("hd", [40, 64, 72, 128])
@pytest.mark.parametrize("ql,kl,qh,kh", [([1], [4096], 4, 1), ([3, 128, 0, 130], [4100, 70, 0, 1], 2, 1), ([4200], [130], 1, 1),
                                         ([1100, 5], [1100, 64], 1, 1), ([512, 3], [100, 900], 8, 1), ([2, 1], [1030, 1], 3, 3)])
def test_walks_that_several_blocks_share(B, dtype, causal, hd, ql, kl, qh, kh):
    """Few blocks with long walks; sequences with fewer tiles than blocks leave some of them nothing.  Putting parts together multiplies them by an
    exponential, which the 2^-19 of a probability hold as well (it is off by 2^-21 at most)."""
    case(B, dtype, ql, kl, qh, kh, hd, causal)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("hd", [64, 128])
def test_shared_walks_agree_bit_for_bit_and_keep_to_themselves(B, dtype, hd):
    """Runs agree; what is in no sequence is NaN and stays as it was; a row of large scores and one of keys that are all the same among the rows."""
    ql, kl = [70, 2], [2050, 4097]
    q, d_o = make(80, 4, hd, dtype, 1), make(80, 4, hd, dtype, 2)
    k, v = make(6200, 2, hd, dtype, 3), make(6200, 2, hd, dtype, 4)
    q[3 + 5] *= 50
    k[10 + 2050:10 + 2050 + 300] = k[10 + 2050].clone()
    for x, at, n in ((q, 3, 72), (d_o, 3, 72), (k, 10, 6147), (v, 10, 6147)):
        x[:at], x[at + n:] = math.nan, math.nan
    kw = dict(q_offsets=offsets(ql, 3), kv_offsets=offsets(kl, 10), q_len=70, kv_len=4097, causal=True, status=torch.zeros(1, dtype=torch.int32, device="cuda"))
    want = reference(q, k, v, d_o, ql, kl, True, hd ** -0.5, q_at=3, k_at=10)
    first = None
    for _ in range(3):
        o, lse = torch.full_like(q, 7), torch.full((4, 80), 7.0, device="cuda")
        dq, dk, dv = torch.full_like(q, 7), torch.full_like(k, 7), torch.full_like(v, 7)
        B.attention_forward(q, k, v, o=o, lse=lse, **kw)
        B.attention_backward(d_o, q, k, v, o, lse, dq=dq, dk=dk, dv=dv, **kw)
        got = [o, lse, dq, dk, dv]
        if first is None:
            first = [x.clone() for x in got]
        assert all(torch.equal(a, b) for a, b in zip(got, first))
    assert int(kw["status"]) == 0
    for name, x, at, n in (("o", o, 3, 72), ("dq", dq, 3, 72), ("dk", dk, 10, 6147), ("dv", dv, 10, 6147)):
        check(x[at:at + n], tuple(y[at:at + n] for y in want[name]), name)
        assert bool((x[:at] == 7).all()) and bool((x[at + n:] == 7).all())
    check(lse[:, 3:75], tuple(y[:, 3:75] for y in want["lse"]), "lse")
    assert bool((lse[:, :3] == 7).all()) and bool((lse[:, 75:] == 7).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("hd", [64, 72, 128])
@pytest.mark.parametrize("ql,kl,qh,kh", [([1], [70], 2, 1), ([1] * 5, [1, 64, 65, 300, 2000], 8, 2), ([4, 0, 1, 3], [200, 5, 0, 1300], 12, 4),
                                         ([21, 20], [21, 700], 3, 1), ([16, 16], [90, 16], 4, 1), ([1, 1], [33, 1100], 64, 1), ([2, 1], [40, 3], 34, 1), ([7], [3], 5, 1),
                                         ([1] * 40, [1 + 61 * i % 200 for i in range(40)], 8, 2), ([i % 4 for i in range(30)], [37 * i % 150 for i in range(30)], 12, 4),
                                         ([1, 2, 1, 0], [4096, 100, 3000, 5], 16, 4), ([1] * 6, [300, 1, 64, 65, 0, 128], 64, 1),
                                         ([21 - i % 3 for i in range(100)], [30 - i % 25 for i in range(100)], 3, 1), ([8] * 20, [1040 - 50 * i for i in range(20)], 16, 2)])
def test_few_queries_of_many_heads_to_a_key_head(B, dtype, causal, hd, ql, kl, qh, kh):
    """All query heads of a key head in one block, and the groups that are just too many for that."""
    case(B, dtype, ql, kl, qh, kh, hd, causal)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("kv", [50, 1100])
def test_single_queries_from_and_to_parts_of_larger_buffers(B, hd, kv):
    n, qh, kh = 40, 8, 2
    qkv = make(n, 2 * qh + 3, hd + 8, BF16, 1)
    q = qkv[:, 1:2 * qh + 1:2, :hd]
    k, v = make(n * kv, kh, hd, BF16, 2), make(n * kv, kh, hd, BF16, 3)
    buf = torch.full((n, qh + 2, hd + 16), 7.0, dtype=BF16, device="cuda")
    lse = torch.full((qh, n), 7.0, device="cuda")
    o, _ = B.attention_forward(q, k, v, sequences=n, o=buf[:, 1:1 + qh, 8:8 + hd], lse=lse)
    want = reference(q, k, v, torch.zeros_like(q), [1] * n, [kv] * n, True, hd ** -0.5)
    check(o, want["o"], "o")
    check(lse, want["lse"], "lse")
    rest = buf.clone()
    rest[:, 1:1 + qh, 8:8 + hd] = 7
    assert bool((rest == 7).all())


def test_shared_walks_on_two_streams_and_replayed(B):
    """Calls whose blocks wait for others of their cluster run beside each other, 64 and 128 channels wide, also from a graph with other offsets."""
    calls = []
    for hd, ql, kl, qh, kh in ((64, [40, 100], [1100, 1500], 8, 4), (128, [1, 2], [2000, 1030], 32, 8)):
        q, d_o = make(sum(ql), qh, hd, BF16, hd), make(sum(ql), qh, hd, BF16, hd + 1)
        k, v = make(sum(kl), kh, hd, BF16, hd + 2), make(sum(kl), kh, hd, BF16, hd + 3)
        kw = dict(q_offsets=offsets(ql), kv_offsets=offsets(kl), q_len=max(ql), kv_len=max(kl))

        def call(q=q, k=k, v=v, d_o=d_o, kw=kw):
            o, lse = B.attention_forward(q, k, v, **kw)
            return (o, lse, *B.attention_backward(d_o, q, k, v, o, lse, **kw))

        calls.append((call, q, k, v, d_o, kw, ql, kl, hd))
    first = [c[0]() for c in calls]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for i in range(20):
        with torch.cuda.stream(side):
            there = [calls[i % 2][0]() for _ in range(3)]
        here = [calls[1 - i % 2][0]() for _ in range(3)]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for x in there for a, b in zip(first[i % 2], x))
        assert all(torch.equal(a, b) for x in here for a, b in zip(first[1 - i % 2], x))
    for call, q, k, v, d_o, kw, ql, kl, hd in calls:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = call()
        for turned in (False, True):
            ql, kl = (ql[::-1], kl[::-1]) if turned else (ql, kl)
            kw["q_offsets"].copy_(offsets(ql))
            kw["kv_offsets"].copy_(offsets(kl))
            graph.replay()
            want = reference(q, k, v, d_o, ql, kl, True, hd ** -0.5)
            for name, x in zip(("o", "lse", "dq", "dk", "dv"), got):
                check(x, want[name], name)
