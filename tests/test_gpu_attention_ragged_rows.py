"""Attention over ragged batches: rows that are in no sequence, and sequences without queries."""
import math

import pytest
import torch

from test_gpu_attention_ragged import BF16, F32, check, make, offsets, reference

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2501_17086_b200 import binding
    return binding


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("causal", [True, False])
def test_rows_of_q_but_no_queries(B, dtype, hd, causal):
    """A buffer for queries that holds none of them (q_len = 0): the gradients of the keys and values that are in a sequence are 0, the
    others stay as they were.  The offsets come from the kernel just before."""
    kl, at = [70, 0, 300, 1], 5
    q, d_o, o = (make(40, 4, hd, dtype, s) for s in (0, 1, 2))
    k, v = make(at + sum(kl) + 9, 2, hd, dtype, 3), make(at + sum(kl) + 9, 2, hd, dtype, 4)
    lse = torch.zeros(4, 40, device="cuda")
    there, none = offsets(kl, at), torch.zeros(len(kl) + 1, dtype=torch.int32, device="cuda")
    big = torch.ones(1 << 26, device="cuda")
    for _ in range(3):
        q_off, k_off = torch.full_like(none, -7), torch.full_like(none, -7)
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        dq, dk, dv = torch.full_like(q, 7.0), torch.full_like(k, 7.0), torch.full_like(v, 7.0)
        torch.cuda.synchronize()
        big.mul_(1.0)
        q_off.copy_(none)
        torch.add(there, 0, out=k_off)
        B.attention_backward(d_o, q, k, v, o, lse, q_offsets=q_off, kv_offsets=k_off, q_len=0, kv_len=300, causal=causal, dq=dq, dk=dk, dv=dv,
                             status=status)
        assert int(status) == 0 and bool((dq == 7).all())
        for t in (dk, dv):
            assert bool((t[at:at + sum(kl)] == 0).all())
            assert bool((t[:at] == 7).all()) and bool((t[at + sum(kl):] == 7).all())


@pytest.mark.parametrize("hd", [64, 80, 128])
@pytest.mark.parametrize("ql,kl,qh,kh", [([100, 128], [2100, 2048], 8, 8), ([128], [4096], 16, 4), ([33, 1, 128], [1025, 3000, 64], 4, 4)])
def test_merges_of_clusters_of_every_size(B, hd, ql, kl, qh, kh):
    """Clusters of two, four and eight blocks whose shares of the rows come in no whole number of steps, calls on one another's heels."""
    q, d_o = make(sum(ql), qh, hd, BF16, 1), make(sum(ql), qh, hd, BF16, 2)
    k, v = make(sum(kl), kh, hd, BF16, 3), make(sum(kl), kh, hd, BF16, 4)
    kw = dict(q_offsets=offsets(ql), kv_offsets=offsets(kl), q_len=max(ql), kv_len=max(kl), causal=True)
    o, lse = B.attention_forward(q, k, v, **kw)
    got = [(o, lse, *B.attention_backward(d_o, q, k, v, o, lse, **kw))]
    for _ in range(20):
        o, lse = B.attention_forward(q, k, v, **kw)
        got.append((o, lse, *B.attention_backward(d_o, q, k, v, o, lse, **kw)))
    want = reference(q, k, v, d_o, ql, kl, True, hd ** -0.5)
    for name, x in zip(("o", "lse", "dq", "dk", "dv"), got[0]):
        check(x, want[name], name)
    for other in got[1:]:
        assert all(torch.equal(a, b) for a, b in zip(got[0], other))


def test_rows_that_are_no_whole_number_of_sequences(B):
    """Refused: the rows that are left over would be in no sequence.  With the length given they are meant to be."""
    q, k = make(100, 4, 64, BF16, 0), make(99, 2, 64, BF16, 1)
    o, lse = B.attention_forward(q, k, k, sequences=3, q_len=33)
    for call in (lambda: B.attention_forward(q, k, k, sequences=3), lambda: B.attention_forward(k, k[:97], k[:97], sequences=3),
                 lambda: B.attention_backward(q, q, k, k, o, lse, sequences=3), lambda: B.attention_forward(q, k, k, sequences=0),
                 lambda: B.attention_forward(q, k, k, q_offsets=offsets([50, 50]), q_len=50)):
        with pytest.raises(B.HbpError) as e:
            call()
        assert e.value.code == 2
    B.attention_forward(k, k, k, sequences=3)
    B.attention_forward(q[:0], k[:0], k[:0], sequences=0)
    B.attention_forward(q, k, k, q_offsets=offsets([50, 40, 10]), q_len=50)


def spoil(*tensors):
    """NaN in the memory that new tensors of these sizes will have."""
    some = [torch.full(t.shape, math.nan, dtype=t.dtype, device="cuda") for t in tensors for _ in range(4)]
    del some


NEW = [([70, 0, 130], [70, 90, 131], 11, 19), ([3], [700], 0, 1), ([1] * 300, [2] * 300, 1, 0), ([0, 0], [0, 5], 40, 0)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("hd", [64, 40, 128])
@pytest.mark.parametrize("ql,kl,at,more", NEW)
def test_new_outputs_of_rows_in_no_sequence(B, dtype, hd, ql, kl, at, more):
    """0, and a log-sum-exp of -infinity, before the first sequence and behind the last; the others as ever."""
    rows = [at + sum(ql) + more, at + sum(kl) + more]
    q, d_o = make(rows[0], 4, hd, dtype, 0), make(rows[0], 4, hd, dtype, 1)
    k, v = make(rows[1], 2, hd, dtype, 2), make(rows[1], 2, hd, dtype, 3)
    want = reference(q, k, v, d_o, ql, kl, True, hd ** -0.5, q_at=at, k_at=at)  # (0 outside)
    kw = dict(q_offsets=offsets(ql, at), kv_offsets=offsets(kl, at), q_len=max(ql), kv_len=max(kl))
    spoil(q, torch.empty(4, rows[0]))
    o, lse = B.attention_forward(q, k, v, **kw)
    spoil(q, k, v)
    got = (o, lse, *B.attention_backward(d_o, q, k, v, o, lse, **kw))
    for name, x in zip(("o", "lse", "dq", "dk", "dv"), got):
        check(x, want[name], name)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_new_outputs_where_lengths_leave_rows_over(B, dtype):
    q, k, v, d_o = (make(100, 2, 64, dtype, s) for s in range(4))
    want = reference(q, k, v, d_o, [33, 33], [40, 40], True, 0.125)
    kw = dict(sequences=2, q_len=33, kv_len=40)
    spoil(q, torch.empty(2, 100))
    o, lse = B.attention_forward(q, k, v, **kw)
    spoil(q, k, v)
    given = torch.full_like(k, 7.0)
    got = (o, lse, *B.attention_backward(d_o, q, k, v, o, lse, dk=given, **kw))
    assert bool((given[80:] == 7).all())  # what is given keeps its rows
    given[80:] = 0
    for name, x in zip(("o", "lse", "dq", "dk", "dv"), got):
        check(x, want[name], name)
    none = torch.zeros(1, dtype=torch.int32, device="cuda")
    spoil(q, torch.empty(2, 100))
    o, lse = B.attention_forward(q, k, v, q_offsets=none, kv_offsets=none, q_len=0, kv_len=0)  # no sequences at all
    assert bool((o == 0).all()) and bool((lse == -math.inf).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("off", [[0, 40, 30, 90], [0, 40, 80, 101], [-3, 40, 80, 90], [0, 70, 80, 90], [90, 40, 60, 20]])
@pytest.mark.parametrize("side", ["q", "kv"])
def test_new_outputs_of_skipped_sequences(B, dtype, off, side):
    """Bad offsets of either side: the sequence's rows of both are 0, those of the others what they are."""
    q, k, v, d_o = (make(100, 2, 64, dtype, s) for s in range(4))
    fine, bad = torch.tensor([0, 30, 60, 90], device="cuda", dtype=torch.int32), torch.tensor(off, device="cuda", dtype=torch.int32)
    kw = dict(q_offsets=bad if side == "q" else fine, kv_offsets=fine if side == "q" else bad, q_len=50, kv_len=50)
    full = lambda: torch.full_like(q, 0.0)  # noqa: E731
    o, lse = full(), torch.full((2, 100), -math.inf, device="cuda")
    want = [o, lse, full(), full(), full()]
    B.attention_forward(q, k, v, o=o, lse=lse, **kw)
    B.attention_backward(d_o, q, k, v, o, lse, dq=want[2], dk=want[3], dv=want[4], **kw)
    spoil(q, lse)
    o, lse = B.attention_forward(q, k, v, **kw)
    spoil(q, k, v)
    got = (o, lse, *B.attention_backward(d_o, q, k, v, o, lse, **kw))
    for name, a, b in zip(("o", "lse", "dq", "dk", "dv"), got, want):
        assert torch.equal(a, b), name


def test_new_outputs_of_a_replayed_graph(B):
    q, k, v, d_o = (make(200, 2, 64, BF16, s) for s in range(4))
    off = offsets([100, 100])
    kw = dict(q_offsets=off, kv_offsets=off, q_len=200, kv_len=200)
    o, lse = B.attention_forward(q, k, v, **kw)
    B.attention_backward(d_o, q, k, v, o, lse, **kw)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o, lse = B.attention_forward(q, k, v, **kw)
        got = (o, lse, *B.attention_backward(d_o, q, k, v, o, lse, **kw))
    for at, lens in ((0, [100, 100]), (7, [90, 20]), (50, [0, 150])):
        off.copy_(offsets(lens, at))
        graph.replay()
        want = reference(q, k, v, d_o, lens, lens, True, 0.125, q_at=at, k_at=at)
        for name, x in zip(("o", "lse", "dq", "dk", "dv"), got):
            check(x, want[name], name)


@pytest.mark.parametrize("off", [[0, 500, 480, 700, 1500, 1490, 1600, 2400], [900, 1300, 1250, 100, 500, 500, 3000, 2999], [5, 20, 21, 22, 23, 24, 25, 30]])
@pytest.mark.parametrize("many", [False, True])
def test_new_outputs_of_many_sequences_some_of_them_skipped(B, off, many):
    """Rows in no sequence that is taken are 0, wherever the offsets go; more sequences than a launch's warps have lanes."""
    if many:
        off = off + [off[-1] + i // 20 for i in range(1, 2000 * 20)]
    rows = 2600
    q, d_o = make(rows, 2, 8, F32, 1), make(rows, 2, 8, F32, 2)
    o32 = torch.tensor(off, device="cuda", dtype=torch.int32)
    kw = dict(q_offsets=o32, kv_offsets=o32, q_len=450, kv_len=450)
    taken = torch.zeros(rows, dtype=torch.bool)
    for a, b in zip(off, off[1:]):
        if 0 <= a <= b <= rows and b - a <= 450:
            taken[a:b] = True
    spoil(q, torch.empty(2, rows))
    o, lse = B.attention_forward(q, q, q, **kw)
    spoil(q, q, q)
    grads = B.attention_backward(d_o, q, q, q, o, lse, **kw)
    taken = taken.cuda()
    assert bool((lse[:, ~taken] == -math.inf).all()) and bool(torch.isfinite(lse[:, taken]).all())
    for x in (o, *grads):
        assert bool((x[~taken] == 0).all()) and bool(torch.isfinite(x).all())
    assert bool((o[taken] != 0).any(-1).all()) if bool(taken.any()) else True
