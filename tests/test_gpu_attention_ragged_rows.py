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
