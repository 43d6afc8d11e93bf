"""Cross entropy with scratch that was made for another number of rows, and whatever it held before.  Bounds as in test_gpu_cross_entropy.py: they allow for
any order of dx's sums."""
import pytest
import torch

from test_gpu_cross_entropy import Case, check

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2501_17086_b200 import binding
    return binding


# (rows, rows that the scratch is made for: it is less than these have)
@pytest.mark.parametrize("dtype,n,more,d,vocab", [(torch.bfloat16, 1007, 1008, 2048, 4099), (torch.bfloat16, 256, 257, 1024, 32003), (torch.float32, 1024, 1025, 520, 8111)])
def test_scratch_of_more_rows(B, dtype, n, more, d, vocab):
    c = Case(n, d, vocab, dtype, 41)
    size = B.cross_entropy_scratch_bytes(dtype, more, vocab, d)
    assert size < B.cross_entropy_scratch_bytes(dtype, n, vocab, d)
    scratch = torch.full((size,), 255, dtype=torch.uint8, device="cuda")  # (NaN in any type)
    want = B.cross_entropy_gradients(c.x, c.w, c.t, d_loss=c.d_loss)
    for dw_dtype in (torch.float32, dtype):
        got = B.cross_entropy_gradients(c.x, c.w, c.t, d_loss=c.d_loss, dw_dtype=dw_dtype, scratch=scratch)
        check(c, *got, c.d_loss)
        assert torch.equal(got[0], want[0]) and torch.equal(got[2], want[2].to(dw_dtype))
    for kw in (dict(with_dx=False), dict(with_dw=False)):
        some = B.cross_entropy_gradients(c.x, c.w, c.t, d_loss=c.d_loss, scratch=scratch, **kw)
        assert all(p is None or torch.equal(p, q) for p, q in zip(some, (want[0], got[1], want[2])))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,d,vocab", [(5, 72, 77), (16, 260, 2100), (33, 264, 1003), (129, 64, 300), (300, 520, 1111), (1000, 128, 5003)])
def test_scratch_may_hold_anything(B, dtype, n, d, vocab):
    c = Case(n, d - d % 8, vocab, dtype, 43, lead=5.0)
    c.x[0] *= 200.0
    size = B.cross_entropy_scratch_bytes(dtype, n, vocab, c.x.shape[1])
    first = None
    for fill in (255, 0, 127):
        scratch = torch.full((size,), fill, dtype=torch.uint8, device="cuda")
        got = [*B.cross_entropy_gradients(c.x, c.w, c.t, d_loss=c.d_loss, scratch=scratch)]
        scratch.fill_(fill)
        got.append(B.cross_entropy(c.x, c.w, c.t, scratch=scratch))
        first = first or got
        assert all(torch.equal(p, q) for p, q in zip(first, got)), fill


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_pieces_with_rows_far_below_the_largest_logit(B, dtype):
    """Each piece has some, but the last; nothing behind the scratch is written."""
    c = Case(1100, 128, 2003, dtype, 47)
    c.x[:900:3] *= 300.0
    size = B.cross_entropy_scratch_bytes(dtype, 256, 2003, 128) + 4 * 2003 * 128 + 256
    scratch = torch.full((size + 4096,), 255, dtype=torch.uint8, device="cuda")
    for dw_dtype in {torch.float32, dtype}:
        got = B.cross_entropy_gradients(c.x, c.w, c.t, d_loss=c.d_loss, dw_dtype=dw_dtype, scratch=scratch[:size])
        assert float(got[0].max()) > 60
        check(c, *got, c.d_loss)
    check(c, B.cross_entropy(c.x, c.w, c.t, scratch=scratch[:size]))
    assert bool((scratch[size:] == 255).all())
