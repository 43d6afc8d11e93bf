"""Rows of a table by tokens, and the table's gradient.  The lookup is one product in float and one rounding: equal to torch's.  The gradient's
sums of n rows are float, in any order off by at most n 2^-24 of the sum of magnitudes; the scale, the sum with `add` and their joint rounding
add three more."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2501_17086_b200 import binding
    return binding


def tokens_of(kind, n, vocab, seed, dtype=torch.int64):
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = torch.randint(0, vocab, (n,), generator=g, device="cuda")
    if kind == "one":
        t = torch.full_like(t, vocab - 1)
    elif kind == "half":  # every second one the same
        t[::2] = vocab // 3
    elif kind == "none":
        t[torch.rand(n, generator=g, device="cuda") < 0.3] = -1
    elif kind == "runs":
        t = torch.arange(n, device="cuda") // 37 % vocab
    return t.to(dtype)


def rows_of(n, d, dtype, seed, stride=None):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(n, stride or d, generator=g, device="cuda").to(dtype)
    return x[:, :d]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,vocab,d,stride", [(1, 1, 8, None), (1, 50000, 768, None), (7, 3, 64, 72), (129, 1000, 1496, 1600), (4099, 131072, 24, None),
                                              (513, 77, 8192, None)])
def test_lookup(B, dtype, n, vocab, d, stride):
    table = rows_of(vocab, d, dtype, 1, stride)
    for token_type in (torch.int32, torch.int64):
        t = tokens_of("none", n, vocab, 2, token_type)
        want = torch.where((t >= 0)[:, None], (table.float() * 2.75)[t.clamp_min(0).long()], 0.0).to(dtype)
        out = torch.full((n, d + 16), 7.0, device="cuda", dtype=dtype)
        got = B.embedding(t, table, scale=2.75, out=out[:, :d])
        assert torch.equal(got, want) and bool((out[:, d:] == 7.0).all())
        assert torch.equal(B.embedding(t, table, scale=2.75), want)


def check_gradient(got, t, d_out, vocab, scale, add):
    d = d_out.shape[1]
    there = (t >= 0) & (t < vocab)
    at, g = t[there].long(), d_out[there].double()
    want = torch.zeros(vocab, d, dtype=torch.float64, device="cuda").index_add_(0, at, g) * scale
    size = torch.zeros(vocab, d, dtype=torch.float64, device="cuda").index_add_(0, at, g.abs()) * abs(scale)
    count = torch.bincount(at, minlength=vocab).double()[:, None]
    base = torch.zeros_like(want) if add is None else add.double()
    off = (got.double() - want - base).abs()
    bound = ((count + 3) * size + 2 * base.abs() * (count > 0)) * 2.0 ** -24
    assert float((off - bound).max()) <= 0


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("kind", ["any", "one", "half", "none", "runs"])
@pytest.mark.parametrize("n,vocab,d", [(1, 1, 8), (1, 70000, 64), (31, 40, 136), (32, 33, 64), (33, 512, 64), (1000, 511, 128), (5000, 65535, 40), (8193, 13, 1032),
                                       (70001, 131072, 16)])
def test_gradient(B, dtype, kind, n, vocab, d):
    t = tokens_of(kind, n, vocab, n + vocab, torch.int32 if n % 2 else torch.int64)
    g = rows_of(n, d, dtype, 3, d + 8)
    first = B.embedding_gradient(t, g, vocab, scale=0.75)
    check_gradient(first, t, g, vocab, 0.75, None)
    assert torch.equal(first, B.embedding_gradient(t, g, vocab, scale=0.75))  # the same bits
    add = rows_of(vocab, d, torch.float32, 4)
    got = B.embedding_gradient(t, g, vocab, scale=0.75, add=add)
    check_gradient(got, t, g, vocab, 0.75, add)
    place = add.clone()
    assert B.embedding_gradient(t, g, vocab, scale=0.75, add=place, d_table=place) is not None
    assert torch.equal(place, got)


def test_gradient_of_no_rows_and_of_one_row_for_all(B):
    none = torch.empty(0, dtype=torch.int64, device="cuda")
    g = torch.empty(0, 64, device="cuda")
    assert torch.equal(B.embedding_gradient(none, g, 11), torch.zeros(11, 64, device="cuda"))
    add = rows_of(11, 64, torch.float32, 1)
    assert torch.equal(B.embedding_gradient(none, g, 11, add=add), add)
    assert B.embedding(none, add).shape == (0, 64)
    t = tokens_of("any", 301, 17, 5)
    row = rows_of(1, 64, torch.bfloat16, 6).expand(301, 64)
    check_gradient(B.embedding_gradient(t, row, 17), t, row, 17, 1.0, None)
    assert torch.equal(B.embedding(t, add[:1].expand(17, 64)), add[:1].expand(301, 64))


def test_tokens_beyond_the_table_are_none_and_reported(B):
    t = torch.tensor([3, 17, -1, 2 ** 40, 0], device="cuda")
    table, status = rows_of(17, 64, torch.float32, 1), torch.zeros(1, dtype=torch.int32, device="cuda")
    out = B.embedding(t, table, status=status)
    assert status.item() == 1 and torch.equal(out[[0, 4]], table[[3, 0]]) and not out[[1, 2, 3]].any()
    status.zero_()
    g = rows_of(5, 64, torch.float32, 2)
    g[1:4] = float("nan")  # what rows without a token hold changes nothing
    got = B.embedding_gradient(t, g, 17, status=status)
    assert status.item() == 1 and torch.equal(got[3], g[0]) and torch.equal(got[0], g[4]) and int(got.any(1).sum()) == 2
    status.zero_()
    B.embedding(t[2:3], table, status=status)
    B.embedding_gradient(t[2:3], g[:1], 17, status=status)
    assert status.item() == 0


def test_values_that_are_not_finite_stay_in_their_row(B):
    t = tokens_of("any", 999, 50, 1)
    g = rows_of(999, 64, torch.bfloat16, 2).clone()
    g[500, 3] = float("inf")
    got = B.embedding_gradient(t, g, 50)
    bad = torch.zeros(50, 64, dtype=torch.bool, device="cuda")
    bad[t[500], 3] = True
    assert torch.equal(~got.isfinite(), bad)
