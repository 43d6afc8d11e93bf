"""The table's gradient with scratch made for a few tokens more, where tiles double and need less, whatever it held."""
import ctypes as C

import pytest
import torch

from test_gpu_embedding import check_gradient, rows_of, tokens_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [65536, 65537, 131072])
@pytest.mark.parametrize("kind", ["any", "half"])
def test_scratch_of_more_tokens(n, kind):
    from paper_2501_17086_b200 import binding as B
    d, vocab = 32, 1009
    need = C.c_size_t()
    assert B.lib.hbp_embedding_gradient_scratch_bytes(n + 1, d, C.byref(need)) == 0
    t, g = tokens_of(kind, n, vocab, 5), rows_of(n, d, torch.bfloat16, 6)
    want = B.embedding_gradient(t, g, vocab, scale=0.5)
    check_gradient(want, t, g, vocab, 0.5, None)
    for fill in (255, 0):
        scratch = torch.full((need.value + 4096,), fill, dtype=torch.uint8, device="cuda")
        got = B.embedding_gradient(t, g, vocab, scale=0.5, scratch=scratch[: need.value])
        assert torch.equal(got, want) and bool((scratch[need.value :] == fill).all())
