"""Cross entropy of bf16 rows of more than 32 MB, whose tiles go down several panels of row blocks, the last of them shorter.  Bounds as in
test_gpu_cross_entropy.py."""
import pytest
import torch

from test_gpu_cross_entropy import Case, check

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2501_17086_b200 import binding
    return binding


# CTA pairs: 16 row blocks of 256 a panel, 18 in all; 33 of 35; single CTAs (up to 128 tokens): 64 of 128, 71 in all
@pytest.mark.parametrize("n,d,vocab", [(4500, 4096, 300), (8791, 2000, 1030), (9000, 2048, 100)])
def test_several_panels(B, n, d, vocab):
    c = Case(n, d, vocab, torch.bfloat16, 51)
    assert n * d * 2 > 32 << 20
    # every seventh row and all of the last 300 lean on another token than their target, by some 45 to 60: a loss above 40, and so a second run
    g = torch.Generator(device="cuda").manual_seed(52)
    other = (c.t.long().clamp_min(0) + 1 + torch.randint(0, vocab - 1, (n,), generator=g, device="cuda")) % vocab
    at = torch.arange(n, device="cuda")
    lean = ((at % 7 == 0) | (at >= n - 300))[:, None]
    w = c.w[other].float()
    c.x.copy_(torch.where(lean, c.x.float() + 52.0 * w / w.square().sum(1, keepdim=True), c.x.float()))
    alone = B.cross_entropy(c.x, c.w, c.t)
    assert bool((alone[-300:][c.t[-300:] >= 0] > 40).all()) and bool((alone[(c.t >= 0) & ~lean[:, 0]] < 40).all())
    check(c, alone)
    loss, dx, dw = B.cross_entropy_gradients(c.x, c.w, c.t, d_loss=c.d_loss)
    check(c, loss, dx, dw, c.d_loss)
