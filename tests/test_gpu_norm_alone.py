"""The norm of a stream alone (a final norm), and its gradients, in both types and at the widths where the kernels' variants change.  Bounds as in
test_gpu_norm_residual.py."""
import pytest
import torch

from test_gpu_norm_residual import E, Inputs, check_backward, check_forward, near, norm

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2501_17086_b200 import binding
    return binding


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("n,d", [(1, 8), (17, 256), (9, 264), (301, 768), (1237, 1496), (65, 2056), (5, 8192), (4001, 128)])
def test_a_final_norm(B, dtype, kind, n, d):
    s = Inputs(n, d, dtype, False, False, True, n + d, 8)
    x, y = B.norm_residual(s.x, kind=kind, w_pre=s.w_pre)
    assert x is s.x
    w = s.w_pre.double()
    xhat, _, err = norm(s.x.double(), kind, 1e-5)
    near(y, xhat * w, err * w.abs() + 2 * E * (xhat * w).abs(), dtype)
    got = B.norm_residual_backward(s.d_y, s.x, kind=kind, w_pre=s.w_pre, with_df=False)
    assert got[1] is None and got[3] is None and got[4] is None
    check_backward(s, s.x, got, kind, 1.0, 1e-5, with_new=False)
    # in place, and without the weights' gradient
    d_y = s.d_y.clone()
    B.norm_residual_backward(d_y, s.x, kind=kind, w_pre=s.w_pre, with_df=False, with_weights=False, dx=d_y)
    assert torch.equal(d_y, got[0])
    # a gradient of the stream itself arrives too
    got = B.norm_residual_backward(s.d_y, s.x, d_new=s.d_new, kind=kind, w_pre=s.w_pre, with_df=False)
    check_backward(s, s.x, got, kind, 1.0, 1e-5)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("n,d", [(3, 72), (301, 768), (33, 4096)])
def test_an_update_alone(B, dtype, kind, n, d):
    s = Inputs(n, d, dtype, True, True, True, n + d, 8)
    kw = s.kw(kind=kind, scale=0.5)
    x_new, y = B.norm_residual(s.x, s.f, with_y=False, **kw)
    assert y is None
    check_forward(s, x_new, None, kind, 0.5, 1e-5)
    got = B.norm_residual_backward(None, None, s.f, s.x, d_new=s.d_new, **kw)
    assert got[2] is None
    check_backward(s, x_new, got, kind, 0.5, 1e-5, with_y=False)
