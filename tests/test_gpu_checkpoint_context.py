"""Contexts that keep their activations in 8 bits, against the fp64 oracle whose cached pre-activations are replaced by the values that are
kept of them.

Bars.  bf16: the repository's 2e-2.  Float: Z of the two sides differs by some 1e-6 of a row's scale, so that one element in 4000 (127 * 1e-6 on either
side of a tie, twice) may get the next code; its gelu' is then off by at most 0.8 / 63.5 of the group's largest value, some 0.04 of the
element: sqrt(2.5e-4) * 0.04 = 6e-4 in the norm; 1e-3."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2501_17086_b200 import binding
    return binding


def kept(z, bf16):
    """What 8 bits keep of z [..., h]: steps of the smallest power of two of which 127 reach the largest of 32 neighbours."""
    z = np.asarray(z, dtype=np.float64)
    if bf16:
        z = torch.from_numpy(z).to(torch.bfloat16).double().numpy()
    h = z.shape[-1]
    g = np.pad(z.reshape(-1, h), ((0, 0), (0, -h % 32))).reshape(-1, (h + 31) // 32, 32)
    m, e = np.frexp(np.abs(g).max(-1, keepdims=True))
    e = np.maximum(np.where(m > 127 / 128, e - 6, e - 7), -126)
    return (np.rint(np.ldexp(g, -e)) * np.ldexp(1.0, e)).reshape(z.reshape(-1, h).shape[0], -1)[:, :h].reshape(z.shape)


def rel(a, b):
    a = a.detach().float().cpu().double().numpy().reshape(b.shape)
    n = np.linalg.norm(b)
    return float(np.linalg.norm(a - b) / n) if n else float(np.linalg.norm(a))


KINDS = ["c1", "c2_twin", "c2_twin_f32", "c4_twin", "c4_twin_f32", "relu_twin", "postln_twin_shift", "postln_twin_shift_bf16"]


@pytest.mark.parametrize("name", KINDS)
@pytest.mark.parametrize("group", [0, 2])
def test_a_stack_with_activations_in_8_bits(B, monkeypatch, name, group):
    from oracle import hbp_oracle as O
    from oracle import run as orun
    from paper_2501_17086_b200 import harness
    from paper_2501_17086_b200.workloads import WORKLOADS, make_inputs
    if group:
        monkeypatch.setenv("HBP_LAYER_GROUP", str(group))
    w = WORKLOADS[name]
    inp = make_inputs(w, "cuda")
    cfg = B.config_from_workload(w)
    bf16, tol = w.dtype == "bf16", 2e-2 if w.dtype == "bf16" else 1e-3
    ctx, params = B.Context(cfg, checkpointed=True), harness.params_for(w, inp)
    assert ctx.modes & 8
    x_all = ctx.forward(params, inp["x0"])
    delta = harness.loss_delta(w, x_all, inp)
    grads, exact_grads, k = ctx.new_grads(), ctx.new_grads(), 2
    g = ctx.backward(params, k, delta, x_all, grads=grads).clone()
    exact = ctx.exact(params, delta, x_all, grads=exact_grads)
    ctx.sync_status()
    stack, x0, groups = orun.build_stack(w, inp)
    xs, caches = O.forward(stack, x0)
    deltas = orun.loss_deltas(w, xs, inp)
    for l in range(w.steps + 1):
        assert rel(x_all[l], xs[l]) <= (2e-2 if bf16 else 1e-5), l  # the forward pass is that of Z itself
    full = O.param_grads(stack, caches, xs, O.highway_bp(stack, caches, deltas, k), groups)
    for c in caches:
        if "z" in c:
            c["z"] = kept(c["z"], bf16)
    want, want_exact = O.highway_bp(stack, caches, deltas, k), O.exact_bp(stack, caches, deltas)
    for l in range(w.steps + 1):
        assert rel(g[l], want[l]) <= tol and rel(exact[l], want_exact[l]) <= tol, l
    for got, at in ((grads, want), (exact_grads, want_exact)):
        for n, v in O.param_grads(stack, caches, xs, at, groups).items():
            assert rel(got["d" + n], v) <= tol, n
            if not bf16 and at is want and n == "W1":  # the kept values make a difference that the bar would show, and a small one
                assert tol < rel(torch.from_numpy(v), full[n]) < 0.1
    ctx.close()


def test_workspaces_and_refusals(B):
    cfg = B.make_config("preln_mlp", "bf16", 8, 256, 4096, hidden=1024)
    full, small = B.workspace_bytes(cfg), B.workspace_bytes(cfg, checkpointed=True)
    n = 8 * 4096 * 1024  # two caches of 2 bytes a value against 1 + 1/32
    assert full - small == 4 * n - n - n // 32
    with pytest.raises(B.HbpError) as e:
        B.workspace_bytes(B.make_config("gru", "f32", 6, 64, 4, in_dim=8, batch=4), checkpointed=True)
    assert e.value.code == 6


def test_the_activation_alone(B):
    """gelu of the kept values without a gradient: what the backward pass gives beside one."""
    z = torch.randn(50, 104, device="cuda")
    _, codes, scales = B.checkpoint_gelu(z)
    _, act = B.checkpoint_gelu_backward(torch.ones_like(z), codes, scales, with_act=True)
    out = torch.empty(50, 104, device="cuda")
    stream = torch.cuda.current_stream().cuda_stream
    assert B.lib.hbp_checkpoint_gelu_backward(0, 50, 104, codes.data_ptr(), scales.data_ptr(), None, 0, None, 0, out.data_ptr(), 104, stream) == 0
    assert torch.equal(out, act)
    assert B.lib.hbp_checkpoint_gelu_backward(0, 50, 104, codes.data_ptr(), scales.data_ptr(), None, 0, None, 0, None, 0, stream) == 1
    assert B.lib.hbp_checkpoint_gelu_backward(0, 50, 104, codes.data_ptr(), scales.data_ptr(), None, 0, None, 0, out.data_ptr(), 100, stream) == 2
