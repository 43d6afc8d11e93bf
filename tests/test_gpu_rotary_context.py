"""A decoder context with rotary positions: states, Highway-BP and exact gradients and parameter gradients against the fp64 oracle whose
attention steps turn queries and keys; and what the context answers around the switch."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2501_17086_b200 import binding
    return binding


def turn_of(seq, dh, r, first, layout, amplitude, base):
    f = base ** (-2.0 * np.arange(r // 2) / r)
    a = (first + np.arange(seq))[:, None] * f
    cos, sin = amplitude * np.cos(a), amplitude * np.sin(a)

    def turn(t, back):
        s = -sin if back else sin
        y = t.copy()
        if layout == "half":
            i, j = slice(0, r // 2), slice(r // 2, r)
        else:
            i, j = slice(0, r, 2), slice(1, r, 2)
        y[..., i], y[..., j] = t[..., i] * cos - t[..., j] * s, t[..., j] * cos + t[..., i] * s
        return y

    return turn


def rel(a, b):
    a = a.detach().float().cpu().double().numpy().reshape(b.shape)
    n = np.linalg.norm(b)
    return float(np.linalg.norm(a - b) / n) if n else float(np.linalg.norm(a))


@pytest.mark.parametrize("name,tol", [("c4_twin_f32", 1e-5), ("c4_twin", 2e-2)])
@pytest.mark.parametrize("layout,part,first,amplitude", [("half", 1.0, 0, 1.0), ("interleaved", 0.5, 1000, 1.1)])
def test_a_decoder_with_rotary_positions(B, name, tol, layout, part, first, amplitude):
    from oracle import hbp_oracle as O
    from oracle import run as orun
    from paper_2501_17086_b200 import harness
    from paper_2501_17086_b200.workloads import WORKLOADS, make_inputs
    w = WORKLOADS[name]
    inp = make_inputs(w, "cuda")
    if w.dtype == "f32":
        # scores of order one: with the workload's own weights they are nearly equal, and positions change less than bf16 rounds
        inp["Wq"], inp["Wk"] = inp["Wq"] * 16, inp["Wk"] * 16
    ctx, params = harness.make_context(w), harness.params_for(w, inp)
    r = int(part * w.head_dim)
    plain = ctx.forward(params, inp["x0"]).clone()
    ctx.set_rotary(B.rotary_spec(r, base=500.0, layout=layout, amplitude=amplitude), first)
    x_all = ctx.forward(params, inp["x0"])
    delta = harness.loss_delta(w, x_all, inp)
    grads = ctx.new_grads()
    k = 2
    g = ctx.backward(params, k, delta, x_all, grads=grads).clone()
    exact = ctx.exact(params, delta, x_all)
    ctx.sync_status()
    stack, x0, groups = orun.build_stack(w, inp)
    for step in stack.steps[0::2]:
        step.turn = turn_of(w.seq, w.head_dim, r, first, layout, amplitude, 500.0)
    xs, caches = O.forward(stack, x0)
    deltas = orun.loss_deltas(w, xs, inp)
    want, want_exact = O.highway_bp(stack, caches, deltas, k), O.exact_bp(stack, caches, deltas)
    want_grads = O.param_grads(stack, caches, xs, want, groups)
    for l in range(w.steps + 1):
        assert rel(x_all[l], xs[l]) <= tol and rel(g[l], want[l]) <= tol and rel(exact[l], want_exact[l]) <= tol, l
    for n, v in want_grads.items():
        assert rel(grads["d" + n], v) <= tol, n
    if w.dtype == "f32":
        assert rel(plain[-1], xs[-1]) > 100 * tol  # the positions do something
    ctx.set_rotary(None)
    assert torch.equal(ctx.forward(params, inp["x0"]), plain)  # and go again
    ctx.close()


def test_switching_positions_asks_for_a_forward_pass_and_other_kinds_refuse(B):
    cfg = B.make_config("preln_transformer", "f32", 1, 64, 32, hidden=64, n_heads=2, head_dim=32, seq=16, batch=2)
    ctx = B.Context(cfg)
    p = {n: torch.zeros(1, 64, 64, device="cuda") for n in ("Wq", "Wk", "Wv", "Wo", "W1", "W2")}
    x = ctx.forward(p, torch.zeros(32, 64, device="cuda"))
    delta = torch.zeros(32, 64, device="cuda")
    ctx.backward(p, 1, delta, x)
    ctx.set_rotary(B.rotary_spec(32))
    with pytest.raises(B.HbpError) as e:
        ctx.backward(p, 1, delta, x)
    assert e.value.code == 4
    for bad, code in ((B.rotary_spec(34), 2), (B.rotary_spec(31), 2), (B.rotary_spec(32, base=0.5), 1)):
        with pytest.raises(B.HbpError) as e:
            ctx.set_rotary(bad)
        assert e.value.code == code
    mlp = B.Context(B.make_config("mlp", "f32", 2, 64, 32, hidden=64))
    with pytest.raises(B.HbpError) as e:
        mlp.set_rotary(B.rotary_spec(32))
    assert e.value.code == 6
    assert B.lib.hbp_context_rotary(None, None, 0) == 1
    assert math.isfinite(float(x.sum()))
