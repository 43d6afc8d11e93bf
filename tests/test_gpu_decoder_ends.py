"""The operators at a decoder's ends and between its blocks used together, captured, on several streams, and at sizes beyond 32 bits."""
import math
import os
import subprocess
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2501_17086_b200 import binding
    return binding


def rel(a, b):
    return float((a.double() - b).norm() / b.norm())


@pytest.mark.parametrize("dtype,tol", [(torch.float32, 1e-5), (torch.bfloat16, 2e-2)])
@pytest.mark.parametrize("tied", [False, True])
def test_a_language_model_step(B, dtype, tol, tied):
    """Tokens, their embedding, two decoder blocks, a final norm, the loss; and back to the gradients of all of it, against automatic
    differentiation in 64 bits from the same values.  Tolerances: the contexts' own, for float and bf16."""
    L, d, heads, hidden, seq, batch, vocab = 2, 128, 2, 256, 96, 3, 1003
    n = seq * batch
    g = torch.Generator(device="cuda").manual_seed(4)

    def normal(*shape, std):
        return (torch.randn(*shape, generator=g, device="cuda") * std).to(dtype)

    params = {k: normal(L, d, d, std=d ** -0.5) for k in ("Wq", "Wk", "Wv", "Wo")}
    params |= {"W1": normal(L, hidden, d, std=d ** -0.5), "W2": normal(L, d, hidden, std=hidden ** -0.5)}
    table = normal(vocab, d, std=0.05)
    head = table if tied else normal(vocab, d, std=0.05)
    w_norm = (1.0 + 0.1 * torch.randn(d, generator=g, device="cuda")).to(dtype)
    tokens = torch.randint(0, vocab, (n,), generator=g, device="cuda")
    targets = torch.roll(tokens.view(batch, seq), -1, 1)
    targets[:, -1] = -1  # a sequence's last token predicts nothing
    targets = targets.reshape(-1)
    count = n - batch
    scale = math.sqrt(d)

    ctx = B.Context(B.make_config("preln_transformer", dtype, L, d, n, hidden=hidden, n_heads=heads, head_dim=d // heads, seq=seq, batch=batch))
    x_all = ctx.forward(params, B.embedding(tokens, table, scale=scale))
    last = x_all[-1]
    _, y = B.norm_residual(last, kind="rms", w_pre=w_norm)
    d_loss = torch.full((1,), 1.0 / count, device="cuda").expand(n)
    loss, dy, d_head = B.cross_entropy_gradients(y, head, targets, d_loss=d_loss)
    delta, _, dw_norm, _, _ = B.norm_residual_backward(dy, last, kind="rms", w_pre=w_norm, with_df=False)
    grads = ctx.new_grads()
    g_all = ctx.exact(params, delta, x_all, grads=grads)
    if tied:  # the table's gradient comes to the head's
        d_table = B.embedding_gradient(tokens, g_all[0], vocab, scale=scale, add=d_head, d_table=d_head)
    else:
        d_table = B.embedding_gradient(tokens, g_all[0], vocab, scale=scale)
    ctx.sync_status()

    P = {k: v.double().requires_grad_(True) for k, v in params.items()}
    T, wn = table.double().requires_grad_(True), w_norm.double().requires_grad_(True)
    H = T if tied else head.double().requires_grad_(True)
    x = T[tokens] * scale

    def ln(t):
        return torch.nn.functional.layer_norm(t, (d,), eps=1e-5)

    mask = torch.ones(seq, seq, dtype=torch.bool, device="cuda").triu(1)
    for i in range(L):
        h = ln(x)
        q, k, v = ((h @ P[w][i].T).view(batch, seq, heads, -1).transpose(1, 2) for w in ("Wq", "Wk", "Wv"))
        s = (q @ k.transpose(-1, -2) / math.sqrt(d // heads)).masked_fill(mask, -math.inf)
        x = x + (s.softmax(-1) @ v).transpose(1, 2).reshape(n, d) @ P["Wo"][i].T
        x = x + torch.nn.functional.gelu(ln(x) @ P["W1"][i].T) @ P["W2"][i].T
    out = x / torch.sqrt((x ** 2).mean(1, keepdim=True) + 1e-5) * wn
    there = targets >= 0
    want = torch.nn.functional.cross_entropy(out @ H.T, targets.clamp_min(0), reduction="none") * there
    want.sum().div(count).backward()

    assert rel(loss, want.detach()) < tol
    assert rel(dw_norm, wn.grad) < tol
    assert rel(d_table, T.grad) < tol
    if not tied:
        assert rel(d_head, H.grad) < tol
    for k in P:
        assert rel(grads["d" + k], P[k].grad) < tol, k


def all_calls(B, dtype, n=300, d=256, vocab=1501, seed=0):
    """(tensors that may change, a call of all operators on them)"""
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, std=1.0):
        return (torch.randn(*shape, generator=g, device="cuda") * std).to(dtype)

    t = {"tokens": torch.randint(-1, vocab, (n,), generator=g, device="cuda"), "table": normal(vocab, d, std=0.05), "x": normal(n, d), "f": normal(n, d), "w": normal(d),
         "gate": normal(d), "dy": normal(n, d, std=0.01)}

    def call():
        e = B.embedding(t["tokens"], t["table"], scale=3.0)
        kw = dict(kind="layer", post=True, w_post=t["w"], gate=t["gate"], scale=0.5, w_pre=t["w"])
        new, y = B.norm_residual(t["x"], t["f"], **kw)
        back = B.norm_residual_backward(t["dy"], new, t["f"], t["x"], d_new=e, **kw)
        alone = B.cross_entropy(y, t["table"], t["tokens"])
        loss, dx, dw = B.cross_entropy_gradients(y, t["table"], t["tokens"])
        return [e, new, y, *back, alone, loss, dx, dw, B.embedding_gradient(t["tokens"], dx, vocab, add=dw)]

    return t, call


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_captured_and_replayed(B, dtype):
    t, call = all_calls(B, dtype)
    call()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        call()
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call()
    for seed in (1, 2, 1):
        other, again = all_calls(B, dtype, seed=seed)
        for k in t:
            t[k].copy_(other[k])
        if seed == 2:
            t["x"] *= 300.0  # (losses that are far from their largest logit: a launch more has something to do)
            other["x"] *= 300.0
            t["table"] *= 20.0
            other["table"] *= 20.0
        graph.replay()
        want = again()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want)), seed


FIRST = """
import sys
sys.path[:0] = sys.argv[1:3]
import torch
from paper_2501_17086_b200 import binding as B
from test_gpu_decoder_ends import all_calls
for dtype in (torch.float32, torch.bfloat16):
    t, call = all_calls(B, dtype)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call()
    graph.replay()
    want = call()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out, want)), dtype
"""


def test_a_process_whose_first_calls_are_captured():
    here = os.path.dirname(os.path.abspath(__file__))
    subprocess.run([sys.executable, "-c", FIRST, os.path.dirname(here), here], check=True, timeout=300)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_streams_at_once(B, dtype):
    """Calls on several streams, none waiting for another, and each after work of its own stream that makes its inputs."""
    sets = [all_calls(B, dtype, n=700 + 100 * i, seed=i) for i in range(3)]
    want = [[o.clone() for o in call()] for _, call in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    for turn in range(5):
        got = []
        for (t, call), s in zip(sets, streams):
            with torch.cuda.stream(s):
                keep = t["x"].clone()
                t["x"].zero_()
                torch.cuda._sleep(200000)
                t["x"].copy_(keep)
                got.append(call())
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert all(torch.equal(p, q) for p, q in zip(a, b)), turn


def test_refused_tensors(B):
    t, _ = all_calls(B, torch.float32, n=8, d=64, vocab=50)
    x, table, tok, w = t["x"], t["table"], t["tokens"], t["w"]
    bad = [
        (lambda: B.embedding(tok.float(), table), 2), (lambda: B.embedding(tok[:, None], table), 2), (lambda: B.embedding(tok, table.half()), 3),
        (lambda: B.embedding(tok, table.T), 2), (lambda: B.embedding(tok, table, out=x.bfloat16()), 2), (lambda: B.embedding(tok, table[:, 1:]), 2),
        (lambda: B.embedding(tok.cpu(), table), 1), (lambda: B.embedding(tok, table, status=tok), 2),
        (lambda: B.embedding_gradient(tok, x[:4], 50), 2), (lambda: B.embedding_gradient(tok, x, 50, add=table[:9]), 2), (lambda: B.embedding_gradient(tok, x, -1), 2),
        (lambda: B.embedding_gradient(tok, x, 50, scratch=w), 5), (lambda: B.embedding_gradient(tok, x, 0), 2),
        (lambda: B.norm_residual(x, x[:4]), 2), (lambda: B.norm_residual(x, x.bfloat16()), 2), (lambda: B.norm_residual(x, w_pre=w[:8]), 2),
        (lambda: B.norm_residual(x, w_pre=w.bfloat16()), 2), (lambda: B.norm_residual(x, gate=w), 1), (lambda: B.norm_residual(x, x_new=x), 1),
        (lambda: B.norm_residual(x, with_y=False), 1), (lambda: B.norm_residual(x, x, y=x.T), 2),
        (lambda: B.norm_residual_backward(None, x), 1), (lambda: B.norm_residual_backward(x, None), 1), (lambda: B.norm_residual_backward(x, x, gate=w), 1),
        (lambda: B.norm_residual_backward(x, x, post=True), 1), (lambda: B.norm_residual_backward(x, x, with_dx=False, with_df=False), 1),
        (lambda: B.norm_residual_backward(x, x, w_pre=w, scratch=w), 5),
        (lambda: B.cross_entropy(x, table[:, :32], tok), 2), (lambda: B.cross_entropy(x, table.bfloat16(), tok), 2), (lambda: B.cross_entropy(x, table, tok[:4]), 2),
        (lambda: B.cross_entropy(x[:, ::2], table, tok), 2), (lambda: B.cross_entropy(x[:1].expand(8, 64), table, tok), 2), (lambda: B.cross_entropy(x, table[:0], tok), 2),
        (lambda: B.cross_entropy(x, table, tok, loss=w), 2), (lambda: B.cross_entropy_gradients(x, table, tok, d_loss=w), 2),
        (lambda: B.cross_entropy_gradients(x, table, tok, with_dx=False, with_dw=False), 1), (lambda: B.cross_entropy_gradients(x, table, tok, dw_dtype=torch.bfloat16), 3),
        (lambda: B.cross_entropy_gradients(x, table, tok, dx=table), 2), (lambda: B.cross_entropy(x, table, tok, scratch=w), 5),
    ]
    for i, (call, code) in enumerate(bad):
        with pytest.raises(B.HbpError) as e:
            call()
        assert e.value.code == code, (i, e.value)


def test_tables_beyond_32_bits(B):
    """More than 2^31 elements: the last rows of a table, of its gradient, of a vocabulary matrix and of a stream."""
    d = 8192
    vocab = (1 << 31) // d + 1001
    g = torch.Generator(device="cuda").manual_seed(1)
    table = torch.empty(vocab, d, device="cuda", dtype=torch.bfloat16)
    table.normal_(0.0, 0.01, generator=g)
    tokens = torch.tensor([0, vocab - 1, 5, vocab - 1, vocab - 700, vocab - 2], device="cuda")
    assert torch.equal(B.embedding(tokens, table), table[tokens])
    d_out = torch.randn(6, d, generator=g, device="cuda").bfloat16()
    got = B.embedding_gradient(tokens, d_out, vocab)
    used = torch.unique(tokens)
    assert torch.equal(got[vocab - 1], d_out[1].float() + d_out[3].float()) and torch.equal(got[vocab - 700], d_out[4].float())
    assert int((got.abs().amax(1) > 0).sum()) == len(used)
    del got
    x = torch.randn(40, d, generator=g, device="cuda").bfloat16()
    targets = torch.arange(40, device="cuda") * 97 + vocab - 4000
    loss, dx, dw = B.cross_entropy_gradients(x, table, targets)
    z = x.double() @ table.double().T
    want = torch.logsumexp(z, 1) - z.gather(1, targets[:, None])[:, 0]
    # a logit is off by (d / 16 + 8) 2^-23 of the sum of magnitudes, some 8192 * 0.8 * 0.008: 3.3e-3; the loss by twice that
    assert float((loss.double() - want).abs().max()) < 7e-3
    dz = torch.softmax(z, 1)
    dz[torch.arange(40, device="cuda"), targets] -= 1.0
    # three roundings of 2^-8 (two for dx) and twice a logit's error, of each term: 2e-2 of the sum of magnitudes
    last = dz[:, -4000:]
    assert bool(((dw[-4000:].double() - last.T @ x.double()).abs() <= 2e-2 * (last.abs().T @ x.double().abs())).all())
    exact = dz @ table.double()
    assert bool(((dx.double() - exact).abs() <= 2e-2 * (dz.abs() @ table.double().abs()) + 2.0 ** -8 * exact.abs()).all())
    del dw, z, dz, exact, last
    w = torch.rand(d, generator=g, device="cuda").bfloat16()
    new, y = B.norm_residual(table, table, kind="rms", post=True, w_post=w, w_pre=w)
    small = table[-3:].clone()
    a, b = B.norm_residual(small, small, kind="rms", post=True, w_post=w, w_pre=w)
    assert torch.equal(new[-3:], a) and torch.equal(y[-3:], b)
    dx, df, *_ = B.norm_residual_backward(y, new, table, kind="rms", post=True, w_post=w, w_pre=w, with_weights=False)
    p, q, *_ = B.norm_residual_backward(b, a, small, kind="rms", post=True, w_post=w, w_pre=w, with_weights=False)
    assert torch.equal(dx[-3:], p) and torch.equal(df[-3:], q)
