"""The cases that the operators at a decoder's ends, and between its blocks, are measured by.

  embedding  rows of a table by tokens, scaled (`binding.embedding`), and the table's gradient (`binding.embedding_gradient`)
  norm       a residual update with its gate and scale, the norm of the block's output before it and the norm of the stream after
             it (`binding.norm_residual`), and its gradients (`binding.norm_residual_backward`)
  loss       softmax cross entropy of a large vocabulary from the last hidden states (`binding.cross_entropy`), and with the
             gradients of hidden states and vocabulary matrix (`binding.cross_entropy_gradients`)

`run` computes them in elementary torch operations in 32 bits (the table's gradient, a long sum, in 64), or, where `own` is true, by the
calls named above.
"""
import math

import torch

own = False

ES = {"f32": 4, "bf16": 2}
DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-5


def _embedding(name, dtype, tokens, vocab, d, train, add=False):
    return {"name": name, "op": "embedding", "dtype": dtype, "tokens": tokens, "vocab": vocab, "d": d, "train": train, "add": add}


def _norm(name, dtype, rows, d, kind, post, gate, backward):
    return {"name": name, "op": "norm", "dtype": dtype, "rows": rows, "d": d, "kind": kind, "post": post, "gate": gate, "backward": backward}


def _loss(name, dtype, rows, d, vocab, train):
    return {"name": name, "op": "loss", "dtype": dtype, "rows": rows, "d": d, "vocab": vocab, "train": train}


def listed():
    return [
        # the next token of a handful of sequences: a launch's latency and nothing else
        _embedding("embedding_few", "bf16", 5, 32000, 768, False),
        # the tokens of a training step of the decoder workload (16 sequences of 1024), lookup and gradient
        _embedding("embedding_train", "bf16", 16384, 50021, 768, True),
        # single precision, the gradient added to that of a vocabulary matrix that is the same table
        _embedding("embedding_tied_f32", "f32", 5003, 10007, 1492, True, True),
        # one step between two blocks for a few rows: latency
        _norm("norm_few", "bf16", 16, 512, "rms", False, False, False),
        # between two blocks of the decoder workload: layer norm of the stream alone
        _norm("norm_block", "bf16", 16384, 768, "layer", False, False, False),
        # norms on both sides of a block, a gate on every channel, the widest stack's width: gradients of all
        _norm("norm_both_sides_backward", "bf16", 16384, 2048, "rms", True, True, True),
        # the same in single precision with layer norms, odd sizes
        _norm("norm_odd_backward_f32", "f32", 1237, 1492, "layer", True, True, True),
        # scores of a few rows: the vocabulary matrix is read once
        _loss("loss_few", "bf16", 16, 1024, 32003, False),
        # evaluation: the loss alone
        _loss("loss_eval", "bf16", 4096, 1024, 50021, False),
        # one step's rows of the decoder workload in half, an odd vocabulary
        _loss("loss_train", "bf16", 8192, 768, 50021, True),
        # the largest: a wide model with a large vocabulary
        _loss("loss_train_large", "bf16", 8192, 2048, 131072, True),
        # single precision, odd sizes
        _loss("loss_train_f32", "f32", 1901, 520, 8111, True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["embedding", "norm", "norm", "loss", "loss"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op == "embedding":
        while True:
            c = _embedding("", dtype, _log(rng, 1, 65536), _log(rng, 30, 150000), 8 * _log(rng, 4, 512), rng.random() < 0.7, rng.random() < 0.4)
            if c["vocab"] * c["d"] <= 1 << 28 and c["tokens"] * c["d"] <= 1 << 26:
                return _bare(c)
    if op == "norm":
        while True:
            backward = rng.random() < 0.5
            c = _norm("", dtype, _log(rng, 1, 32768), 8 * _log(rng, 4, 1024), rng.choice(["layer", "rms"]), rng.random() < 0.5, rng.random() < 0.5, backward)
            # (fewer than four rows have gradients of weights that are single products)
            if c["rows"] * c["d"] <= 1 << 25 and not (backward and c["rows"] < 4):
                return _bare(c)
    while True:
        train = rng.random() < 0.6
        c = _loss("", dtype, _log(rng, 1, 16384), 8 * _log(rng, 8, 512), _log(rng, 50, 140000), train)
        limit = 3e10 if dtype == "f32" else 2.1e12
        if c["rows"] * c["d"] * c["vocab"] <= limit and c["rows"] * c["vocab"] <= 1 << 30 and c["vocab"] * c["d"] <= 1 << 28:
            return _bare(c)


def _bare(c):
    return {k: v for k, v in c.items() if k != "name"}


# ------------------------------------------------------------------------------------------------- inputs
def _tokens(g, n, vocab):
    """As in text: a few tokens are a large part of it, most are rare."""
    u = torch.rand(n, generator=g, device="cuda", dtype=torch.float64)
    t = ((vocab + 1.0) ** u - 1.0).long().clamp(0, vocab - 1)  # density 1 / (rank + 1)
    # tokenizers do not number by frequency alone
    return (t * 7919 + 13) % vocab if math.gcd(7919, vocab) == 1 else t


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = DTYPE[case["dtype"]]

    def normal(*shape, std=1.0, mean=0.0):
        return (torch.randn(*shape, generator=g, device="cuda") * std + mean).to(dt)

    s = {"case": case}
    if case["op"] == "embedding":
        n, v, d = case["tokens"], case["vocab"], case["d"]
        s["tokens"] = _tokens(g, n, v)
        s["table"] = normal(v, d, std=0.02)
        s["scale"] = math.sqrt(d)
        if case["train"]:
            s["d_out"] = normal(n, d, std=2.0 ** -8)
            if case["add"]:
                s["first"] = torch.randn(v, d, generator=g, device="cuda") * 2.0 ** -8
    elif case["op"] == "norm":
        n, d = case["rows"], case["d"]
        # a stream: a few channels are much larger than the rest
        spread = torch.where(torch.rand(d, generator=g, device="cuda") < 0.02, 12.0, 1.0)
        s["x"] = (torch.randn(n, d, generator=g, device="cuda") * spread).to(dt)
        s["f"] = normal(n, d, std=0.3)
        s["w_pre"] = normal(d, std=0.2, mean=1.0)
        s["w_post"] = normal(d, std=0.2, mean=1.0) if case["post"] else None
        s["gate"] = normal(d, std=0.02, mean=0.9) if case["gate"] else None
        s["scale"] = 0.5
        if case["backward"]:  # what the forward pass has left, and the two gradients that arrive
            s["x_new"] = _new_stream(s, lambda t: t.float()).to(dt)
            s["d_new"], s["d_y"] = normal(n, d, std=2.0 ** -8), normal(n, d, std=2.0 ** -8)
    else:
        n, d, v = case["rows"], case["d"], case["vocab"]
        s["w"] = normal(v, d, std=0.02)
        t = _tokens(g, n, v)
        # hidden states of a trained model: some of them already point at their target
        lead = torch.rand(n, 1, generator=g, device="cuda") * 12.0
        wt = s["w"][t].float()
        s["x"] = (torch.randn(n, d, generator=g, device="cuda") + lead * wt / wt.norm(dim=1, keepdim=True).clamp_min(1e-6)).to(dt)
        # a tenth of the rows is padding or prompt
        s["targets"] = torch.where(torch.rand(n, generator=g, device="cuda") < 0.1, -1, t)
        s["targets"][0] = t[0]
        if case["train"]:
            s["d_loss"] = torch.full((n,), 1.0 / n, device="cuda")
    return s


# ------------------------------------------------------------------------------------------------- one pass
def run(state):
    if own:
        return _calls(state)
    return {"embedding": _plain_embedding, "norm": _plain_norm, "loss": _plain_loss}[state["case"]["op"]](state)


def _calls(s):
    from paper_2501_17086_b200 import binding
    c = s["case"]
    if c["op"] == "embedding":
        out = {"out": binding.embedding(s["tokens"], s["table"], scale=s["scale"])}
        if c["train"]:
            out["d_table"] = binding.embedding_gradient(s["tokens"], s["d_out"], c["vocab"], scale=s["scale"], add=s.get("first"))
        return out
    if c["op"] == "norm":
        kw = dict(kind=c["kind"], eps=EPS, post=c["post"], w_post=s["w_post"], gate=s["gate"], scale=s["scale"], w_pre=s["w_pre"])
        if c["backward"]:
            names = ("dx", "df", "dw_pre", "dw_post", "da")
            got = binding.norm_residual_backward(s["d_y"], s["x_new"], s["f"], s["x"], d_new=s["d_new"], **kw)
            return {k: t for k, t in zip(names, got) if t is not None}
        x_new, y = binding.norm_residual(s["x"], s["f"], **kw)
        return {"x_new": x_new, "y": y}
    if not c["train"]:
        return {"loss": binding.cross_entropy(s["x"], s["w"], s["targets"])}
    loss, dx, dw = binding.cross_entropy_gradients(s["x"], s["w"], s["targets"], d_loss=s["d_loss"], dw_dtype=s["w"].dtype)
    return {"loss": loss, "dx": dx, "dw": dw}


# ------------------------------------------------------------------------------------------------- the plain forms
def _plain_embedding(s):
    c = s["case"]
    out = {"out": (s["table"][s["tokens"]].float() * s["scale"]).to(s["table"].dtype)}
    if c["train"]:
        g = torch.zeros(c["vocab"], c["d"], dtype=torch.float64, device="cuda").index_add_(0, s["tokens"], s["d_out"].double()) * s["scale"]
        out["d_table"] = (g + s["first"]).float() if c["add"] else g.float()
    return out


def _normed(x, kind):
    """x normalised over its rows, and what it was divided by."""
    if kind == "layer":
        x = x - x.mean(-1, keepdim=True)
    r = (x.square().mean(-1, keepdim=True) + EPS).rsqrt()
    return x * r, r


def _norm_back(g, xhat, r, kind):
    """The gradient of a row from that of its normalised values."""
    out = g - xhat * (g * xhat).mean(-1, keepdim=True)
    if kind == "layer":
        out = out - g.mean(-1, keepdim=True)
    return out * r


def _new_stream(s, wide):
    h = wide(s["f"])
    if s["case"]["post"]:
        h = _normed(h, s["case"]["kind"])[0] * wide(s["w_post"])
    x = wide(s["x"])
    return (x if s["gate"] is None else wide(s["gate"]) * x) + s["scale"] * h


def _plain_norm(s):
    c, dt = s["case"], s["x"].dtype
    if not c["backward"]:
        x_new = _new_stream(s, lambda t: t.float()).to(dt)
        return {"x_new": x_new, "y": (_normed(x_new.float(), c["kind"])[0] * s["w_pre"].float()).to(dt)}
    d_y = s["d_y"].float()
    xhat, r = _normed(s["x_new"].float(), c["kind"])
    t = s["d_new"].float() + _norm_back(d_y * s["w_pre"].float(), xhat, r, c["kind"])
    out = {"dw_pre": (d_y * xhat).sum(0)}
    out["dx"] = (t if s["gate"] is None else t * s["gate"].float()).to(dt)
    if s["gate"] is not None:
        out["da"] = (t * s["x"].float()).sum(0)
    u = t * s["scale"]
    if c["post"]:
        fhat, r = _normed(s["f"].float(), c["kind"])
        out["dw_post"] = (u * fhat).sum(0)
        u = _norm_back(u * s["w_post"].float(), fhat, r, c["kind"])
    out["df"] = u.to(dt)
    return out


def _plain_loss(s):
    c, dt = s["case"], s["x"].dtype
    x, w, t = s["x"].float(), s["w"].float(), s["targets"]
    there = t >= 0
    at = t.clamp_min(0)[:, None]
    z = x @ w.T
    z -= z.amax(1, keepdim=True)
    zt = z.gather(1, at)
    z.exp_()
    total = z.sum(1, keepdim=True)
    loss = torch.where(there, (total.log() - zt)[:, 0], 0.0)
    if not c["train"]:
        return {"loss": loss}
    z *= (torch.where(there, s["d_loss"], 0.0)[:, None] / total)
    z.scatter_add_(1, at, -torch.where(there, s["d_loss"], 0.0)[:, None])
    return {"loss": loss, "dx": (z @ w).to(dt), "dw": (z.T @ x).to(dt)}


# ------------------------------------------------------------------------------------------------- the definitions in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "embedding":
        v, scale = case["vocab"], s["scale"]
        out = {"out": s["table"].double().index_select(0, s["tokens"]) * scale}
        if case["train"]:
            order = torch.argsort(s["tokens"], stable=True)
            ends = torch.bincount(s["tokens"], minlength=v).cumsum(0)
            upto = torch.cat([torch.zeros(1, case["d"], dtype=torch.float64, device="cuda"), s["d_out"].double()[order].cumsum(0)])
            starts = torch.cat([ends.new_zeros(1), ends[:-1]])
            out["d_table"] = scale * (upto[ends] - upto[starts])
            if case["add"]:
                out["d_table"] += s["first"].double()
        return out
    if case["op"] == "norm":
        return _exact_norm(case, s)
    return _exact_loss(case, s)


def _exact_norm(case, s):
    layer = case["kind"] == "layer"

    def norm(t):
        m = t.mean(1, keepdim=True) if layer else 0.0
        return (t - m) / torch.sqrt(((t - m) ** 2).mean(1, keepdim=True) + EPS)

    def leaf(name):
        return None if s[name] is None else s[name].double().requires_grad_(True)

    x, f, w_pre, w_post, gate = (leaf(k) for k in ("x", "f", "w_pre", "w_post", "gate"))
    with torch.enable_grad():
        h = norm(f) * w_post if case["post"] else f
        new = (x if gate is None else gate * x) + s["scale"] * h
        if not case["backward"]:  # the stream is stored in its type, and the norm after it reads that
            stored = new.detach().to(s["x"].dtype).double()
            return {"x_new": new.detach(), "y": (norm(stored) * w_pre).detach()}
        stored = s["x_new"].double().requires_grad_(True)
        (norm(stored) * w_pre).backward(s["d_y"].double())
        new.backward(s["d_new"].double() + stored.grad)
    out = {"dx": x.grad, "df": f.grad, "dw_pre": w_pre.grad}
    if gate is not None:
        out["da"] = gate.grad
    if w_post is not None:
        out["dw_post"] = w_post.grad
    return out


def _exact_loss(case, s):
    n, v, d = case["rows"], case["vocab"], case["d"]
    x, w = s["x"].double(), s["w"].double()
    loss = torch.zeros(n, dtype=torch.float64, device="cuda")
    dx, dw = (torch.zeros_like(x), torch.zeros_like(w)) if case["train"] else (None, None)
    step = max(1, (1 << 27) // v)
    for lo in range(0, n, step):
        rows = torch.arange(lo, min(n, lo + step), device="cuda")
        rows = rows[s["targets"][rows] >= 0]
        if not len(rows):
            continue
        t = s["targets"][rows]
        lp = torch.log_softmax(x[rows] @ w.T, 1)
        loss[rows] = -lp[torch.arange(len(rows), device="cuda"), t]
        if case["train"]:
            dz = lp.exp_()
            dz[torch.arange(len(rows), device="cuda"), t] -= 1.0
            dz *= s["d_loss"][rows].double()[:, None]
            dx[rows] = dz @ w
            dw += dz.T @ x[rows]
    return {"loss": loss, "dx": dx, "dw": dw} if case["train"] else {"loss": loss}


# ------------------------------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    es = ES[case["dtype"]]
    if case["op"] == "embedding":
        n, v, d = case["tokens"], case["vocab"], case["d"]
        looked = 8 * n + (n + min(n, v)) * d * es
        if not case["train"]:
            return {"bytes": looked, "flops": n * d}
        return {"bytes": looked + n * d * es + v * d * (8 if case["add"] else 4), "flops": 3 * n * d}
    n, d = case["rows"], case["d"]
    if case["op"] == "norm":
        if not case["backward"]:
            return {"bytes": 4 * n * d * es, "flops": n * d * (20 if case["post"] else 12)}
        read = 3 + case["gate"] + case["post"]  # both gradients and the stream; its old values for the gate's, the block's output for its norm's
        return {"bytes": (read + 2) * n * d * es, "flops": n * d * (40 if case["post"] else 24)}
    v = case["vocab"]
    if not case["train"]:
        return {"bytes": (n + v) * d * es + 12 * n, "flops": 2 * n * v * d + 4 * n * v}
    return {"bytes": 2 * (n + v) * d * es + 16 * n, "flops": 6 * n * v * d + 8 * n * v}
