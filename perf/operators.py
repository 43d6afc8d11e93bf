"""The cases that the stand-alone operators of a decoder's training step are measured by.

  rotary      rotary positions on the queries and keys of a block (`binding.rotary`), and its gradient
  attention   attention over ragged batches with grouped heads (`binding.attention_forward`) and its backward pass,
              which recomputes the probabilities (`binding.attention_backward`)
  checkpoint  an activation kept in 8 bits and read back (`binding.checkpoint_store`, `binding.checkpoint_load`)
  gelu        GELU whose input is kept in 8 bits, and its backward pass from those (`binding.checkpoint_gelu`,
              `binding.checkpoint_gelu_backward`)

`run` computes them in elementary torch operations in 32 bits (angles in 64), or, where `own` is true, by the calls
named above.
"""
import math

import torch

own = False

ES = {"f32": 4, "bf16": 2}
DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
GROUP = 32  # channels that share one scale of an 8-bit checkpoint


def _rotary(name, dtype, tokens, q_heads, kv_heads, head_dim, rotary_dim, layout, scaling="none", factor=1.0, far=2048, inverse=False):
    return {"name": name, "op": "rotary", "dtype": dtype, "tokens": tokens, "q_heads": q_heads, "kv_heads": kv_heads,
            "head_dim": head_dim, "rotary_dim": rotary_dim, "layout": layout, "scaling": scaling, "factor": factor,
            "far": far, "inverse": inverse}


def _attention(name, dtype, sequences, q_len, kv_len, q_heads, kv_heads, head_dim, causal, ragged, train):
    return {"name": name, "op": "attention", "dtype": dtype, "sequences": sequences, "q_len": q_len, "kv_len": kv_len,
            "q_heads": q_heads, "kv_heads": kv_heads, "head_dim": head_dim, "causal": causal, "ragged": ragged, "train": train}


def _checkpoint(name, dtype, rows, channels):
    return {"name": name, "op": "checkpoint", "dtype": dtype, "rows": rows, "channels": channels}


def _gelu(name, dtype, rows, channels):
    return {"name": name, "op": "gelu", "dtype": dtype, "rows": rows, "channels": channels}


def listed():
    return [
        # one token of a narrow decoder: a launch's latency and nothing else
        _rotary("rotary_one_token", "bf16", 1, 4, 4, 64, 64, "half"),
        # the queries and keys of one block of the decoder workload (16 sequences of 1024, 12 heads)
        _rotary("rotary_block", "bf16", 16384, 12, 12, 64, 64, "half"),
        # the gradient in single precision: part of the head turns, positions far beyond the trained length
        _rotary("rotary_far_grad_f32", "f32", 5003, 16, 4, 128, 96, "interleaved", "by_parts", 16.0, 131072, True),
        # a handful of short ragged sequences, as in a small fine-tuning batch: latency and padding
        _attention("attn_short_ragged", "bf16", 5, 77, 77, 4, 4, 64, True, True, True),
        # one block of the decoder workload, forward and backward
        _attention("attn_block_train", "bf16", 8, 1024, 1024, 12, 12, 64, True, False, True),
        # long sequences, four query heads to a key head, 128 wide: the largest
        _attention("attn_long_grouped_train", "bf16", 2, 4096, 4096, 16, 4, 128, True, False, True),
        # ragged sequences that attend to ragged others in both directions, an odd head width, forward only
        _attention("attn_cross_forward", "bf16", 12, 509, 1301, 10, 5, 80, False, True, False),
        # single precision, more queries than keys in part of the rows' sequences
        _attention("attn_train_f32", "f32", 6, 421, 397, 6, 2, 64, True, True, True),
        # the input of one block's products in the decoder workload
        _checkpoint("checkpoint_block", "bf16", 16384, 768),
        # an odd number of rows, a last group that is not full
        _checkpoint("checkpoint_odd_f32", "f32", 1237, 1492),
        # the widest activation of one layer of the 64-layer workload (8192 rows, 4096 hidden)
        _gelu("gelu_layer", "bf16", 8192, 4096),
        # the stack of 32 rows that fits one launch
        _gelu("gelu_tiny_f32", "f32", 32, 256),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rotary", "attention", "attention", "checkpoint", "gelu"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op == "rotary":
        head = 8 * rng.randint(2, 16)
        turned = head if rng.random() < 0.5 else 8 * rng.randint(1, head // 8)
        kv = rng.choice([1, 2, 4, 6])
        q = kv * rng.choice([1, 2, 3, 4])
        scaling = rng.choice(["none", "linear", "by_parts"])
        return _bare(_rotary("", dtype, _log(rng, 1, 16384), q, kv, head, turned, rng.choice(["half", "interleaved"]), scaling,
                             1.0 if scaling == "none" else rng.choice([2.0, 8.0, 40.0]), _log(rng, 16, 1 << 20), rng.random() < 0.5))
    if op == "attention":
        while True:
            n, q = _log(rng, 1, 24), _log(rng, 1, 4096)
            same = rng.random() < 0.6
            kv = q if same else _log(rng, 1, 4096)
            kv_heads = rng.choice([1, 2, 4, 6])
            q_heads = kv_heads * rng.choice([1, 2, 4])
            # (rows that see one key only have gradients of zero, and what rounding leaves of them: forward passes alone)
            c = _attention("", dtype, n, q, kv, q_heads, kv_heads, rng.choice([64, 64, 128, 128, 8 * rng.randint(2, 16)]),
                           rng.random() < 0.7, rng.random() < 0.6, rng.random() < 0.6 and kv >= 16)
            # no more than the largest listed case costs, in either form
            limit = 6e7 if dtype == "f32" else 2.6e8
            if n * q_heads * q * kv <= limit and n * max(q, kv) <= 32768:
                return _bare(c)
    rows, channels = _log(rng, 1, 16384), 8 * _log(rng, 2, 1024)
    while rows * channels > (1 << 25):
        rows = max(1, rows // 2)
    return _bare(_checkpoint("", dtype, rows, channels) if op == "checkpoint" else _gelu("", dtype, rows, channels))


def _bare(c):
    return {k: v for k, v in c.items() if k != "name"}


# ------------------------------------------------------------------------------------------------- inputs
def _lengths(case, longest):
    """The sequences' lengths: all alike, or spread from one (or none at all, for the second) to the longest."""
    n = case["sequences"]
    if not case["ragged"] or n == 1:
        return [longest] * n
    out = [max(1, longest * ((i * 7) % n + 1) // n) for i in range(n)]
    out[0] = longest
    if n > 3:
        out[2] = 0
    return out


def _offsets(lengths):
    out = [0]
    for l in lengths:
        out.append(out[-1] + l)
    return out


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = DTYPE[case["dtype"]]

    def normal(*shape, std=1.0):
        return (torch.randn(*shape, generator=g, device="cuda") * std).to(dt)

    s = {"case": case}
    if case["op"] == "rotary":
        n, h = case["tokens"], case["head_dim"]
        s["q"], s["k"] = normal(n, case["q_heads"], h), normal(n, case["kv_heads"], h)
        s["positions"] = torch.randint(0, case["far"], (n,), generator=g, device="cuda", dtype=torch.int32)
    elif case["op"] == "attention":
        ql, kl = _lengths(case, case["q_len"]), _lengths(case, case["kv_len"])
        qo, ko = _offsets(ql), _offsets(kl)
        h = case["head_dim"]
        s["q"] = normal(qo[-1], case["q_heads"], h)
        s["k"], s["v"] = normal(ko[-1], case["kv_heads"], h), normal(ko[-1], case["kv_heads"], h)
        if case["train"]:
            s["d_o"] = normal(qo[-1], case["q_heads"], h, std=2.0 ** -10)
        s["q_offsets"] = torch.tensor(qo, device="cuda", dtype=torch.int32)
        s["kv_offsets"] = torch.tensor(ko, device="cuda", dtype=torch.int32)
        s["scale"] = 1.0 / math.sqrt(h)
    else:
        rows, d = case["rows"], case["channels"]
        # activations of a trained net: a few channels are much larger than the rest
        spread = torch.where(torch.rand(d, generator=g, device="cuda") < 0.02, 12.0, 1.0)
        s["x"] = (torch.randn(rows, d, generator=g, device="cuda") * spread).to(dt)
        if case["op"] == "gelu":
            s["d_act"] = normal(rows, d, std=2.0 ** -8)
    return s


# ------------------------------------------------------------------------------------------------- one pass
def run(state):
    if own:
        return _calls(state)
    return {"rotary": _plain_rotary, "attention": _plain_attention, "checkpoint": _plain_checkpoint,
            "gelu": _plain_gelu}[state["case"]["op"]](state)


def _calls(s):
    from paper_2501_17086_b200 import binding
    c = s["case"]
    if c["op"] == "rotary":
        q, k = binding.rotary(s["q"], s["k"], positions=s["positions"], rotary_dim=c["rotary_dim"], layout=c["layout"],
                              scaling=c["scaling"], factor=c["factor"], trained_length=TRAINED, amplitude=_amplitude(c),
                              inverse=c["inverse"])
        return {"q": q, "k": k}
    if c["op"] == "attention":
        ragged = {} if not c["ragged"] else {"q_offsets": s["q_offsets"], "kv_offsets": s["kv_offsets"]}
        kw = dict(sequences=c["sequences"], q_len=c["q_len"], kv_len=c["kv_len"], causal=c["causal"], scale=s["scale"], **ragged)
        o, lse = binding.attention_forward(s["q"], s["k"], s["v"], **kw)
        out = {"o": o, "lse": lse}
        if c["train"]:
            out["dq"], out["dk"], out["dv"] = binding.attention_backward(s["d_o"], s["q"], s["k"], s["v"], o, lse, **kw)
        return out
    if c["op"] == "checkpoint":
        codes, scales = binding.checkpoint_store(s["x"])
        return {"x": binding.checkpoint_load(codes, scales, s["x"].dtype)}
    act, codes, scales = binding.checkpoint_gelu(s["x"])
    dz, act8 = binding.checkpoint_gelu_backward(s["d_act"], codes, scales, with_act=True)
    return {"act": act, "dz": dz, "act8": act8}


# ------------------------------------------------------------------------------------------------- the plain forms
BASE, TRAINED, FAST, SLOW = 10000.0, 4096, 32.0, 1.0


def _amplitude(case):
    return 0.1 * math.log(case["factor"]) + 1.0 if case["scaling"] == "by_parts" else 1.0


def _turn(x, cos, sin, layout):
    """x [n, heads, r] turned: pairs are (i, i + r/2) in the half layout, (2i, 2i + 1) in the interleaved one."""
    if layout == "half":
        a, b = x.chunk(2, -1)
        return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    a, b = x[..., 0::2], x[..., 1::2]
    return torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)


def _plain_rotary(s):
    c = s["case"]
    r = c["rotary_dim"]
    freq = BASE ** (-torch.arange(0, r, 2, device="cuda", dtype=torch.float64) / r)
    if c["scaling"] == "linear":
        freq = freq / c["factor"]
    elif c["scaling"] == "by_parts":
        keep = ((TRAINED * freq / (2 * math.pi) - SLOW) / (FAST - SLOW)).clamp(0, 1)
        freq = freq * ((1 - keep) / c["factor"] + keep)
    angle = s["positions"].double()[:, None] * freq
    cos, sin = ((t * _amplitude(c)).float()[:, None] for t in (angle.cos(), angle.sin()))
    if c["inverse"]:
        sin = -sin

    def one(x):
        x32 = x.float()
        return torch.cat([_turn(x32[..., :r], cos, sin, c["layout"]), x32[..., r:]], -1).to(x.dtype)

    return {"q": one(s["q"]), "k": one(s["k"])}


def _padded(offsets, longest):
    """Rows of the padded batch [sequences, longest] in the packed one, and which of them there are."""
    at = torch.arange(longest, device="cuda")
    there = at < (offsets[1:] - offsets[:-1])[:, None]
    return torch.where(there, offsets[:-1, None] + at, 0), there


def _plain_attention(s):
    c = s["case"]
    group = c["q_heads"] // c["kv_heads"]
    qi, qt = _padded(s["q_offsets"], c["q_len"])
    ki, kt = _padded(s["kv_offsets"], c["kv_len"])

    def heads(x, at, there, rep):  # [sequences, heads, rows, width]
        x = torch.where(there[..., None, None], x.float()[at], 0.0).transpose(1, 2)
        return x.repeat_interleave(rep, 1) if rep > 1 else x

    q, k, v = heads(s["q"], qi, qt, 1), heads(s["k"], ki, kt, group), heads(s["v"], ki, kt, group)
    seen = kt[:, None, None, :] & qt[:, None, :, None]
    if c["causal"]:  # the last query sees the last key
        nq, nk = qt.sum(1), kt.sum(1)
        i, j = torch.arange(c["q_len"], device="cuda"), torch.arange(c["kv_len"], device="cuda")
        seen = seen & (j <= i[:, None] + (nk - nq)[:, None, None])[:, None]
    score = torch.where(seen, (q @ k.transpose(-1, -2)) * s["scale"], -math.inf)
    top = score.amax(-1, keepdim=True)
    p = (score - torch.where(top > -math.inf, top, 0.0)).exp()
    total = p.sum(-1, keepdim=True)
    lse = torch.where(total > 0, top + total.log(), -math.inf)
    p = p / torch.where(total > 0, total, 1.0)
    o = p @ v

    def packed(x, there):  # back to [rows, heads, width]
        return x.transpose(1, 2)[there]

    out = {"o": packed(o, qt).to(s["q"].dtype), "lse": packed(lse, qt)[..., 0].T.contiguous()}
    if c["train"]:
        d_o = heads(s["d_o"], qi, qt, 1)
        dv = p.transpose(-1, -2) @ d_o
        dp = d_o @ v.transpose(-1, -2)
        ds = p * (dp - (d_o * o).sum(-1, keepdim=True)) * s["scale"]
        dq, dk = ds @ k, ds.transpose(-1, -2) @ q
        dk, dv = (t.unflatten(1, (c["kv_heads"], group)).sum(2) for t in (dk, dv))
        out.update(dq=packed(dq, qt).to(s["q"].dtype), dk=packed(dk, kt).to(s["q"].dtype), dv=packed(dv, kt).to(s["q"].dtype))
    return out


def _codes(x):
    """x [rows, d] in groups of 32 channels: whole numbers of at most 127 and the powers of two that they count."""
    rows, d = x.shape
    x = torch.nn.functional.pad(x.float(), (0, -d % GROUP)).view(rows, -1, GROUP)
    m, e = torch.frexp(x.abs().amax(-1, keepdim=True))  # the largest is m * 2^e, 1/2 <= m < 1 (or zero)
    e = torch.where(m > 127 / 128, e - 6, e - 7).clamp(-126, 127)
    return torch.ldexp(x, -e).round(), e


def _values(codes, e, d):
    return torch.ldexp(codes, e).flatten(1)[:, :d]


def _plain_checkpoint(s):
    return {"x": _values(*_codes(s["x"]), s["x"].shape[1]).to(s["x"].dtype)}


def _gelu_of(z):
    phi = 0.5 * torch.erfc(-z * 0.5 ** 0.5)
    return z * phi, phi + z * torch.exp(-0.5 * z * z) * (0.5 / math.pi) ** 0.5


def _plain_gelu(s):
    dt = s["x"].dtype
    z8 = _values(*_codes(s["x"]), s["x"].shape[1])
    act8, slope = _gelu_of(z8)
    return {"act": _gelu_of(s["x"].float())[0].to(dt), "dz": (s["d_act"].float() * slope).to(dt), "act8": act8.to(dt)}


# ------------------------------------------------------------------------------------------------- the definitions in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "rotary":
        r, n = case["rotary_dim"], case["tokens"]
        pairs = r // 2
        out = {}
        turn = []
        for i in range(pairs):  # radians a position
            f = BASE ** (-2.0 * i / r)
            if case["scaling"] == "linear":
                f /= case["factor"]
            if case["scaling"] == "by_parts":
                turns = TRAINED * f / (2 * math.pi)
                w = min(1.0, max(0.0, (turns - SLOW) / (FAST - SLOW)))
                f = (1 - w) * f / case["factor"] + w * f
            turn.append(f)
        angle = s["positions"].double()[:, None] * torch.tensor(turn, dtype=torch.float64, device="cuda")
        spin = torch.polar(torch.full_like(angle, _amplitude(case)), -angle if case["inverse"] else angle)[:, None]
        for name in ("q", "k"):
            x = s[name].double()
            if case["layout"] == "half":
                z = torch.complex(x[..., :pairs], x[..., pairs:r]) * spin
                y = torch.cat([z.real, z.imag, x[..., r:]], -1)
            else:
                z = torch.view_as_complex(x[..., :r].reshape(n, -1, pairs, 2).contiguous()) * spin
                y = torch.cat([torch.view_as_real(z).reshape(n, -1, r), x[..., r:]], -1)
            out[name] = y
        return out
    if case["op"] == "attention":
        return _exact_attention(case, s)
    x = s["x"].double()
    rows, d = x.shape
    x8 = torch.empty_like(x)
    for lo in range(0, d, GROUP):
        part = x[:, lo:lo + GROUP]
        most = part.abs().amax(1, keepdim=True)
        step = torch.exp2(torch.ceil(torch.log2(most.clamp_min(2.0 ** -140) / 127.0)).clamp_min(-126))
        step = torch.where(most > 127 * step, 2 * step, step)  # where the logarithm was rounded past a border
        step = torch.where((most <= 63.5 * step) & (step > 2.0 ** -126), step / 2, step)
        x8[:, lo:lo + GROUP] = torch.round(part / step) * step
    if case["op"] == "checkpoint":
        return {"x": x8}

    def upper(z):  # the normal distribution's cumulative function
        return torch.special.ndtr(z)

    dens = torch.exp(-x8 ** 2 / 2) / math.sqrt(2 * math.pi)
    return {"act": x * upper(x), "dz": s["d_act"].double() * (upper(x8) + x8 * dens), "act8": x8 * upper(x8)}


def _exact_attention(case, s):
    qo, ko = s["q_offsets"].tolist(), s["kv_offsets"].tolist()
    group = case["q_heads"] // case["kv_heads"]
    q, k, v = s["q"].double(), s["k"].double(), s["v"].double()
    o = torch.zeros_like(q)
    lse = torch.full((case["q_heads"], q.shape[0]), -math.inf, dtype=torch.float64, device="cuda")
    dq, dk, dv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    for b in range(case["sequences"]):
        rows, cols = slice(qo[b], qo[b + 1]), slice(ko[b], ko[b + 1])
        nq, nk = qo[b + 1] - qo[b], ko[b + 1] - ko[b]
        if nq == 0 or nk == 0:
            continue
        hidden = torch.zeros(nq, nk, dtype=torch.bool, device="cuda")
        if case["causal"]:
            hidden = torch.ones_like(hidden).triu(nk - nq + 1)
        empty = hidden.all(1)
        for h in range(case["q_heads"]):
            kh = h // group
            score = (q[rows, h] @ k[cols, kh].T * s["scale"]).masked_fill(hidden, -math.inf)
            l = torch.logsumexp(score, 1)
            p = torch.exp(score - torch.where(empty, 0.0, l)[:, None])
            lse[h, rows] = l
            o[rows, h] = p @ v[cols, kh]
            if case["train"]:
                d_o = s["d_o"][rows, h].double()
                inner = d_o @ v[cols, kh].T
                ds = p * (inner - (d_o * o[rows, h]).sum(1, keepdim=True))
                dq[rows, h] = s["scale"] * (ds @ k[cols, kh])
                dk[cols, kh] += s["scale"] * (ds.T @ q[rows, h])
                dv[cols, kh] += p.T @ d_o
    return {"o": o, "lse": lse, "dq": dq, "dk": dk, "dv": dv} if case["train"] else {"o": o, "lse": lse}


# ------------------------------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    es = ES[case["dtype"]]
    if case["op"] == "rotary":
        heads = case["q_heads"] + case["kv_heads"]
        return {"bytes": case["tokens"] * (2 * es * heads * case["head_dim"] + 4), "flops": 3 * case["tokens"] * heads * case["rotary_dim"]}
    if case["op"] == "attention":
        ql, kl = _lengths(case, case["q_len"]), _lengths(case, case["kv_len"])
        pairs = 0
        for nq, nk in zip(ql, kl):
            if case["causal"]:  # query i sees the first i + nk - nq + 1 keys
                lo = max(0, nq - nk)
                pairs += sum(range(lo + nk - nq + 1, nk + 1)) if nk else 0
            else:
                pairs += nq * nk
        q, k = sum(ql) * case["q_heads"] * case["head_dim"] * es, sum(kl) * case["kv_heads"] * case["head_dim"] * es
        product = 2 * pairs * case["q_heads"] * case["head_dim"]
        lse = 4 * sum(ql) * case["q_heads"]
        if case["train"]:  # q, k, v, the output and its gradient once each, three gradients written
            return {"bytes": 4 * q + 4 * k + lse, "flops": 7 * product}
        return {"bytes": 2 * q + 2 * k + lse, "flops": 2 * product}
    n = case["rows"] * case["channels"]
    kept = n + n // GROUP
    if case["op"] == "checkpoint":  # written, and read back
        return {"bytes": 2 * n * es + 2 * kept, "flops": 3 * n}
    return {"bytes": 5 * n * es + 2 * kept, "flops": 40 * n}
