"""Refusals of the stand-alone operators of a decoder's step, all before any CUDA call: no GPU needed.  Pointers are made up and
never followed."""
import ctypes as C

import pytest

OK, INVALID, SHAPE, DTYPE, WORKSPACE, UNSUPPORTED = 0, 1, 2, 3, 5, 6
P = 0x10000  # 16-byte aligned, never followed


@pytest.fixture(scope="module")
def B():
    from paper_2501_17086_b200.build import build_library
    build_library()
    from paper_2501_17086_b200 import binding
    return binding


def test_struct_layouts_match_the_header(B):
    assert C.sizeof(B.hbp_heads) == 24
    assert C.sizeof(B.hbp_rotary_spec) == 36
    assert C.sizeof(B.hbp_attention) == 80


def _rotary(B, spec=None, dtype=0, rows=4, q_heads=2, kv_heads=1, head_dim=64, positions=None, size=0, period=0, q=None, qo=None, k=None, ko=None):
    spec = B.rotary_spec(64) if spec is None else spec
    q, qo = q or B.hbp_heads(P, 128, 64), qo or B.hbp_heads(P + 4096, 128, 64)
    k, ko = k or B.hbp_heads(P + 8192, 64, 64), ko or B.hbp_heads(P + 12288, 64, 64)
    return B.lib.hbp_rotary(C.byref(spec), 0, dtype, rows, q_heads, kv_heads, head_dim, positions, size, 0, period, C.byref(q), C.byref(qo),
                            C.byref(k), C.byref(ko), None)


def test_rotary_refusals(B):
    S = B.rotary_spec
    assert _rotary(B, rows=0) == OK                                    # nothing to do
    assert _rotary(B, dtype=5) == DTYPE
    assert _rotary(B, rows=-1) == SHAPE
    assert _rotary(B, q_heads=0) == SHAPE
    assert _rotary(B, head_dim=62) == SHAPE
    assert _rotary(B, head_dim=264, spec=S(64)) == SHAPE               # wider than 256
    for bad in (S(63), S(0), S(66)):                                   # odd, none, wider than the head
        assert _rotary(B, spec=bad) == SHAPE
    for bad in (S(64, base=1.0), S(64, base=float("nan")), S(64, scaling="linear", factor=0.5), S(64, amplitude=float("inf")),
                S(64, scaling="by_parts", factor=2.0), S(64, scaling="by_parts", factor=2.0, trained_length=10.0, fast=1.0, slow=1.0)):
        assert _rotary(B, spec=bad) == INVALID
    bad = S(64)
    bad.layout = 2
    assert _rotary(B, spec=bad) == UNSUPPORTED
    bad = S(64)
    bad.scaling = -1
    assert _rotary(B, spec=bad) == UNSUPPORTED
    assert _rotary(B, period=-1) == INVALID
    assert _rotary(B, positions=P, size=2) == INVALID
    assert _rotary(B, positions=P + 4, size=8) == SHAPE
    assert _rotary(B, q=B.hbp_heads(0, 128, 64)) == INVALID
    assert _rotary(B, q=B.hbp_heads(P + 4, 128, 64)) == SHAPE
    assert _rotary(B, ko=B.hbp_heads(P, 66, 64)) == SHAPE
    assert _rotary(B, qo=B.hbp_heads(P, 192, 64)) == INVALID           # in place, other rows
    for rs, hs in ((0, 64), (64, 64), (128, 0), (-128, 64)):             # outputs on one another
        assert _rotary(B, qo=B.hbp_heads(P + 4096, rs, hs)) == SHAPE, (rs, hs)
    with pytest.raises(B.HbpError) as e:
        S(64, layout="other")
    assert e.value.code == UNSUPPORTED


def _attention(B, backward=False, tensors=None, lse=P, scratch=P, scratch_bytes=1 << 20, **change):
    a = B.hbp_attention(1, 1, 2, 4, 2, 64, 16, 16, 32, 32, None, None, 0.125, None)
    for name, v in change.items():
        setattr(a, name, v)
    t = [C.byref(x) for x in (tensors or [B.hbp_heads(P, 256, 64)] * (8 if backward else 4))]
    if backward:
        return B.lib.hbp_attention_backward(C.byref(a), *t[:5], lse, *t[5:], scratch, scratch_bytes, None)
    return B.lib.hbp_attention_forward(C.byref(a), *t, lse, None)


@pytest.mark.parametrize("backward", [False, True])
def test_attention_refusals(B, backward):
    def call(**kw):
        return _attention(B, backward, **kw)

    assert call(sequences=0) == OK                                      # nothing to do
    assert call(dtype=2) == DTYPE
    for kw in (dict(sequences=-1), dict(q_heads=0), dict(kv_heads=0), dict(kv_heads=3), dict(head_dim=0), dict(head_dim=136),
               dict(head_dim=68), dict(dtype=0, head_dim=66), dict(q_len=-1), dict(q_len=17), dict(kv_len=17), dict(q_rows=-1),
               dict(q_rows=1 << 31), dict(kv_rows=1 << 31), dict(q_len=33, q_offsets=P), dict(kv_len=33, kv_offsets=P),
               dict(q_offsets=P + 2), dict(status=P + 1)):
        assert call(**kw) == SHAPE, kw
    assert call(scale=float("nan")) == INVALID
    assert call(lse=None) == INVALID
    n = 8 if backward else 4
    good = B.hbp_heads(P, 256, 64)
    for i in range(n):
        for bad, code in ((B.hbp_heads(0, 256, 64), INVALID), (B.hbp_heads(P + 8, 256, 64), SHAPE), (B.hbp_heads(P, 260, 64), SHAPE),
                          (B.hbp_heads(P, 256, 4), SHAPE), (B.hbp_heads(P, -256, 64), SHAPE)):
            assert call(tensors=[bad if j == i else good for j in range(n)]) == code, (i, bad.row_stride)
    for i in ((5, 6, 7) if backward else (3,)):  # outputs whose rows or heads lie on one another; heads before rows is another matter
        for rs, hs in ((0, 64), (256, 0), (192, 64), (256, 56), (48, 2048)):
            assert call(tensors=[B.hbp_heads(P, rs, hs) if j == i else good for j in range(n)], kv_heads=4) == SHAPE, (i, rs, hs)
    if backward:
        assert call(scratch=None) == WORKSPACE
        assert call(scratch_bytes=4 * 4 * 32 - 1) == WORKSPACE
        assert call(scratch=P + 4) == WORKSPACE
        assert B.attention_scratch_bytes(4, 32) == 4 * 4 * 32
    assert B.lib.hbp_attention_forward(None, None, None, None, None, None, None) == INVALID
    assert B.lib.hbp_attention_scratch_bytes(None, None) == INVALID


def test_checkpoint_refusals(B):
    lib = B.lib

    def gelu(dtype=1, rows=4, d=64, z=P, ldz=64, act=P + 4096, lda=64, codes=P, scales=P):
        return lib.hbp_checkpoint_gelu(dtype, rows, d, z, ldz, act, lda, codes, scales, None)

    def back(dtype=1, rows=4, d=64, g=P, ldg=64, dz=P + 4096, ldz=64, act=None, lda=0, codes=P, scales=P):
        return lib.hbp_checkpoint_gelu_backward(dtype, rows, d, codes, scales, g, ldg, dz, ldz, act, lda, None)

    assert gelu(rows=0) == OK and back(rows=0) == OK
    assert gelu(dtype=2) == DTYPE
    for kw in (dict(rows=-1), dict(d=0), dict(d=68), dict(dtype=0, d=66, ldz=68, lda=68), dict(ldz=56), dict(ldz=68), dict(lda=60), dict(z=P + 2),
               dict(act=P + 8), dict(codes=P + 4), dict(rows=1 << 62)):
        assert gelu(**kw) == SHAPE, kw
    for kw in (dict(z=None), dict(act=None), dict(codes=None), dict(scales=None), dict(act=P, lda=72)):
        assert gelu(**kw) == INVALID, kw
    for kw in (dict(act=P + 8, lda=64), dict(act=P, lda=56), dict(dz=P + 2)):
        assert back(**kw) == SHAPE, kw
    for kw in (dict(g=None), dict(dz=None), dict(codes=None), dict(scales=None), dict(dz=P, ldz=72)):
        assert back(**kw) == INVALID, kw
    assert lib.hbp_checkpoint_store(1, 4, 64, None, 64, P, P, None) == INVALID
    assert lib.hbp_checkpoint_store(1, 4, 64, P, 32, P, P, None) == SHAPE
    assert lib.hbp_checkpoint_load(1, 4, 64, P, P, None, 64, None) == INVALID
    assert lib.hbp_checkpoint_load(7, 4, 64, P, P, P, 64, None) == DTYPE
    assert lib.hbp_checkpoint_load(1, 0, 64, None, None, None, 64, None) == OK


def test_fresh_outputs_are_named_by_known_bits(B):
    """hbp_attention's `fresh` lies before `status` (its ctypes structure leaves the four bytes out)."""
    for bits, code in ((1 << 5, INVALID), (-1, INVALID), (31, OK)):
        for backward in (False, True):
            a = B.hbp_attention(1, 1, 0, 4, 2, 64, 0, 0, 0, 0, None, None, 0.125, None)  # (no sequences, no rows: nothing to do)
            C.c_int32.from_buffer(a, B.hbp_attention.status.offset - 4).value = bits
            t = C.byref(B.hbp_heads(P, 256, 64))
            got = (B.lib.hbp_attention_backward(C.byref(a), t, t, t, t, t, P, t, t, t, P, 1 << 20, None) if backward else
                   B.lib.hbp_attention_forward(C.byref(a), t, t, t, t, P, None))
            assert got == code, (bits, backward)


def test_tensors_that_ask_for_gradients_are_refused(B):
    """Where gradients are recorded; elsewhere the next check speaks (here that of the device)."""
    import torch
    x, plain = torch.zeros(4, 2, 64, requires_grad=True), torch.zeros(4, 2, 64)
    m, codes, scales = torch.zeros(4, 64, requires_grad=True), torch.zeros(4, 64, dtype=torch.int8), torch.zeros(4, 2, dtype=torch.uint8)
    calls = [lambda: B.rotary(x), lambda: B.attention_forward(x, plain, plain), lambda: B.attention_backward(x, x, x, x, x, x), lambda: B.checkpoint_store(m),
             lambda: B.checkpoint_gelu(m), lambda: B.checkpoint_gelu_backward(m, codes, scales)]
    for call in calls:
        with pytest.raises(B.HbpError) as e:
            call()
        assert e.value.code == UNSUPPORTED
        with torch.no_grad(), pytest.raises(B.HbpError) as e:
            call()
        assert e.value.code == INVALID
    with torch.no_grad(), pytest.raises(B.HbpError) as e:
        B.rotary(plain, plain)
    assert e.value.code == INVALID
