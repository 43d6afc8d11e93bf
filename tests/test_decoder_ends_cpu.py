"""Refusals of the operators at a decoder's ends and between its blocks, all before any CUDA call: no GPU needed.  Pointers are made up and
never followed."""
import ctypes as C

import pytest

OK, INVALID, SHAPE, DTYPE, WORKSPACE, UNSUPPORTED = 0, 1, 2, 3, 5, 6
P = 0x10000  # 256-byte aligned, never followed


@pytest.fixture(scope="module")
def B():
    from paper_2501_17086_b200.build import build_library
    build_library()
    from paper_2501_17086_b200 import binding
    return binding


def test_struct_layouts_match_the_header(B):
    assert C.sizeof(B.hbp_norm) == 56
    assert C.sizeof(B.hbp_rows) == 16
    assert C.sizeof(B.hbp_vocabulary) == 72


def test_embedding_refusals(B):
    def call(dtype=1, rows=0, vocab=100, d=64, tokens=P, size=8, table=P, ldt=64, scale=1.0, out=P, ldo=64, status=None):
        return B.lib.hbp_embedding(dtype, rows, vocab, d, tokens, size, table, ldt, scale, out, ldo, status, None)

    assert call() == OK  # nothing to do
    assert call(dtype=2) == DTYPE
    for kw in (dict(rows=-1), dict(rows=(1 << 30) + 1), dict(vocab=0), dict(vocab=(1 << 30) + 1), dict(d=0), dict(d=60), dict(dtype=0, d=62), dict(tokens=P + 4),
               dict(tokens=P + 2, size=4), dict(status=P + 2), dict(rows=1, table=P + 8), dict(rows=1, out=P + 8), dict(rows=1, ldt=56), dict(rows=1, ldt=68),
               dict(rows=1, ldt=-64), dict(rows=1, ldo=0), dict(rows=1, ldo=56)):
        assert call(**kw) == SHAPE, kw
    for kw in (dict(size=2), dict(scale=float("nan")), dict(scale=float("inf")), dict(rows=1, tokens=None), dict(rows=1, table=None), dict(rows=1, out=None)):
        assert call(**kw) == INVALID, kw


def test_embedding_gradient_refusals(B):
    need = C.c_size_t()
    assert B.lib.hbp_embedding_gradient_scratch_bytes(1000, 64, C.byref(need)) == OK
    assert B.lib.hbp_embedding_gradient_scratch_bytes(-1, 64, C.byref(need)) == SHAPE
    assert B.lib.hbp_embedding_gradient_scratch_bytes(1000, 64, None) == INVALID

    def call(dtype=1, rows=1000, vocab=100, d=64, tokens=P, size=8, g=P, ldd=64, scale=1.0, add=None, table=P, scratch=P, nbytes=need.value, status=None):
        return B.lib.hbp_embedding_gradient(dtype, rows, vocab, d, tokens, size, g, ldd, scale, add, table, scratch, nbytes, status, None)

    assert call(rows=0, add=P) == OK  # in place, nothing to add
    assert call(dtype=7) == DTYPE
    for kw in (dict(rows=-1), dict(vocab=0), dict(d=68), dict(g=P + 2), dict(ldd=32), dict(ldd=-64), dict(add=P + 4), dict(table=P + 8), dict(tokens=P + 1)):
        assert call(**kw) == SHAPE, kw
    for kw in (dict(table=None), dict(tokens=None), dict(g=None), dict(size=1), dict(scale=float("nan"))):
        assert call(**kw) == INVALID, kw
    for kw in (dict(scratch=None), dict(nbytes=need.value - 1), dict(scratch=P + 8)):
        assert call(**kw) == WORKSPACE, kw


def _norm(B, **change):
    n = B.hbp_norm(1, 0, 4, 64, 0, 1e-5, 1.0, None, None, None)
    for name, v in change.items():
        setattr(n, name, v)
    return n


def test_norm_refusals(B):
    R = B.hbp_rows

    def forward(x=R(P, 64), f=R(P + 4096, 64), new=R(P + 8192, 64), y=R(P + 12288, 64), **change):
        return B.lib.hbp_norm_residual(C.byref(_norm(B, **change)), *[C.byref(t) for t in (x, f, new, y)], None)

    def backward(dy=R(P, 64), dn=R(P + 4096, 64), new=R(P + 8192, 64), f=R(P + 12288, 64), x=R(P + 16384, 64), dx=R(P + 20480, 64), df=R(P + 24576, 64), w=(None, None, None),
                 scratch=P, nbytes=1 << 20, **change):
        return B.lib.hbp_norm_residual_backward(C.byref(_norm(B, **change)), *[C.byref(t) for t in (dy, dn, new, f, x, dx, df)], *w, scratch, nbytes, None)

    none = R(None, 0)
    assert forward(rows=0) == OK and backward(rows=0) == OK
    for call in (forward, backward):
        assert call(dtype=3) == DTYPE
        assert call(kind=2) == UNSUPPORTED
        for kw in (dict(rows=-1), dict(rows=1 << 31), dict(d=0), dict(d=60), dict(d=8200), dict(w_pre=P + 4), dict(gate=P + 8), dict(w_post=P + 2), dict(f=R(P + 8, 64)),
                   dict(f=R(P, 68)), dict(f=R(P, 32)), dict(x=R(P, -64))):
            assert call(**kw) == SHAPE, kw
        for kw in (dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(scale=float("nan"))):
            assert call(**kw) == INVALID, kw
    for kw in (dict(x=none), dict(new=none), dict(f=none), dict(f=none, new=none, y=none), dict(f=none, new=none, gate=P), dict(f=none, new=none, post=1),
               dict(y=R(P + 8192, 64)), dict(new=R(P, 72)), dict(y=R(P + 4096, 72)), dict(y=R(P, 72))):
        assert forward(**kw) == INVALID, kw
    for kw in (dict(new=R(P, 0)), dict(y=R(P, 0))):  # an output of one row for all
        assert forward(**kw) == SHAPE, kw
    for kw in (dict(dx=R(P, 0)), dict(df=R(P, 48)), dict(w=(P + 4, None, None))):
        assert backward(**kw) == SHAPE, kw
    for kw in (dict(dy=none, dn=none), dict(new=none), dict(f=none, post=1), dict(x=none, w=(None, None, P)), dict(w=(None, P, None)), dict(dy=none, w=(P, None, None)),
               dict(dx=none, df=none), dict(df=R(P + 20480, 64)), dict(dx=R(P, 72)), dict(df=R(P + 16384, 128))):
        assert backward(**kw) == INVALID, kw
    need = C.c_size_t()
    assert B.lib.hbp_norm_residual_scratch_bytes(4, 64, C.byref(need)) == OK
    for kw in (dict(scratch=None), dict(scratch=P + 4), dict(nbytes=need.value - 1)):
        assert backward(w=(P, None, None), **kw) == WORKSPACE, kw
    assert B.lib.hbp_norm_residual_scratch_bytes(4, 8200, C.byref(need)) == SHAPE
    assert B.lib.hbp_norm_residual_scratch_bytes(4, 64, None) == INVALID
    assert B.lib.hbp_norm_residual(None, None, None, None, None, None) == INVALID
    with pytest.raises(B.HbpError) as e:
        B.norm_residual(None, kind="other")
    assert e.value.code == UNSUPPORTED


def test_cross_entropy_refusals(B):
    def vocabulary(**change):
        v = B.hbp_vocabulary(1, 1000, 64, 8, 100, P, 64, P, 64, P, None)
        for name, x in change.items():
            setattr(v, name, x)
        return v

    need = B.cross_entropy_scratch_bytes(__import__("torch").bfloat16, 100, 1000, 64)

    def loss(out=P, scratch=P, nbytes=need, **change):
        return B.lib.hbp_cross_entropy(C.byref(vocabulary(**change)), out, scratch, nbytes, None)

    def grads(d_loss=P, stride=1, out=P, dx=P, lddx=64, dw=P, dw_dtype=0, lddw=64, scratch=P, nbytes=need, **change):
        return B.lib.hbp_cross_entropy_gradients(C.byref(vocabulary(**change)), d_loss, stride, out, dx, lddx, dw, dw_dtype, lddw, scratch, nbytes, None)

    assert loss(rows=0) == OK and grads(rows=0, dw=None) == OK
    for call in (loss, grads):
        assert call(dtype=2) == DTYPE
        for kw in (dict(rows=-1), dict(rows=(1 << 30) + 1), dict(vocab=0), dict(vocab=(1 << 30) + 1), dict(d=60), dict(d=0), dict(d=1 << 25), dict(targets=P + 4),
                   dict(status=P + 2), dict(x=P + 8), dict(w=P + 8), dict(ldx=56), dict(ldx=68), dict(ldx=0), dict(ldw=0), dict(out=P + 2)):
            assert call(**kw) == SHAPE, kw
        for kw in (dict(target_bytes=2), dict(x=None), dict(w=None), dict(targets=None), dict(out=None)):
            assert call(**kw) == INVALID, kw
        for kw in (dict(scratch=None), dict(scratch=P + 128), dict(nbytes=1000)):
            assert call(**kw) == WORKSPACE, kw
    for kw in (dict(stride=-1), dict(d_loss=P + 2), dict(dx=P + 8), dict(lddx=0), dict(lddx=56), dict(dw=P + 4), dict(lddw=60), dict(lddw=66)):
        assert grads(**kw) == SHAPE, kw
    assert grads(dx=None, dw=None) == INVALID
    assert grads(dw_dtype=2) == DTYPE
    assert grads(dtype=0, dw_dtype=1) == DTYPE
    assert B.lib.hbp_cross_entropy(None, P, P, need, None) == INVALID
    assert B.lib.hbp_cross_entropy_scratch_bytes(None, 0, None) == INVALID


def test_scratch_grows_with_rows_up_to_a_piece(B):
    import torch
    for dtype in (torch.float32, torch.bfloat16):
        for grads in (False, True):
            sizes = [B.cross_entropy_scratch_bytes(dtype, n, 131072, 1024, grads) for n in (0, 1, 256, 4096, 65536, 1 << 20)]
            assert sizes[0] == 0 and sizes[1] <= sizes[2] <= sizes[3] and max(sizes) < 7 << 30


def test_tensors_that_ask_for_gradients_are_refused(B):
    """Where gradients are recorded; elsewhere the next check speaks (here that of the device)."""
    import torch
    x, w, t = torch.zeros(4, 64, requires_grad=True), torch.zeros(9, 64), torch.zeros(4, dtype=torch.int64)
    calls = [lambda: B.embedding(t, x), lambda: B.embedding_gradient(t, x, 9), lambda: B.norm_residual(x), lambda: B.norm_residual_backward(x, w), lambda: B.cross_entropy(x, w, t),
             lambda: B.cross_entropy_gradients(x, w, t)]
    for call in calls[2:]:
        with pytest.raises(B.HbpError) as e:
            call()
        assert e.value.code == UNSUPPORTED
    for call in calls:
        with torch.no_grad(), pytest.raises(B.HbpError) as e:
            call()
        assert e.value.code == INVALID
