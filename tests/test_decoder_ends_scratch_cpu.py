"""Scratch that is enough for some number of rows is enough for fewer, as batches of different lengths share it.  No GPU needed: the calls are made
by a process that sees no device, where one that gets past its checks ends with HBP_ERR_CUDA before anything is launched; pointers are made
up and never followed."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CROSS_ENTROPY = """
import ctypes as C
import torch
from paper_2501_17086_b200 import binding as B
assert torch.cuda.device_count() == 0
P, CUDA = 0x10000, 7
SHAPES = [(torch.bfloat16, v, d) for v, d in ((4099, 2048), (8192, 4096), (32003, 1024), (131072, 1024), (32003, 4096), (300, 64), (50021, 768), (7, 8192))]
SHAPES += [(torch.float32, v, d) for v, d in ((8111, 520), (32003, 1024), (5003, 512), (20011, 2052), (3, 4096), (20011, 4))]
wrong = []
for dtype, vocab, d in SHAPES:
    bf16 = dtype == torch.bfloat16
    rows = sorted({*range(1, 40), *range(120, 140), 255, 256, 257, 511, 512, 513, *range(16, 2400, 16), *range(2400, 70000, 1100), 1 << 20})
    for grads in (False, True):
        size = {n: B.cross_entropy_scratch_bytes(dtype, n, vocab, d, grads) for n in rows}
        least = 1 << 62  # that any number of rows from here on has
        for n in reversed(rows):
            least = min(least, size[n])
            v = B.hbp_vocabulary(int(bf16), vocab, d, 8, n, P, d, P, d, P, None)
            if not grads:
                if B.lib.hbp_cross_entropy(C.byref(v), P, P, least, None) != CUDA:
                    wrong.append((dtype, vocab, d, n, "loss"))
                continue
            for dx, dw, type_w in ((P, P, 0), (P, P, int(bf16)), (P, None, 0), (None, P, int(bf16))):
                if B.lib.hbp_cross_entropy_gradients(C.byref(v), P, 1, P, dx, d, dw, type_w, d, P, least, None) != CUDA:
                    wrong.append((dtype, vocab, d, n, dx, dw, type_w))
assert not wrong, (len(wrong), wrong[:20])
"""


def test_scratch_of_many_rows_is_enough_for_fewer():
    from paper_2501_17086_b200.build import build_library
    build_library()
    env = {**os.environ, "CUDA_VISIBLE_DEVICES": "", "PYTHONPATH": ROOT}
    done = subprocess.run([sys.executable, "-c", CROSS_ENTROPY], env=env, capture_output=True, text=True, timeout=300)
    assert done.returncode == 0, done.stderr[-2000:]


EMBEDDING_GRADIENT = """
import ctypes as C
import torch
from paper_2501_17086_b200 import binding as B
assert torch.cuda.device_count() == 0
P, CUDA = 0x10000, 7
def size(n, d):
    need = C.c_size_t()
    assert B.lib.hbp_embedding_gradient_scratch_bytes(n, d, C.byref(need)) == 0
    return need.value
ends = [1 << 16, 1 << 17, 1 << 18, 1 << 19, 1 << 20]
rows = sorted({*range(0, 300), *range(300, 1 << 20, 4099), *ends, *(n + 1 for n in ends), *(n - 1 for n in ends), 1 << 30})
for d in (8, 24, 768, 8192):
    sizes = [size(n, d) for n in rows]
    assert sizes == sorted(sizes), d
    for n, more in zip(rows, sizes[1:]):
        if n:
            assert B.lib.hbp_embedding_gradient(1, n, 1000, d, P, 8, P, d, 1.0, None, P, P, more, None, None) == CUDA, (n, d)
"""


def test_scratch_of_many_tokens_is_enough_for_fewer():
    from paper_2501_17086_b200.build import build_library
    build_library()
    env = {**os.environ, "CUDA_VISIBLE_DEVICES": "", "PYTHONPATH": ROOT}
    done = subprocess.run([sys.executable, "-c", EMBEDDING_GRADIENT], env=env, capture_output=True, text=True, timeout=300)
    assert done.returncode == 0, done.stderr[-2000:]
