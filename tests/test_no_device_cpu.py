"""A process that sees no GPU gets an error status from the calls that would launch, and lives.  Pointers are made up and never followed."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CALLS = """
import ctypes as C, sys
import torch
from paper_2501_17086_b200 import binding as B
assert torch.cuda.device_count() == 0
P, CUDA, dtype = 0x10000, 7, int(sys.argv[1])
def vocabulary(rows):
    return C.byref(B.hbp_vocabulary(dtype, 1000, 64, 8, rows, P, 64, P, 64, P, None))
for rows in (1, 100, 300):
    got = [B.lib.hbp_cross_entropy(vocabulary(rows), P, P, 1 << 30, None),
           B.lib.hbp_cross_entropy_gradients(vocabulary(rows), P, 1, P, P, 64, P, 0, 64, P, 1 << 30, None),
           B.lib.hbp_embedding(dtype, rows, 1000, 64, P, 8, P, 64, 1.0, P, 64, None, None),
           B.lib.hbp_embedding_gradient(dtype, rows, 1000, 64, P, 8, P, 64, 1.0, None, P, P, 1 << 30, None, None)]
    n, r = B.hbp_norm(dtype, 0, rows, 64, 0, 1e-5, 1.0, None, None, None), [C.byref(B.hbp_rows(P + i * (1 << 20), 64)) for i in range(7)]
    got += [B.lib.hbp_norm_residual(C.byref(n), *r[:4], None), B.lib.hbp_norm_residual_backward(C.byref(n), *r, P, None, None, P, 1 << 30, None)]
    assert got == [CUDA] * len(got), (rows, got)
"""


@pytest.mark.parametrize("dtype", [0, 1])
def test_calls_without_a_device_return_an_error(dtype):
    from paper_2501_17086_b200.build import build_library
    build_library()
    env = {**os.environ, "CUDA_VISIBLE_DEVICES": "", "PYTHONPATH": ROOT}
    done = subprocess.run([sys.executable, "-c", CALLS, str(dtype)], env=env, capture_output=True, text=True, timeout=300)
    assert done.returncode == 0, (done.returncode, done.stderr[-2000:])
