"""Builds libhbp.so (sm_100a only, nvcc) and the extension module _calls.so (marshalling of the short calls, g++ with torch's
headers) next to this file; no GPU needed."""
from __future__ import annotations

import importlib.metadata
import os
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libhbp.so")
CALLS = os.path.join(HERE, "_calls.so")
CALLS_FOR = os.path.join(HERE, "_build", "calls.for")  # what the extension module was built against
SOURCES = ["hbp_api.cu", "gemm_simt.cu", "gemm_tc.cu", "gemm_f32.cu", "gemm_parts.cu", "gemm_cell.cu", "few_rows.cu", "scan.cu", "scan_static.cu", "scan_ring.cu", "attention.cu", "attention_tc.cu", "rnn.cu", "rnn_persistent.cu", "rnn_cluster.cu", "cell_cluster.cu", "gru.cu", "lstm.cu", "diag.cu", "rotary.cu",
           "checkpoint.cu", "attention_ragged.cu", "attention_ragged_tc.cu"]


def _built_for() -> str:
    return f"torch {importlib.metadata.version('torch')}, python {sys.version}"


def _stale() -> bool:
    if not os.path.exists(LIB) or not os.path.exists(CALLS) or not os.path.exists(CALLS_FOR):
        return True
    with open(CALLS_FOR) as f:
        if f.read() != _built_for():
            return True
    t = min(os.path.getmtime(LIB), os.path.getmtime(CALLS))
    deps = [os.path.join(CSRC, f) for f in os.listdir(CSRC)] + [os.path.join(ROOT, "include", "hbp.h")]
    return any(os.path.getmtime(d) > t for d in deps)


def build_library(force: bool = False, verbose: bool = False) -> str:
    if not force and not _stale():
        return LIB
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    obj_dir = os.path.join(HERE, "_build")
    os.makedirs(obj_dir, exist_ok=True)
    common = [nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-O3", "-lineinfo", "-std=c++17",
              "-Xcompiler", "-fPIC", "-I" + os.path.join(ROOT, "include"), "-I" + CSRC]
    if verbose:
        common += ["-Xptxas", "-v"]
    calls = _compile_calls(obj_dir)
    procs, objs = [], []
    for src in SOURCES:
        obj = os.path.join(obj_dir, src.replace(".cu", ".o"))
        objs.append(obj)
        procs.append((src, subprocess.Popen(common + ["-c", os.path.join(CSRC, src), "-o", obj],
                                            stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
    failed = False
    for src, p in procs + [("calls.cpp", calls)]:
        out, _ = p.communicate()
        if out.strip():
            print(out, file=sys.stderr)
        if p.returncode != 0 and p is not calls:
            failed = True
    if failed:
        raise RuntimeError("nvcc failed")
    subprocess.check_call([nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-shared", "-o", LIB] + objs + ["-lcudart"])
    if calls.returncode != 0:  # (the library is there: contexts work without the extension module)
        raise RuntimeError("g++ failed: no extension module for the short calls")
    _link_calls(obj_dir)
    with open(CALLS_FOR, "w") as f:
        f.write(_built_for())
    return LIB


def _compile_calls(obj_dir: str) -> subprocess.Popen:
    import torch
    base = os.path.join(os.path.dirname(torch.__file__), "include")
    cuda = os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "include")
    return subprocess.Popen(["g++", "-O2", "-std=c++17", "-fPIC", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
                             "-isystem", base, "-isystem", os.path.join(base, "torch", "csrc", "api", "include"), "-isystem", cuda,
                             "-isystem", sysconfig.get_paths()["include"], "-I" + os.path.join(ROOT, "include"), "-c",
                             os.path.join(CSRC, "calls.cpp"), "-o", os.path.join(obj_dir, "calls.o")],
                            stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)


def _link_calls(obj_dir: str) -> None:
    import torch
    libs = os.path.join(os.path.dirname(torch.__file__), "lib")
    subprocess.check_call(["g++", "-shared", "-o", CALLS, os.path.join(obj_dir, "calls.o"), "-L" + HERE, "-lhbp", "-L" + libs, "-ltorch_python", "-ltorch_cpu",
                           "-lc10_cuda", "-lc10", "-Wl,-rpath,$ORIGIN"])


if __name__ == "__main__":
    print(build_library(force="--force" in sys.argv, verbose="-v" in sys.argv))
