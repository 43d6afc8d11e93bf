"""The extension module of the short calls: what works without it, and when it is built anew.  No GPU needed."""
import os
import shutil
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def build():
    from paper_2501_17086_b200 import build
    build.build_library()
    return build


def test_contexts_do_without_the_extension_module(build, tmp_path):
    package = tmp_path / "paper_2501_17086_b200"
    package.mkdir()
    for name in ("__init__.py", "binding.py", "workloads.py"):
        shutil.copy(os.path.join(build.HERE, name), package / name)
    os.symlink(build.LIB, package / "libhbp.so")
    program = """
from paper_2501_17086_b200 import binding
from paper_2501_17086_b200.workloads import WORKLOADS
assert binding.workspace_bytes(binding.config_from_workload(WORKLOADS["c1"])) > 0
assert binding.attention_scratch_bytes(4, 32) == 512
for call in (lambda: binding.rotary(None), lambda: binding.checkpoint_store(None), lambda: binding.attention_forward(None, None, None)):
    try:
        call()
    except ImportError as e:
        assert "_calls.so" in str(e)
    else:
        raise AssertionError
"""
    subprocess.run([sys.executable, "-c", program], cwd=tmp_path, check=True, env={**os.environ, "PYTHONPATH": str(tmp_path)}, timeout=300)


def test_another_torch_or_python_makes_it_stale(build, monkeypatch):
    assert not build._stale()
    monkeypatch.setattr(build.importlib.metadata, "version", lambda name: "0.0")
    assert build._stale()
    monkeypatch.undo()
    monkeypatch.setattr(build.sys, "version", "0.0")
    assert build._stale()
    monkeypatch.undo()
    monkeypatch.setattr(build, "CALLS_FOR", build.CALLS_FOR + ".none")
    assert build._stale()
