"""The C library is built from nvcc's sources alone; the extension that reads torch's tensors is a build of its own, and
belongs to the interpreter and the torch that it was built with."""
import os
import subprocess
import sys

import pytest
import torch

from paper_2601_07396_b200 import binding as sc
from paper_2601_07396_b200 import build as sc_build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_the_library_does_not_wait_for_the_extension(monkeypatch):
    def refuse(*args, **kwargs):
        raise RuntimeError("no host compiler")
    monkeypatch.setattr(sc_build, "build_calls", refuse)
    assert sc_build.build() == sc_build.LIB and os.path.exists(sc_build.LIB)


def test_the_library_is_built_without_torch():
    """build.py by itself, in an interpreter that has no torch and no C++ compiler."""
    sc_build.build()
    code = ("import sys, importlib.util; sys.modules['torch'] = None\n"
            f"spec = importlib.util.spec_from_file_location('alone', {sc_build.__file__!r})\n"
            "m = importlib.util.module_from_spec(spec); spec.loader.exec_module(m)\n"
            "m.CALLS_SOURCE = m.__file__ + '.missing'; print(m.build())\n")
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, env=dict(os.environ, CXX="/bin/false"), timeout=300)
    assert r.returncode == 0 and r.stdout.strip().endswith("libsvdcache.so"), r.stdout + r.stderr


def test_an_extension_of_another_torch_is_not_loaded(monkeypatch):
    here = sc_build.build_calls()
    assert os.path.exists(here) and here == sc_build.calls_path()
    monkeypatch.setattr(torch, "__version__", "9.9.9")
    monkeypatch.setattr(sc, "_calls", None)
    assert sc_build.calls_path() != here
    with pytest.raises(RuntimeError, match="missing"):
        sc.calls()


def test_the_extension_loads_here(monkeypatch):
    sc_build.build_calls()
    monkeypatch.setattr(sc, "_calls", None)
    assert callable(sc.calls().gemm)
