"""The build and the loading of the paged cache's calls: the library needs neither torch nor Python's headers, and a module
for another torch is refused before a tensor is looked into."""
import os
import subprocess
import sys

import pytest
import torch

from paper_2509_09754_b200 import build as B
from paper_2509_09754_b200 import paged as P


def test_the_library_is_built_where_torch_is_not():
    B.build_library()                                                      # (what is up to date is not compiled again)
    code = "import runpy, sys; sys.argv = ['build.py']; runpy.run_path(%r, run_name='__main__')" % B.__file__
    r = subprocess.run([sys.executable, "-I", "-S", "-c", "import importlib.util as u; assert u.find_spec('torch') is None\n"
                        + code], capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stderr
    assert r.stdout.strip().endswith("liblava.so") and "torch" in r.stderr


def test_what_the_calls_need_is_named(monkeypatch):
    assert B.missing_for_calls() == []
    monkeypatch.setattr(B.shutil, "which", lambda name: None)
    monkeypatch.setattr(B.sysconfig, "get_paths", lambda: {"include": "/nowhere"})
    assert B.missing_for_calls() == ["g++", "Python.h"]


def test_a_module_for_another_torch_is_refused(monkeypatch):
    assert P.load_paged_calls().torch_version == torch.__version__
    monkeypatch.setattr(P, "_CALLS", None)
    monkeypatch.setattr(torch, "__version__", "1.0")
    with pytest.raises(RuntimeError, match="built for torch .* this is torch 1.0"):
        P.load_paged_calls()
    assert P._CALLS is None


def test_a_module_that_does_not_load_is_refused(monkeypatch, tmp_path):
    (tmp_path / "_paged_calls.so").write_bytes(b"none")
    monkeypatch.setattr(P, "library_path", lambda: os.path.join(tmp_path, "liblava.so"))
    monkeypatch.setattr(P, "_CALLS", None)
    with pytest.raises(RuntimeError, match="built for another torch"):
        P.load_paged_calls()
