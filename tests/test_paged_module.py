"""The compiled module of the calls on pages: what is said where it is missing, and when it is built again."""

import importlib.util
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def run(code):
    return subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=300)


def test_the_package_without_the_module():
    """Layers are there; a call on pages says what is missing and how to build it."""
    r = run("""
import sys
sys.modules["paper_2410_01805_b200._paged"] = None   # (as a file that cannot be loaded)
import paper_2410_01805_b200 as P
assert P.LocretLayer and P.lib.locret_pages_step
for name in ("Pages", "pages_step", "norm_rope", "norm_rope_grad", "paged_attention", "rope_turns"):
    try:
        getattr(P, name)
    except ImportError as e:
        assert "build.py" in str(e) and "_paged" in str(e), e
    else:
        raise SystemExit(name)
try:
    P.no_such_name
except AttributeError:
    print("told")
""")
    assert r.returncode == 0 and r.stdout.strip() == "told", r.stderr[-2000:]


def _build():
    spec = importlib.util.spec_from_file_location("_locret_build_test", os.path.join(ROOT, "paper_2410_01805_b200", "build.py"))
    b = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(b)
    return b


@pytest.mark.parametrize("other", ["torch 1.0.0, cpython-312-x86_64-linux-gnu", "torch 2.11.0+cu128, cpython-399-x86_64-linux-gnu"])
def test_a_module_for_another_torch_or_python_is_built_again(other, monkeypatch):
    b = _build()
    assert not b.module_needs_build()   # (the tests' configuration has built it)
    monkeypatch.setattr(b, "built_for", lambda: other)
    assert b.module_needs_build()
    assert any(other in part for part in b.module_command())


def test_the_module_says_what_it_was_built_for():
    import torch
    from paper_2410_01805_b200 import _paged
    assert torch.__version__ in _paged.__doc__


def test_a_module_that_cannot_be_built_is_explained(monkeypatch, tmp_path):
    b = _build()
    monkeypatch.setattr(b, "needs_build", lambda: False)
    monkeypatch.setattr(b, "module_needs_build", lambda: True)
    for compiler in (str(tmp_path / "none"), "false"):   # not there, or failing
        monkeypatch.setenv("CXX", compiler)
        with pytest.raises(RuntimeError, match="g\\+\\+"):
            b.build()
