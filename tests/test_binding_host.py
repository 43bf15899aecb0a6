"""What the binding needs of its surroundings, on the host."""
import os
import subprocess
import sys
import warnings

import pytest

from paper_1707_04585_b200 import binding as B
from paper_1707_04585_b200 import build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_planning_needs_no_torch():
    """Everything in front of a launch works without torch, as on a machine that only plans."""
    code = """
import sys
sys.modules["torch"] = None
from paper_1707_04585_b200 import binding as B
c = B.Context(-1)
n = B.revnet_act_ckpt_bytes(c, 65, 100)
assert n == B._ck_bytes(65, 100), n
assert B.revnet_rmsnorm_workspace_bytes(c, B.norm_desc(100, 64)) > 0 and B.revnet_linear_wgrad_workspace_bytes(c, B.wgrad_desc(100, 64, 64)) > 0
assert B.revnet_transition_kept_bytes(c, B.TransitionDesc(2, 6, 6, 16, 24, 3, 2, 1, 1e-5, 0, 16))[0] > 0
c.close()
"""
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr


def test_the_library_is_built_where_the_module_of_direct_calls_cannot_be(monkeypatch, tmp_path, capfd):
    old = tmp_path / "_direct.so"
    monkeypatch.setattr(build, "DIRECT", str(old))
    for command in (["g++", "-c", str(tmp_path / "missing.cpp")], [str(tmp_path / "no-such-compiler")]):
        old.write_bytes(b"of an earlier source")
        monkeypatch.setattr(build, "_direct_command", lambda: command)
        assert build.build() == build.LIB            # (the library itself is up to date)
        assert not old.exists() and "_direct.so is not built" in capfd.readouterr().err


def test_the_module_of_direct_calls_goes_stale_with_torch(monkeypatch):
    build.build()
    assert not build._direct_stale()
    folder, version = build._torch()
    monkeypatch.setattr(build, "_torch", lambda: (folder, "9.9.9+cu000"))
    assert build._direct_stale()
    monkeypatch.setattr(build, "_torch", lambda: None)           # nothing to build it against
    assert not build._direct_stale() and build._direct_command() is None


def test_a_module_of_other_versions_is_not_used_and_says_so(monkeypatch, tmp_path):
    import torch
    assert B._find_direct(torch.__version__).built_for == build.versions(torch.__version__)
    with pytest.warns(RuntimeWarning, match="built for torch"):
        assert B._find_direct("9.9.9") is None
    monkeypatch.setitem(sys.modules, "paper_1707_04585_b200._direct", None)      # an import that fails
    monkeypatch.delattr("paper_1707_04585_b200._direct", raising=False)
    with pytest.warns(RuntimeWarning, match="not used"):
        assert B._find_direct(torch.__version__) is None
    monkeypatch.setattr(build, "DIRECT", str(tmp_path / "none.so"))
    with warnings.catch_warnings():
        warnings.simplefilter("error")
        assert B._find_direct(torch.__version__) is None         # none was built: no warning
