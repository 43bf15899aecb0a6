"""What the binding needs of its surroundings, on the host."""
import os
import subprocess
import sys

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
