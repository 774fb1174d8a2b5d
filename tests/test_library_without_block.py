"""A library without the gated recurrence and the norm serves the scan; a call of theirs raises (host only: a library of stubs,
in a process of its own, since a process binds one library)."""
import os
import re
import subprocess
import sys

import pytest

from paper_2312_00752_b200 import binding as K

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SCRIPT = """
import ctypes, torch
from paper_2312_00752_b200 import binding as K
lib = K.load_library()
assert K.status_string(0) == "stub" and K.checkpoint_steps() == 7
assert K.fwd_workspace_bytes(K.ssm_problem_t(2, 100, 64, 16, K.SSM_BF16, 3)) == 7
K._native()
x, v = torch.zeros(2, 3, 4), torch.zeros(4)
calls = {"gated": [lambda: K.ssm_gated_fwd(x, x), lambda: K.ssm_gated_bwd(x, x, None, None, x), lambda: K.ssm_gated_step(x[0], x[0], None, None, x[0])],
         "norm": [lambda: K.ssm_norm_fwd(x, v), lambda: K.ssm_norm_bwd(x, v, x, x)]}
for call in calls["gated"] + calls["norm"]:
    try:
        call()
    except K.SsmScanError as e:
        assert "the library has no gated recurrence and norm" in str(e), e
    else:
        raise AssertionError("not refused")
print("served")
"""


def _stubs(path, names):
    source = path.with_suffix(".c")
    source.write_text("".join(f'const char* {n}(int c) {{ return "stub"; }}\n' if n == "ssm_status_string" else
                              f"unsigned long {n}(void) {{ return 7; }}\n" for n in names))
    subprocess.run(["gcc", "-shared", "-fPIC", "-o", str(path), str(source)], check=True)
    return path


@pytest.mark.parametrize("kept", [lambda n: not n.startswith(("ssm_gated", "ssm_norm")), lambda n: not n.startswith("ssm_norm")])
def test_the_scan_is_served_and_the_block_refused(tmp_path, kept):
    lib = _stubs(tmp_path / "libstub.so", [n for n in K.EXPORTED_SYMBOLS if kept(n)])
    run = subprocess.run([sys.executable, "-c", SCRIPT], cwd=ROOT, capture_output=True, text=True,
                         env={**os.environ, "SSM_SCAN_LIBRARY": str(lib)})
    assert run.returncode == 0 and "served" in run.stdout, run.stderr


def test_a_library_without_the_scan_is_not_taken(tmp_path):
    lib = _stubs(tmp_path / "libstub.so", [n for n in K.EXPORTED_SYMBOLS if n != "ssm_scan_fwd"])
    run = subprocess.run([sys.executable, "-c", "from paper_2312_00752_b200 import binding as K; K.load_library()"], cwd=ROOT,
                         capture_output=True, text=True, env={**os.environ, "SSM_SCAN_LIBRARY": str(lib)})
    assert run.returncode != 0 and re.search(r"undefined symbol: ssm_scan_fwd\b", run.stderr)
