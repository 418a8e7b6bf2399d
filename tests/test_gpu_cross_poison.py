"""The norm and rotation at given positions and cross attention on the LDS-poison build
(GPU): every workgroup first fills its LDS with NaN bit patterns, so a read before the
write that it depends on (a copy not waited for, a missing barrier) shows in the results.

The operators' own tests run on it, once, in a child process (the binding loads one
library per process)."""
import os
import subprocess
import sys

import pytest

from paper_2609_35110_amd import build as pkg_build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CASES = ["tests/test_gpu_norm_rope.py", "tests/test_gpu_cross_attn.py", "tests/test_gpu_cross_tiles.py",
         "tests/test_gpu_cross_grads.py", "tests/test_gpu_cross_run.py"]


@pytest.mark.gpu
def test_operators_on_the_lds_poison_build():
    lib = pkg_build.POISON_LIB
    if not os.path.exists(lib):
        pytest.fail("libsol_poison.so is not built; run __graft_entry__.build()")
    code = ("import sys, pytest\n"
            "from paper_2609_35110_amd import sol\n"
            "sol.LIB_PATH = %r\n"
            "rc = pytest.main(%r + ['-v', '-x', '-p', 'no:cacheprovider', '-m', 'gpu', '--timeout', '120',"
            " '--timeout-method', 'thread'])\n"
            "print('library loaded:', sol.lib()._name)\n"
            "sys.exit(rc)\n" % (lib, CASES))
    print("poison build: %d files" % len(CASES), flush=True)
    res = subprocess.run([sys.executable, "-u", "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=110)
    out = res.stdout + res.stderr
    print(out[-500:], flush=True)
    assert res.returncode == 0, "the operators failed on the LDS-poison build:\n" + out[-6000:]
    assert "library loaded: " + lib in out
