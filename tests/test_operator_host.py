"""Rotary positions, chunk attention and sampling without a GPU: their planning and
checks under AddressSanitizer and UndefinedBehaviorSanitizer
(tests/host/operators_check.cpp), and their kernels' registers from the compiler's
remarks (no kernel may spill a vector register)."""

import os
import shutil
import subprocess

import pytest

from test_kernel_resources import HIPCC, spills

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2606_02544_amd", "csrc")


@pytest.mark.skipif(shutil.which("g++") is None, reason="g++ not available")
def test_planning_under_sanitizers(tmp_path):
    exe = str(tmp_path / "operators_check")
    cmd = ["g++", "-std=c++17", "-O1", "-g", "-fno-omit-frame-pointer",
           "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
           "-I" + os.path.join(ROOT, "include"), "-I" + CSRC,
           os.path.join(CSRC, "simsd_plan.cpp"), os.path.join(CSRC, "simsd_ops_plan.cpp"),
           os.path.join(ROOT, "tests", "host", "operators_check.cpp"), "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stdout + r.stderr
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:verify_asan_link_order=0",
               UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    r = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=600)
    assert r.returncode == 0, r.stdout + r.stderr
    assert ", 0 failed" in r.stdout, r.stdout + r.stderr


@pytest.mark.skipif(not os.path.exists(HIPCC) and shutil.which("hipcc") is None, reason="hipcc not available")
@pytest.mark.parametrize("source", ["simsd_rotary.hip", "simsd_chunk.hip", "simsd_sample.hip"])
def test_no_vgpr_spills(source):
    found = spills(source)
    assert found, "no kernel resource remarks parsed"
    assert not [(name, n) for name, n in found.items() if n]
