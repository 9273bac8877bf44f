"""The attention kernels' units on the host: every range of every block has one workgroup.  No GPU."""
import os
import shutil
import subprocess

import pytest

from paper_2508_17892_amd import build as hip_build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

pytestmark = pytest.mark.skipif(shutil.which("hipcc") is None, reason="hipcc not on PATH")


@pytest.fixture(scope="module")
def driver():
    out = os.path.join(ROOT, "_build", "sanitize")
    os.makedirs(out, exist_ok=True)
    exe = os.path.join(out, "attn_units_driver")
    if not os.path.exists(hip_build.LIB):
        hip_build.build()
    subprocess.run(["hipcc", *hip_build.FLAGS, "-Xarch_host", "-fsanitize=undefined", "-Xarch_host", "-fno-sanitize-recover=all", "-fno-gpu-sanitize",
                    "-o", exe, os.path.join(ROOT, "tests", "sanitize", "attn_units_driver.hip"), "-L" + hip_build.HERE, "-l:libilre.so", "-Wl,-rpath," + hip_build.HERE,
                    "-Xarch_host", "-fsanitize=undefined"], check=True, capture_output=True)
    return exe


def test_every_range_has_one_workgroup(driver):
    run = subprocess.run([driver], capture_output=True, text=True, timeout=300)
    assert run.returncode == 0 and " 0 failures" in run.stdout, (run.stdout[-3000:], run.stderr[-2000:])
    assert "runtime error" not in run.stderr, run.stderr[-2000:]
