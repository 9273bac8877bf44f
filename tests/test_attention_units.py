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


def test_the_gpu_tests_reach_every_kind_of_block(driver):
    """Each kernel (rows of a workgroup), for pages and for prompts, with and without a window, whole and cut into ranges."""
    import test_gpu_attention as whole
    import test_gpu_attention_blocks as blocks

    code = {"f32": 0, "bf16": 1}
    calls = [("paged", dtype, q, kv, Hq, Hkv, mask) for q, kv, Hq, Hkv, _, _, dtype, mask in whole.CASES + blocks.CHUNKS]
    calls += [("paged", dtype, q, kv, Hq, Hkv, dict(sink=sink, window=window)) for q, kv, Hq, Hkv, dtype, sink, window in blocks.STREAMS]
    calls += [("prompt", dtype, q, kv or q, Hq, Hkv, mask) for q, kv, Hq, Hkv, dtype, mask in whole.PROMPTS]
    calls += [("prompt", dtype, q, q, Hq, Hkv, mask) for q, Hq, Hkv, dtype, mask in blocks.PROMPTS]
    calls += [("prompt", dtype, q, q, Hq, Hkv, dict(sink=sink, window=window)) for q, Hq, Hkv, dtype, sink, window in blocks.PACKED]
    text = "".join(f"{code[dtype]} {sum(q)} {len(q)} {Hq} {Hkv} {max(q)} {max(kv)} {sum(kv)} {mask.get('sink', 0)} {mask.get('window', 0)}\n"
                   for _, dtype, q, kv, Hq, Hkv, mask in calls)
    run = subprocess.run([driver, "plan"], input=text, capture_output=True, text=True, timeout=60)
    lines = run.stdout.split("\n")[:-1]
    assert run.returncode == 0 and len(lines) == len(calls)
    reached = set()
    for (kind, dtype, *_, mask), line in zip(calls, lines):
        rows, nsplit = map(int, line.split())
        reached |= {(kind, dtype, rows, "window" if mask.get("window") else "whole"), (kind, dtype, rows, "cut" if nsplit > 1 else "not cut")}
    wanted = {(kind, dtype, rows, how) for kind in ("paged", "prompt") for dtype, rows in (("bf16", 128), ("bf16", 256), ("f32", 128))
              for how in ("window", "whole", "cut", "not cut")}
    wanted |= {(kind, dtype, 32, "whole") for kind in ("paged", "prompt") for dtype in ("bf16", "f32")}
    assert not wanted - reached, sorted(wanted - reached)
