"""The units of attention over quantised caches and under drafted trees on the host: every range of every block has one workgroup.  No GPU."""
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
    exe = os.path.join(out, "attn_codes_driver")
    if not os.path.exists(hip_build.LIB):
        hip_build.build()
    subprocess.run(["hipcc", *hip_build.FLAGS, "-Xarch_host", "-fsanitize=undefined", "-Xarch_host", "-fno-sanitize-recover=all", "-fno-gpu-sanitize",
                    "-o", exe, os.path.join(ROOT, "tests", "sanitize", "attn_codes_driver.hip"), "-L" + hip_build.HERE, "-l:libilre.so", "-Wl,-rpath," + hip_build.HERE,
                    "-Xarch_host", "-fsanitize=undefined"], check=True, capture_output=True)
    return exe


def test_every_range_has_one_workgroup(driver):
    run = subprocess.run([driver], capture_output=True, text=True, timeout=300)
    assert run.returncode == 0 and " 0 failures" in run.stdout, (run.stdout[-3000:], run.stderr[-2000:])
    assert "runtime error" not in run.stderr, run.stderr[-2000:]


def test_the_gpu_tests_reach_every_kernel(driver):
    """Each kernel (rows of a workgroup), with and without a window, whole and cut into ranges; trees over every kind of cache."""
    import test_gpu_quant_cache as gpu

    code = {"f32": 0, "bf16": 1}
    calls = [("paged", f, dtype, q, kv, Hq, Hkv, mask, 0) for f in (1, 2) for q, kv, Hq, Hkv, _, _, dtype, mask in gpu.ATTENTION]
    calls += [("tree", f, dtype, q, kv, Hq, Hkv, {}, 0) for f in (0, 1, 2) for q, kv, Hq, Hkv, _, _, dtype in gpu.TREES]
    text = "".join(f"{f} {int(kind == 'tree')} {code[dtype]} {sum(q)} {len(q)} {Hq} {Hkv} {max(q)} {max(kv)} {sum(kv)} {mask.get('sink', 0)} {mask.get('window', 0)} {beside}\n"
                   for kind, f, dtype, q, kv, Hq, Hkv, mask, beside in calls)
    run = subprocess.run([driver, "plan"], input=text, capture_output=True, text=True, timeout=60)
    lines = run.stdout.split("\n")[:-1]
    assert run.returncode == 0 and len(lines) == len(calls)
    reached = set()
    for (kind, f, dtype, *_, mask, _), line in zip(calls, lines):
        rows, nsplit, _ = map(int, line.split())
        reached |= {(kind, f, dtype, rows, "window" if mask.get("window") else "whole"), (kind, f, dtype, rows, "cut" if nsplit > 1 else "not cut")}
    wanted = {("paged", f, dtype, rows, how) for f in (1, 2) for dtype, rows in (("bf16", 16), ("bf16", 32), ("bf16", 128), ("bf16", 256), ("f32", 16))
              for how in ("window", "whole", "cut", "not cut")}
    wanted |= {("tree", 0, dtype, rows, how) for dtype, rows in (("bf16", 32), ("bf16", 128), ("bf16", 256), ("f32", 32), ("f32", 128)) for how in ("cut", "not cut")}
    wanted |= {("tree", f, dtype, rows, how) for f in (1, 2) for dtype, rows in (("bf16", 16), ("bf16", 32), ("bf16", 128), ("bf16", 256), ("f32", 16)) for how in ("cut", "not cut")}
    assert not wanted - reached, sorted(wanted - reached)


def test_the_gpu_tests_reach_several_heads_a_workgroup(driver):
    import test_gpu_quant_cache as gpu

    text = "".join(f"{f} 0 1 {sum(q)} {len(q)} {Hq} {Hkv} {max(q)} {most} {total} {mask.get('sink', 0)} {mask.get('window', 0)} 1\n" for f, q, _, Hq, Hkv, _, mask, most, total, _ in gpu.BESIDE)
    run = subprocess.run([driver, "plan"], input=text, capture_output=True, text=True, timeout=60)
    got = [tuple(map(int, line.split())) for line in run.stdout.split("\n")[:-1]]
    assert [(16, heads) for *_, heads in gpu.BESIDE] == [(rows, heads) for rows, _, heads in got]
    assert {(f, heads, nsplit > 1) for (f, *_), (_, nsplit, heads) in zip(gpu.BESIDE, got)} == {(1, 2, True), (1, 2, False), (1, 4, True), (1, 4, False), (2, 4, True), (2, 4, False)}
