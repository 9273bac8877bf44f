"""How calls over quantised caches are cut up, on the host.  No GPU."""
import os
import shutil
import subprocess

import pytest

from paper_2508_17892_amd import build as hip_build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CUS = 256

pytestmark = pytest.mark.skipif(shutil.which("hipcc") is None, reason="hipcc not on PATH")


@pytest.fixture(scope="module")
def plans():
    out = os.path.join(ROOT, "_build", "sanitize")
    os.makedirs(out, exist_ok=True)
    exe = os.path.join(out, "attn_plan_driver")
    if not os.path.exists(hip_build.LIB):
        hip_build.build()
    subprocess.run(["hipcc", *hip_build.FLAGS, "-o", exe, os.path.join(ROOT, "tests", "sanitize", "attn_plan_driver.hip"), "-L" + hip_build.HERE, "-l:libilre.so",
                    "-Wl,-rpath," + hip_build.HERE], check=True, capture_output=True)

    def run(calls):
        """(rows, tokens of a tile, ranges, tiles of a range) of every call, and the microseconds a plan took."""
        text = "".join(" ".join(map(str, c)) + "\n" for c in calls)
        got = subprocess.run([exe], input=text, capture_output=True, text=True, timeout=300, check=True).stdout.split("\n")[:-1]
        assert len(got) == len(calls) + 1
        return [tuple(map(int, line.split())) for line in got[:-1]], float(got[-1])

    return run


def skewed():
    """One new token for each of many requests, of which few have long contexts."""
    for n in (40, 100, 128, 129, 192, 300, 512, 1024, 4096):
        for longest in (9000, 32768, 131072, 1000003):
            for rest in (1, 300, 1000):
                for Hq, Hkv in ((32, 8), (28, 4), (8, 2), (16, 16)):
                    yield n, longest, rest, Hq, Hkv


@pytest.mark.parametrize("fmt", [1, 2])
@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("beside", [0, 1])
def test_no_range_is_much_longer_than_a_compute_units_share(plans, fmt, dtype, beside):
    """However many requests there are beside it, a long context is cut: no workgroup walks more tiles than stay whole, five or a compute unit's share of all and what a merge costs, but where 256 ranges or
    the workgroups of a launch do not go further."""
    cases = list(skewed())
    got, _ = plans([(fmt, 0, dtype, n, n, Hq, Hkv, 1, longest, longest + (n - 1) * rest, 0, 0, beside) for n, longest, rest, Hq, Hkv in cases])
    for (n, longest, rest, Hq, Hkv), (rows, tile, ranges, each) in zip(cases, got):
        heads = 128 // tile  # kv heads a workgroup
        share = (-(-longest // tile) + (n - 1) * -(-rest // tile)) * Hkv / heads / CUS
        assert rows == 16
        # (twice: the library knows the sum of the lengths, of which each list's last tile may be a part)
        assert each <= max(2 * max(share + 4, 5), -(-longest // tile) / 256 + 1), (n, longest, rest, Hq, Hkv, ranges, each, share)


def test_the_gpu_tests_have_a_long_context_that_is_cut(plans):
    import test_gpu_quant_cache_long as gpu

    kv = gpu.uneven(0)
    got, _ = plans([(fmt, 0, dtype, len(kv), len(kv), 8, 8, 1, max(kv), sum(kv), 0, 0, beside) for fmt in (1, 2) for dtype in (0, 1) for beside in (0, 1)])
    assert all(rows == 16 and ranges > 4 for rows, _, ranges, _ in got), got


def test_the_gpu_tests_reach_every_kernel_of_fill_and_read(plans):
    """A fill kernel is one for the states' type, the cache's, where the other channel of a pair is, and how many wavefronts share a token; a read kernel for the types and how many rows a lane has."""
    import test_gpu_quant_cache_long as long

    def kernels(tokens, rows):
        got = subprocess.run([os.path.join(ROOT, "_build", "sanitize", "attn_plan_driver"), "fill"], input="".join(f"{t} {r}\n" for t, r in zip(tokens, rows)),
                             capture_output=True, text=True, timeout=60, check=True).stdout
        return [tuple(map(int, line.split())) for line in got.split("\n")[:-1]]

    types = [(dtype, fmt) for dtype in ("bf16", "f32") for fmt in ("plain", "fp8", "fp4")]
    where = lambda pairing, rotary: "next" if pairing == "interleaved" else "lane" if rotary == 128 else "elsewhere"  # noqa: E731
    calls = [(dtype, fmt, where(pairing, rotary), sum(long.FILL_SHAPES[shape][0])) for shape, dtype, fmt, pairing, rotary in long.FILL_CALLS]
    reached = {(*c[:3], n) for c, (n, _) in zip(calls, kernels([c[3] for c in calls], [1] * len(calls)))}
    assert not {(*t, w, n) for t in types for w in ("lane", "elsewhere", "next") for n in (8, 4, 1)} - reached
    assert [n for n, _ in kernels([512, 513, 4095, 4096], [1] * 4)] == [8, 4, 4, 1] and {512, 513, 4095, 4096} <= {c[3] for c in calls}
    heads = {(long.FILL_SHAPES[shape][2], long.FILL_SHAPES[shape][3]) for shape, *_ in long.FILL_CALLS}
    assert {(28, 4), (32, 8), (64, 8)} <= heads  # several steps of eight query heads, a last one that is not full, and more than a token's wavefronts
    calls = [(dtype, fmt, sum(long.READ_ROWS[r][1]) * long.READ_ROWS[r][2]) for r, fmt, dtype in long.READS]
    reached = {(dtype, fmt) for (dtype, fmt, _), (_, n) in zip(calls, kernels([1] * len(calls), [c[2] for c in calls])) if n == 4}
    assert reached == set(types)
    assert kernels([1] * 3, [777 * 2, 1 << 18, (1 << 18) + 1]) == [(8, 1), (8, 1), (8, 4)]  # (the other reads of the tests: one row a lane)


def test_a_plan_takes_no_time(plans):
    """(A search tile by tile took 27 us for a million tokens, 55 ms for two thousand million.)"""
    calls = [(1, 0, 1, 128, 128, 32, 8, 1, longest, longest + 127 * 1000, 0, 0, 0) for longest in (1000003, 100000000, 2000000000)] * 20
    _, us = plans(calls)
    assert us < 100, us
