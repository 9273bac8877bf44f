"""Pins of the fp64 attention and rotary oracle, the host-side frequency table, and the kernels' integer arithmetic on rows and tiles.  No GPU."""
import os
import shutil
import subprocess

import numpy as np
import pytest
import torch

import paper_2508_17892_amd as il
from oracle import attention as oa

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_attention_is_the_library_softmax_with_the_mask_written_out():
    rng = np.random.default_rng(0)
    for n, m, sink, window, causal in ((5, 9, 0, 0, True), (9, 9, 2, 3, True), (4, 4, 0, 1, True), (3, 8, 0, 0, False), (6, 4, 0, 0, True)):
        q, k, v = rng.normal(size=(n, 4, 8)), rng.normal(size=(m, 2, 8)), rng.normal(size=(m, 2, 8))
        out, lse, _, _ = oa.attend(q, k, v, causal=causal, sink=sink, window=window)
        for i in range(n):
            p = m - n + i
            seen = [t for t in range(m) if (not causal or t <= p) and (window == 0 or t > p - window or t < sink)]
            for h in range(4):
                if not seen:
                    assert lse[i, h] == -np.inf and (out[i, h] == 0).all()
                    continue
                x = torch.tensor(k[seen, h // 2] @ q[i, h] / np.sqrt(8))
                assert np.isclose(lse[i, h], torch.logsumexp(x, 0).item(), rtol=1e-13)
                assert np.allclose(out[i, h], (torch.softmax(x, 0).numpy()[:, None] * v[seen, h // 2]).sum(0), rtol=1e-12, atol=1e-14)


def test_rope_is_a_rotation_that_only_distances_matter_to():
    rng = np.random.default_rng(1)
    for pairing in ("half", "interleaved"):
        f, m = oa.frequencies(32, 10000.0)
        x, y = rng.normal(size=(1, 1, 48)), rng.normal(size=(1, 1, 48))
        a = oa.rope(x, [1000], f, m, pairing)
        assert np.isclose((a ** 2).sum(), (x ** 2).sum()) and (a[..., 32:] == x[..., 32:]).all()
        assert np.allclose(oa.rope(a, [-1000], f, m, pairing), x)
        dots = [(oa.rope(x, [p + 17], f, m, pairing) * oa.rope(y, [p], f, m, pairing)).sum() for p in (0, 5, 100003)]
        assert np.allclose(dots, dots[0], rtol=1e-9)
    # by hand: a quarter turn of pair 0
    assert np.allclose(oa.rope(np.array([[[1.0, 2.0, 3.0, 4.0]]]), [1], [np.pi / 2, 0.0], 1.0, "half"), [[[-3.0, 2.0, 1.0, 4.0]]])
    assert np.allclose(oa.rope(np.array([[[1.0, 2.0, 3.0, 4.0]]]), [1], [np.pi / 2, 0.0], 1.0, "interleaved"), [[[-2.0, 1.0, 3.0, 4.0]]])


@pytest.mark.parametrize("rotary", [16, 64, 96, 128])
@pytest.mark.parametrize("name,code,kw", [
    ("plain", il.ILRE_ROPE_PLAIN, {}),
    ("linear", il.ILRE_ROPE_LINEAR, dict(factor=4.0)),
    ("bands", il.ILRE_ROPE_BANDS, dict(factor=8.0, low=1.0, high=4.0, original_len=8192)),
    ("parts", il.ILRE_ROPE_PARTS, dict(factor=16.0, low=1.0, high=32.0, original_len=4096)),
])
@pytest.mark.parametrize("base", [10000.0, 500000.0])
def test_frequency_table(rotary, name, code, kw, base):
    want, magnitude = oa.frequencies(rotary, base, name, **kw)
    got = il.ilre_rope_frequencies(rotary, base, scaling=code, **kw)
    assert got.rotary == rotary and np.isclose(got.magnitude, magnitude, rtol=1e-15)
    assert np.allclose(np.array(got.inv_freq)[:rotary // 2], want, rtol=1e-13, atol=0)


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="hipcc not on PATH")
def test_rows_tiles_ranges_and_page_columns():
    from paper_2508_17892_amd import build as hip_build

    out = os.path.join(ROOT, "_build", "sanitize")
    os.makedirs(out, exist_ok=True)
    exe = os.path.join(out, "attn_blocks_driver")
    subprocess.run(["hipcc", *hip_build.FLAGS, "-Xarch_host", "-fsanitize=undefined", "-Xarch_host", "-fno-sanitize-recover=all", "-fno-gpu-sanitize",
                    "-o", exe, os.path.join(ROOT, "tests", "sanitize", "attn_blocks_driver.hip"), "-Xarch_host", "-fsanitize=undefined"],
                   check=True, capture_output=True)
    run = subprocess.run([exe], capture_output=True, text=True, timeout=120,
                         env=dict(os.environ, UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1"))
    assert run.returncode == 0 and ", 0 failures" in run.stdout, (run.stdout[-2000:], run.stderr[-2000:])
    assert "runtime error" not in run.stderr, run.stderr[-2000:]
