"""Pins of the oracle of quantised caches, head norms, positions along axes and drafted trees.  No GPU."""
import numpy as np
import pytest
import torch

from oracle import attention as oa
from oracle import quant_cache as oq


def test_codes_are_the_formats_numbers():
    want = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    got = oq.code_values("fp8")
    assert np.array_equal(got, want, equal_nan=True) and np.nanmax(got) == 448 and np.isnan(got[[127, 255]]).all()
    assert oq.code_values("fp4").tolist() == [0, 0.5, 1, 1.5, 2, 3, 4, 6, 0, -0.5, -1, -1.5, -2, -3, -4, -6]


def test_rounding_is_the_librarys():
    """torch's conversion rounds to nearest, ties to even, too: on halves between all codes, next to them, and at random."""
    half = oq.code_values("fp8")[:127]
    mid = (half[1:] + half[:-1]) / 2
    x = np.concatenate([half, mid, np.nextafter(mid, 0), np.nextafter(mid, 500), np.random.default_rng(0).uniform(0, 448, 2000)])[:64 * 31]
    rows = np.concatenate([x.reshape(64, 31), np.full((64, 1), 448.0)], 1).reshape(16, 128)  # every block of 32 has a scale of one
    codes, scales = oq.store(rows, "fp8")
    assert (scales == 127).all()
    want = torch.tensor(rows).float().to(torch.float8_e4m3fn)  # (next to a half in fp64 is the half in fp32: those are left out)
    exact = rows.astype(np.float32).astype(np.float64) == rows
    assert (codes[exact] == want.view(torch.uint8).numpy()[exact]).all()
    up, down = np.nextafter(17.0, 100), np.nextafter(17.0, 0)  # 17 is halfway between 16 and 18
    row = np.full(128, 448.0)
    row[:6] = [17, up, down, 19, -17, -up]
    assert oq.read(*oq.store(row, "fp8"), "fp8")[:6].tolist() == [16, 18, 16, 20, -16, -18]


@pytest.mark.parametrize("fmt", ["fp8", "fp4"])
def test_store_by_hand(fmt):
    top = 6.0 if fmt == "fp4" else 448.0
    x = np.zeros((1, 128))
    x[0, 0] = top          # block 0: scale one
    x[0, 32] = top * 1.001  # block 1: one power more
    x[0, 64] = -top * 2.0 ** -130  # block 2: the least scale
    codes, scales = oq.store(x, fmt)
    assert scales.tolist() == [[127, 128, 1, 1]]
    back = oq.read(codes, scales, fmt)
    assert back[0, 0] == top and back[0, 32] == top and back[0, 96:].tolist() == [0] * 32
    assert back[0, 64] == {"fp8": -448 * 2.0 ** -130, "fp4": -0.5 * 2.0 ** -126}[fmt]  # 6 2^-130 is 0.375 2^-126: the nearest code is 0.5
    x[0, 5], x[0, 70] = np.inf, np.nan
    codes, scales = oq.store(x, fmt)
    assert scales.tolist() == [[255, 128, 255, 1]] and np.isnan(oq.read(codes, scales, fmt)[0, :32]).all()
    rng = np.random.default_rng(1)
    x = rng.normal(size=(50, 128)) * np.exp(rng.normal(size=(50, 1)) * 5)
    back = oq.read(*oq.store(x, fmt), fmt)
    # half a step: 2^-4 of a number, or of the least normal code (2^-6 of 448 and up) in its block; fp4: 2^-2, least normal code 1 of 6
    block = np.abs(x).reshape(50, 4, 32).max(-1).repeat(32, -1)
    rel, least = (2.0 ** -4, 2.0 ** -6 / 224) if fmt == "fp8" else (2.0 ** -2, 1 / 3)
    assert (np.abs(back - x) <= rel * np.maximum(np.abs(x), least * block)).all()
    again = oq.store(back, fmt)
    assert (oq.read(*again, fmt) == back).all()  # what is there already stays


def test_norm_and_axes():
    rng = np.random.default_rng(2)
    x = rng.normal(size=(5, 3, 128))
    y = oq.norm(x, None, 0.0)
    assert np.allclose((y ** 2).mean(-1), 1.0)
    w = rng.normal(size=128)
    assert np.allclose(oq.norm(x, w, 1e-6, 1.0), oq.norm(x, None, 1e-6) * (1 + w))
    f, m = oa.frequencies(64, 10000.0)
    pos = rng.integers(0, 1000, (3, 5))
    for pairing in ("half", "interleaved"):
        one = oq.rope_axes(x, pos[:1], [0] * 32, f, m, pairing)
        assert np.allclose(one, oa.rope(x, pos[0], f, m, pairing), atol=1e-12)
        axes = [j % 3 for j in range(32)]
        got = oq.rope_axes(x, pos, axes, f, m, pairing)
        for a in range(3):  # the pairs of an axis are as if it were the only one
            alone = oa.rope(x, pos[a], f, m, pairing)
            for j in range(a, 32, 3):
                at = [j, j + 32] if pairing == "half" else [2 * j, 2 * j + 1]
                assert np.allclose(got[..., at], alone[..., at], atol=1e-12)


def test_a_chain_of_drafted_tokens_is_causal_attention():
    rng = np.random.default_rng(3)
    n, m = 37, 50
    q, k, v = rng.normal(size=(n, 4, 16)), rng.normal(size=(m, 2, 16)), rng.normal(size=(m, 2, 16))
    words = np.array([[(((1 << (i + 1)) - 1) >> (32 * w)) & 0xFFFFFFFF for w in range(2)] for i in range(n)], dtype=np.uint32)
    got, want = oq.attend_seen(q, k, v, oq.tree_seen(words, n, m)), oa.attend(q, k, v)
    for a, b in zip(got[:3], want[:3]):
        assert np.allclose(a, b, atol=1e-12)
