"""Caches of 8- and 4-bit codes with a scale for every 32 channels, norms of heads, positions along axes and attention under any mask, in fp64 from their
definitions.  numpy only."""
from __future__ import annotations

import numpy as np

BLOCK = 32


def code_values(fmt):
    """The numbers that the codes 0, 1, ... stand for, sign bit included (fp8: 256 of them, two NaN)."""
    if fmt == "fp4":
        half = [m * 0.5 if e == 0 else (1 + m / 2) * 2.0 ** (e - 1) for e in range(4) for m in range(2)]
    else:
        half = [m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7) for e in range(16) for m in range(8)]
        half[-1] = np.nan
    return np.array(half + [-x for x in half])


def read(codes, scales, fmt):
    """codes uint8 [..., 128] (fp8) or [..., 64] (fp4), scales uint8 [..., 4] -> numbers [..., 128]; scale byte 255 is NaN."""
    if fmt == "fp4":
        codes = np.stack((codes & 15, codes >> 4), -1).reshape(*codes.shape[:-1], 128)
    scale = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return code_values(fmt)[codes] * np.repeat(scale, BLOCK, axis=-1)


def store(x, fmt):
    """What a cache holds for x fp64 [..., 128]: (codes, scales).  The scale is the smallest power of two from 2^-126 on that brings the block's largest magnitude down to
    the largest code; the code the nearest one, the even one of two."""
    half = code_values(fmt)[:128 if fmt == "fp8" else 8]
    half = half[~np.isnan(half)]
    y = np.asarray(x, np.float64).reshape(*x.shape[:-1], x.shape[-1] // BLOCK, BLOCK)
    bad = ~np.isfinite(y).all(-1)
    y = np.where(bad[..., None], 0.0, y)
    top = np.abs(y).max(-1)
    powers = 2.0 ** np.arange(-126.0, 128)
    e = np.searchsorted(half[-1] * powers, top)  # the first power that is large enough
    t = np.abs(y) / powers[e][..., None]
    above = np.minimum(np.searchsorted(half, t), len(half) - 1)
    below = np.maximum(above - 1, 0)
    up, down = half[above] - t, t - half[below]
    code = np.where((up < down) | ((up == down) & (above % 2 == 0)), above, below)
    code = np.where(np.signbit(y) & ~bad[..., None], code + (128 if fmt == "fp8" else 8), code).astype(np.uint8).reshape(x.shape)
    scales = np.where(bad, 255, e + 1).astype(np.uint8)
    return (code if fmt == "fp8" else code[..., 0::2] | (code[..., 1::2] << 4)), scales


def norm(x, weight, eps, offset=0.0):
    x = np.asarray(x, np.float64)
    w = 1.0 if weight is None else np.asarray(weight, np.float64) + offset
    return x / np.sqrt((x ** 2).mean(-1, keepdims=True) + eps) * w


def angle(positions, inv_freq):
    """(cosine, sine) in fp64 of the products positions * inv_freq as they are, not rounded to fp64: at position 2^30 that would be 2^-24 of an angle's turn.  Each product in two parts, exact in a float of
    64 bits: positions of 31 bits times the upper 32 and the lower 21 of a frequency."""
    assert np.finfo(np.longdouble).nmant >= 63
    p, f = np.asarray(positions, np.longdouble), np.asarray(inv_freq, np.float64)
    assert (np.abs(p) <= 2 ** 31).all()
    c = f * (2.0 ** 21 + 1)
    upper = c - (c - f)
    a, b = p * upper.astype(np.longdouble), p * (f - upper).astype(np.longdouble)
    return tuple(x.astype(np.float64) for x in (np.cos(a) * np.cos(b) - np.sin(a) * np.sin(b), np.sin(a) * np.cos(b) + np.cos(a) * np.sin(b)))


def rope_axes(x, positions, axes, inv_freq, magnitude=1.0, pairing="half"):
    """x [T, H, d] turned, pair j by positions[axes[j]] (positions [number of axes, T])."""
    y = np.array(x, dtype=np.float64)
    r = 2 * len(inv_freq)
    cos, sin = (t[:, None, :] for t in angle(np.asarray(positions)[list(axes)].T, inv_freq))
    first = slice(0, r // 2) if pairing == "half" else slice(0, r, 2)
    second = slice(r // 2, r) if pairing == "half" else slice(1, r, 2)
    u, w = np.array(y[..., first]), np.array(y[..., second])
    y[..., first] = magnitude * (u * cos - w * sin)
    y[..., second] = magnitude * (w * cos + u * sin)
    return y


def tree_seen(words, n, m):
    """bool [n, m]: which of a sequence's m tokens its last n, the drafted ones, see; words uint32 [n, words]."""
    seen = np.zeros((n, m), bool)
    for i in range(n):
        for t in range(m):
            j = t - (m - n)
            seen[i, t] = j < 0 or (j < 32 * words.shape[1] and int(words[i, j // 32]) >> (j % 32) & 1 == 1)
    return seen


def attend_seen(q, k, v, seen, scale=None):
    """attention.attend's results for the mask seen [n, m]."""
    n, Hq, d = q.shape
    m, Hkv, _ = k.shape
    scale = 1.0 / np.sqrt(d) if scale is None else scale
    out, size = np.zeros((n, Hq, d)), np.zeros((n, Hq, d))
    lse, reach = np.full((n, Hq), -np.inf), np.zeros((n, Hq))
    for i in range(n):
        at = np.flatnonzero(seen[i])
        if not len(at):
            continue
        for h in range(Hq):
            kh, vh = k[at, h // (Hq // Hkv)], v[at, h // (Hq // Hkv)]
            x = kh @ q[i, h] * scale
            top = x.max()
            w = np.exp(x - top)
            lse[i, h] = top + np.log(w.sum())
            w /= w.sum()
            out[i, h], size[i, h] = w @ vh, w @ np.abs(vh)
            reach[i, h] = (np.abs(kh) @ np.abs(q[i, h]) * scale).max()
    return out, lse, size, reach
