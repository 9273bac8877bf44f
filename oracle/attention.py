"""Rotary positions and masked attention in fp64, written from their formulas, one row at a time where that is the definition.  numpy only; a sequence's keys
and values come as plain arrays, so that the tests keep the paging to themselves."""
from __future__ import annotations

import numpy as np


def sees(p, t, kv_len, causal=True, sink=0, window=0):
    """Whether the row at position p sees token t."""
    return (t < kv_len) & ((t <= p) | (not causal)) & ((window == 0) | (t > p - window) | (t < sink))


def attend(q, k, v, *, causal=True, sink=0, window=0, scale=None, absent=None):
    """q [n, Hq, d], k and v [m, Hkv, d] fp64; the last of the n rows stands at token m - 1.  absent: bool [m], tokens that are not there.
    Returns out [n, Hq, d], lse [n, Hq] (-inf and zeros for rows that see nothing), and what a tolerance is made of: sum_t p |v| [n, Hq, d],
    and the largest sum_i |q_i k_ti| scale of a row [n, Hq]."""
    n, Hq, d = q.shape
    m, Hkv, _ = k.shape
    scale = 1.0 / np.sqrt(d) if scale is None else scale
    out, size = np.zeros((n, Hq, d)), np.zeros((n, Hq, d))
    lse, reach = np.full((n, Hq), -np.inf), np.zeros((n, Hq))
    if n == 0 or m == 0:
        return out, lse, size, reach
    p, t = m - n + np.arange(n)[:, None], np.arange(m)[None, :]
    seen = sees(p, t, m, causal, sink, window)
    if absent is not None:
        seen = seen & ~absent[None, :]
    some = seen.any(1)
    used = seen.any(0)
    for h in range(Hq):
        kh, vh = np.where(used[:, None], k[:, h // (Hq // Hkv)], 0.0), np.where(used[:, None], v[:, h // (Hq // Hkv)], 0.0)
        x = np.where(seen, q[:, h] @ kh.T * scale, -np.inf)
        top = np.where(some, x.max(1, initial=-np.inf), 0.0)
        w = np.exp(x - top[:, None])
        total = w.sum(1)
        w = w / np.where(some, total, 1.0)[:, None]
        out[:, h], size[:, h] = w @ vh, w @ np.abs(vh)
        lse[some, h] = top[some] + np.log(total[some])
        reach[:, h] = (np.abs(q[:, h]) @ np.abs(kh).T * scale).max(1, initial=0.0)
    return out, lse, size, reach


def frequencies(rotary, base, scaling="plain", factor=1.0, low=1.0, high=4.0, original_len=0):
    """(inv_freq [rotary / 2], magnitude) of the four kinds of scaling."""
    f = base ** (-np.arange(0, rotary, 2, dtype=np.float64) / rotary)
    if scaling == "linear":
        return f / factor, 1.0
    if scaling == "bands":
        wavelength = 2 * np.pi / f
        mixed = (original_len / wavelength - low) / (high - low)
        return np.where(wavelength <= original_len / high, f, np.where(wavelength >= original_len / low, f / factor, mixed * f + (1 - mixed) * f / factor)), 1.0
    if scaling == "parts":
        def number(turns):  # of the pair that makes so many turns
            return rotary / 2 * np.log(original_len / (2 * np.pi * turns)) / np.log(base)
        a, b = max(np.floor(number(high)), 0), min(np.ceil(number(low)), rotary - 1)
        r = np.clip((np.arange(rotary // 2) - a) / max(b - a, 1e-3), 0, 1)
        return (1 - r) * f + r * f / factor, 1 + 0.1 * np.log(factor)
    return f, 1.0


def rope(x, positions, inv_freq, magnitude=1.0, pairing="half"):
    """x [T, H, d] fp64 turned by positions [T]; the channels behind 2 len(inv_freq) as they are."""
    y = np.array(x, dtype=np.float64)
    r = 2 * len(inv_freq)
    a = np.asarray(positions, dtype=np.float64)[:, None, None] * np.asarray(inv_freq)[None, None, :]
    first = slice(0, r // 2) if pairing == "half" else slice(0, r, 2)
    second = slice(r // 2, r) if pairing == "half" else slice(1, r, 2)
    u, w = x[..., first].astype(np.float64), x[..., second].astype(np.float64)
    y[..., first] = magnitude * (u * np.cos(a) - w * np.sin(a))
    y[..., second] = magnitude * (w * np.cos(a) + u * np.sin(a))
    return y
