"""The oracle's angles of far positions, against angles reduced in whole numbers.  No GPU."""
import math
from fractions import Fraction

import numpy as np

from oracle import quant_cache as oq


def _pi(bits):
    """pi * 2^bits, rounded down, by Machin's formula."""
    one = 1 << (bits + 20)

    def arctan_of_inverse(n):
        term, total, k = one // n, 0, 0
        while term:
            total += (term // (2 * k + 1)) * (-1) ** k
            term //= n * n
            k += 1
        return total

    return 4 * (4 * arctan_of_inverse(5) - arctan_of_inverse(239)) >> 20


def test_angles_of_far_positions():
    two_pi = Fraction(2 * _pi(300), 1 << 300)
    rng = np.random.default_rng(5)
    freqs = np.concatenate((500000.0 ** (-np.arange(0, 64, 5) / 64.0), [1.0, 0.75, 1 / 3, 1e-9]))
    for p in [0, 1, -1, 1000003, -999999, 2 ** 31 - 1, -2 ** 31] + rng.integers(-2 ** 31, 2 ** 31, 40).tolist():
        cos, sin = oq.angle(np.full(len(freqs), p), freqs)
        for f, c, s in zip(freqs.tolist(), cos, sin):
            a = p * Fraction(f)
            a -= round(a / two_pi) * two_pi
            assert abs(math.cos(float(a)) - c) <= 2.0 ** -51 and abs(math.sin(float(a)) - s) <= 2.0 ** -51, (p, f)
