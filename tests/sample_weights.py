"""The fixed-point weights of sampling, as its kernels make them from a difference of logits, and rows built from them whose sums lie where they should."""
from fractions import Fraction

import numpy as np

LOG2E, LN2, SQRT_HALF = 1.44269504088896340736, 0.69314718055994530942, 0.70710678118654752440
SERIES = [1 / 39916800, 1 / 3628800, 1 / 362880, 1 / 40320, 1 / 5040, 1 / 720, 1 / 120, 1 / 24, 1 / 6, 0.5, 1.0, 1.0]


def fma(a, b, c):
    return float(Fraction(a) * Fraction(b) + Fraction(c))       # a fraction becomes the nearest double


def weight(below):
    """round(2^43 exp(-below)) at temperature 1, operation by operation."""
    y = min(below * LOG2E, 46.0)
    n = float(np.floor(y))
    z = (0.5 - (y - n)) * LN2
    p = SERIES[0]
    for c in SERIES[1:]:
        p = fma(p, z, c)
    return int(fma(p, 2.0 ** (43 - int(n)) * SQRT_HALF, 2.0 ** 52)) - (1 << 52)
