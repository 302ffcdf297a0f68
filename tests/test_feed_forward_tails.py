"""The lower tail of GELU, g times the normal distribution function, where 1 + erf would cancel: relative to the value, however small it is."""
import math

import numpy as np

from oracle import feed_forward as F

TAIL = -np.arange(16.0, 97.0) / 8   # -2 to -12, bf16 numbers


def test_oracle_gelu_keeps_its_digits_in_the_lower_tail():
    """Against the integral of the density from g down, by Simpson's rule on exp(-t^2 / 2) / exp(-g^2 / 2): nothing there cancels."""
    t = np.linspace(0.0, 12.0, 24001)
    weights = np.where(np.arange(t.size) % 2 == 1, 4.0, 2.0)
    weights[[0, -1]] = 1.0
    for g in TAIL:
        density = math.exp(-g * g / 2) / math.sqrt(2 * math.pi)
        below = density * float((weights * np.exp(g * t - t * t / 2)).sum()) * (t[1] - t[0]) / 3
        value, slope = (float(v[0]) for v in F.activation(np.array([g]), "gelu"))
        assert abs(value - g * below) <= 1e-11 * abs(g * below), g
        assert abs(slope - (below + g * density)) <= 1e-11 * abs(slope), g
