"""The oracle's weights of decided pairs, against exact rational arithmetic on the exponentials' values (CPU)."""
from fractions import Fraction
import math

import pytest

from oracle import preference


@pytest.mark.parametrize("smoothing", [0.0, 0.125, 1.0])
@pytest.mark.parametrize("z", [0.0, 3.0, -3.0, 20.0, -20.0, 40.0, -40.0, 100.0, -100.0])
def test_weights(z, smoothing):
    _, _, _, w, _ = preference.preference([[0.0], [0.0]], [0, 0], [0, 1, 2], [-z, 0.0], 1.0, smoothing, 1.0)
    e = Fraction(math.exp(-abs(z)))
    sigma = (1 if z >= 0 else e) / (1 + e)
    want = sigma - (1 - Fraction(smoothing))
    assert abs(Fraction(w[0]) - want) <= abs(want) * Fraction(1, 10 ** 12) and w[1] == -w[0]
