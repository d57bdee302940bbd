"""How exact the angle of a rotary position is as the call forms it (CPU; the same steps in the same precision).

theta = position * inv_freq radians: the host divides the frequency by 2 pi in fp64, the kernel multiplies by the
position and takes off the whole turns in fp64, and the rest becomes fp32.  The header allows 2^-23 + 2^-51 |theta|
radians.  The exact turn comes from 80 decimal digits.
"""
import math
from decimal import Decimal, getcontext

import numpy as np
import pytest


@pytest.mark.parametrize("freq,position", [(1.0, 4096), (1.0, 2 ** 27), (1.0, 2 ** 31 - 1), (30.0, 131072),
                                           (1e3, 2 ** 31 - 1), (1e6, 2 ** 31 - 1)])
def test_the_stated_error_of_an_angle(freq, position):
    getcontext().prec = 80
    two_pi = 2 * Decimal("3.14159265358979323846264338327950288419716939937510582097494459230781640628620899862803")
    rng = np.random.default_rng(int(freq) + position)
    for _ in range(500):
        f, p = float(np.float32(freq * rng.random())), int(rng.integers(-position, position))
        t = float(p) * (f / (2.0 * 3.14159265358979323846))
        t = float(np.float32(t - np.rint(t)))
        exact = Decimal(f) * p / two_pi
        off = abs(Decimal(t) - (exact - exact.to_integral_value())) % 1
        off = float(min(off, 1 - off)) * 2 * math.pi
        assert off <= 2.0 ** -23 + 2.0 ** -51 * f * abs(p)
