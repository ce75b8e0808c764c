"""Infinities of a block's output and its residual come out where, and with the sign, that
the formulas give them; the other values of their tokens keep their bounds."""
import math

import pytest

from test_residual_norm import dev, rand  # noqa: F401
from test_residual_norm_ranges import run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("after", ["none", "rms", "layer"])
@pytest.mark.parametrize("before", ["none", "rms", "layer"])
def test_infinities(dev, after, before, dtype):  # noqa: F811
    for bad in (math.inf, -math.inf):
        for scale in (0.7, -2.0):
            R, A = rand(2, 200, 20), rand(1, 200, 20)
            R[150, 11], R[3, 0], R[199, 19] = bad, -bad, bad
            run(dev, 200, 20, dtype, after, before, scale, True, True, R=R, eps=1e-6)
            A[7, 3], R[8, 3] = bad, bad
            run(dev, 200, 20, dtype, after, before, scale, False, True, A=A, R=R, eps=1e-6)
