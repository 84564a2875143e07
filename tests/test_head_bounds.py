"""The bound of the singular values that sage_orthogonalize scales its parts by, through what it refuses. No call here reaches a GPU."""
import ctypes as C

import numpy as np
import pytest

from paper_2510_02470_amd import binding
from paper_2510_02470_amd.binding import SAGE_ERR_ARG, SAGE_F32, SAGE_OK


def _rc(*triples):
    coef = (C.c_float * (3 * len(triples)))(*[v for t in triples for v in t])
    return binding.lib().sage_orthogonalize(None, SAGE_F32, 0, 1, 1, 1, 1, coef, len(triples), 0.0, 1.0, None, 1, 1, None, 0, None)


@pytest.mark.parametrize("c", [1e-30, -1e-30, 1e-38, 1e-20, -1e-12, 1e-9, 0.0])
def test_nearly_cubic_polynomials_keep_their_extreme(c):
    """600 s - 600 s^3 + c s^5 is 231 inside of the interval and next to 0 at its end, however small c is; times 5 it passes 2^10."""
    assert _rc((600.0, -600.0, c), (4.0, 0.0, 0.0)) == SAGE_OK
    assert _rc((600.0, -600.0, c), (5.0, 0.0, 0.0)) == SAGE_ERR_ARG
    assert _rc((-600.0, 600.0, c), (5.0, 0.0, 0.0)) == SAGE_ERR_ARG


def test_bounds_are_those_of_a_grid():
    """A polynomial, and then a factor that takes its largest value over the first interval (a little wider than [0, 1]) just below
    2^10, and just above."""
    rng = np.random.default_rng(1)
    s = np.linspace(0.0, 1.0 + 2.0 ** -10, 20001)
    for i in range(3000):
        a, b, c = (float(np.float32(v)) for v in rng.standard_normal(3) * 10.0 ** rng.uniform([-2, -2, -14], [1, 1, 1]))
        if i % 5 == 0:
            b = float(np.float32(-a * rng.uniform(0.3, 1.2)))
        top = float(np.abs(a * s + b * s ** 3 + c * s ** 5).max())
        f = 1024.0 / top
        if f > 1000.0:
            continue
        # (2^-10 is added to the bound after every step)
        assert _rc((a, b, c), (f * (1 - 2.0 ** -8), 0.0, 0.0)) == SAGE_OK, (a, b, c)
        assert _rc((a, b, c), (f * (1 + 2.0 ** -12), 0.0, 0.0)) == SAGE_ERR_ARG, (a, b, c)


def test_coefficients_of_up_to_1024_are_taken():
    """Greater ones are not, also where what they make of singular values stays below 2^10."""
    assert _rc((1024.0, -1024.0, 0.0)) == SAGE_OK and _rc((-1024.0, 1024.0, 0.0)) == SAGE_OK and _rc((0.0, 1000.0, -1024.0)) == SAGE_OK
    for t in ((1025.0, -1025.0, 0.0), (2000.0, -2000.0, 0.0), (0.0, -1025.0, 1024.0), (0.0, 1024.0, -1025.0)):
        assert _rc(t) == SAGE_ERR_ARG
