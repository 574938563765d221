"""The rotation's frequencies and fractions of a turn, where signs and sizes are unusual.  No GPU."""
import ctypes
import math
from fractions import Fraction

import numpy as np
import pytest

from paper_2608_01655_gb300 import build as ppbuild

TWO_PI = Fraction("6.28318530717958647692528676655900576839433879875021")


@pytest.fixture(scope="module")
def lib():
    ppbuild.build()
    from paper_2608_01655_gb300 import binding
    return binding


def _turns(lib, f):
    f = np.ascontiguousarray(f, np.float64)
    out = np.zeros(len(f), np.uint64)
    P = lambda a: a.ctypes.data_as(ctypes.c_void_p)
    assert lib._lib.pp_rotary_turns(len(f), P(f), P(out)) == lib.PP_OK
    return [int(x) for x in out]


SIZES = [1e-9, 1e-4, 3e-13, 1e-18, 1e-19, 3.4e-19, 1e-30, 0.1, 1.0, 6.2, 7.0, 1e5, 1e9]


@pytest.mark.parametrize("sign", [1, -1])
def test_turns_are_the_nearest_fractions(lib, sign):
    """Off by the quotient's own rounding (2 pi by 2^-54 and the division by 2^-53 of itself, below 2^-52 together) and
    half a step of 2^-64."""
    for x, got in zip(SIZES, _turns(lib, [sign * x for x in SIZES])):
        exact = sign * Fraction(x) / TWO_PI
        off = Fraction(got, 1 << 64) - exact
        off -= round(off)                                   # whole turns do not matter
        assert abs(off) <= abs(exact) * Fraction(1, 1 << 52) + Fraction(1, 1 << 65), x


def test_turns_of_opposite_frequencies_are_opposite(lib):
    for a, b in zip(_turns(lib, SIZES), _turns(lib, [-x for x in SIZES])):
        assert (a + b) % (1 << 64) == 0


def test_angles_of_small_negative_frequencies_at_far_positions(lib):
    """-1e-9 radians a token at the last position: 2^-52 of the angle and a 2^31st of 2^-65 turns."""
    position = (1 << 31) - 1
    got = _turns(lib, [-1e-9])[0]
    part = position * got % (1 << 64)
    angle = Fraction(part - (1 << 64 if part >> 63 else 0), 1 << 64) * TWO_PI
    assert abs(angle + Fraction(1e-9) * position) <= 2.2 * 2.0 ** -52 + 2 * math.pi * 2.0 ** (31 - 65)


@pytest.mark.parametrize("args", [(4, 1e4, 1, 9, -math.inf, 2), (4, 1e4, 1, 9, 1, math.inf), (4, 1e4, 1, 9, -math.inf, math.inf),
                                  (64, 1e-320, 1, 0, 1, 2), (4, 1e-300, 1e-200, 0, 1, 2), (4, 1e4, 5e-324, 0, 1, 2)])
def test_frequencies_that_are_no_numbers_are_refused(lib, args):
    """Ramps without an end, and powers and quotients beyond the largest number."""
    out = np.full(64, 7.0)
    assert lib._lib.pp_rotary_frequencies(*args, out.ctypes.data_as(ctypes.c_void_p)) == lib.PP_EINVAL
    assert (out == 7).all() and lib.last_error()


def test_a_ramp_is_not_looked_at_without_an_original_context(lib):
    out = np.zeros(4)
    assert lib._lib.pp_rotary_frequencies(4, 16.0, 2.0, 0.0, -math.inf, math.nan, out.ctypes.data_as(ctypes.c_void_p)) == lib.PP_OK
    assert np.allclose(out, [0.5, 0.25, 0.125, 0.0625], rtol=1e-15, atol=0)


def test_pairs_that_keep_their_frequency_do_so_whatever_the_factor(lib):
    out = np.zeros(2)
    assert lib._lib.pp_rotary_frequencies(2, 4.0, 5e-324, 1e6, 1.0, 2.0, out.ctypes.data_as(ctypes.c_void_p)) == lib.PP_OK
    assert out.tolist() == [1.0, 0.5]
