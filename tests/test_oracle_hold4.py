"""The oracle's 4-bit values at the ends of the range (CPU)."""
import math

import numpy as np
import pytest

import oracle


@pytest.mark.parametrize("bad", [math.nan, -math.nan, math.inf, -math.inf, 3.5 * 2.0 ** 126, -3.75 * 2.0 ** 126, 2.0 ** 130])
def test_groups_that_are_held_as_nan(bad):
    x = np.random.default_rng(1).standard_normal(96)
    y = x.copy()
    y[40] = bad
    got, want = oracle.hold4(y), oracle.hold4(x)
    assert np.isnan(got[32:64]).all()
    assert np.array_equal(got[:32], want[:32]) and np.array_equal(got[64:], want[64:])


def test_largest_held_magnitude():
    x = np.zeros(32)
    x[3], x[4] = -3.5 * 2.0 ** 126 * (1 - 2.0 ** -24), 2.0 ** 126
    got = oracle.hold4(x)
    assert got[3] == -3 * 2.0 ** 126 and got[4] == 2.0 ** 126 and not got[5:].any()
