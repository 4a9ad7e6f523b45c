"""What a cache in 4 bits holds, by definition: multiples of a group's scale that seven of them reach to the group's largest entry."""
import numpy as np
import pytest

import q4_util as Q
from oracle import layer_oracle as L


@pytest.mark.parametrize("seed", range(4))
def test_held_values_are_multiples_of_the_scale(seed):
    rng = np.random.default_rng(seed)
    x = (rng.standard_normal((300, 16)) * 2.0 ** rng.uniform(-20, 12, (300, 1))).astype(np.float32)
    x[::7, 3] *= 9
    s = np.array([L.q4_scale(g) for g in x])[:, None]
    c, b = Q.quantise(x)
    assert np.array_equal(Q.scale_of(b), s)
    n = L.q4_held(x) / s
    assert np.array_equal(n, np.rint(n)) and np.all(np.abs(n) <= 7) and np.array_equal(n, c)
    # the largest entry of a group within the scales' range takes the last code (its quotient is 7 but for the scale's rounding, 1/16)
    largest = np.abs(x).max(1)
    inside = (largest >= 7 * 2.0 ** -20) & (largest <= 7 * 1792.0)
    assert inside.sum() > 250 and np.all(np.abs(n).max(1)[inside] == 7)
    assert np.all(np.abs(n * s - x)[inside] <= s[inside] / 2 * (1 + 2.0 ** -22))     # (codes come from fp32 quotients)
