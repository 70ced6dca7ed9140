"""The fp64 oracle where a weight channel has no scale (no GPU)."""
import math

import numpy as np
import pytest

from oracle import operators as O


@pytest.mark.parametrize("scale", [math.nan, math.inf])
@pytest.mark.parametrize("at", [0, 2, 4])
def test_a_channel_without_a_scale_reaches_every_token(scale, at):
    g = np.random.default_rng(at)
    x, qq, pq = g.standard_normal((3, 8)), g.integers(-127, 128, (5, 8)), g.integers(-127, 128, (6, 5))
    x[2] = 0
    s = np.ones(5)
    s[at] = scale
    Y, hq = O.compact_fwd_i8(x, qq, s, pq, np.ones(6))
    assert np.isnan(Y).all() and not hq.any()
