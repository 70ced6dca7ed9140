"""The fp64 oracle where a weight channel has no scale, and where a teacher's list does not sum to one (no GPU)."""
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


@pytest.mark.parametrize("K,shift,tau", [(4, -0.7, 1.0), (4, -0.2, 2.5), (9, -0.3, 1.0), (9, 0.4, 1.0), (9, 0.4, 2.0), (8, 0.1, 0.7)])
def test_gradient_is_the_difference_quotient_of_the_loss(K, shift, tau):
    g = np.random.default_rng(3)
    V = 9
    t, s = g.standard_normal(V) * 2, g.standard_normal(V) * 1.5
    idx = np.argsort(-t)[:K]
    lse = math.log(np.exp(t / tau).sum()) + shift
    _, grad, _ = O.distill_row(s, t[idx], idx, lse, 0.75, tau)
    h = 1e-5
    for v in range(V):
        d = np.zeros(V)
        d[v] = h
        diff = (O.distill_row(s + d, t[idx], idx, lse, 0.75, tau)[0] - O.distill_row(s - d, t[idx], idx, lse, 0.75, tau)[0]) / (2 * h)
        # h^2 / 6 of the third derivative, and four roundings (2^-52 of a loss below 8) over 2 h
        assert abs(diff - grad[v]) < 1e-9 / tau ** 3 + 4 * 8 * 2.0 ** -52 / (2 * h), v
