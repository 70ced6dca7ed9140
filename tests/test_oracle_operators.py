"""The fp64 oracle of the 8-bit products and of the distillation loss against what must hold (no GPU)."""
import math
from fractions import Fraction

import numpy as np
import pytest

from oracle import operators as O


def test_rounding_is_that_of_the_exact_quotient():
    g = np.random.default_rng(1)
    x = np.concatenate([g.standard_normal((20, 40)).astype(np.float32), np.float32(2.0) ** g.integers(-140, 100, (4, 40)), g.integers(-254, 255, (20, 40)) / np.float32(2)], dtype=np.float32)
    q, scale = O.quantize_rows(x)
    for row, qr, sc in zip(x, q, scale):
        amax = max(abs(Fraction(float(v))) for v in row)
        assert sc == np.float32(amax) / np.float32(127)
        for v, n in zip(row, qr):
            assert n == round(127 * Fraction(float(v)) / amax)      # Fraction rounds half to even


def test_rows_without_a_scale():
    q, scale = O.quantize_rows([[0.0, 0.0], [1.0, math.inf], [math.nan, 1.0], [-3.0, 1.5]])
    assert scale[0] == 0 and np.isnan(scale[1]) and np.isnan(scale[2]) and scale[3] == np.float32(3) / np.float32(127)
    assert q.tolist() == [[0, 0], [0, 0], [0, 0], [-127, 64]]        # 63.5 goes to the even neighbour


def test_compact_forward_of_exact_values():
    # identity factors at full scale: both quantisations keep what they are given
    eye = 127 * np.eye(4, dtype=np.int64)
    x = np.array([[127, -64, 3, 0], [0, 0, 0, 0]], dtype=np.float64)
    Y, hq = O.compact_fwd_i8(x, eye, np.full(4, 1 / 127), eye, np.full(4, 1 / 127))
    np.testing.assert_allclose(Y, x, rtol=1e-7)
    assert hq.tolist() == [[127, -64, 3, 0], [0, 0, 0, 0]]


CASES = [(True, 1.0), (True, 2.5), (False, 1.0), (False, 0.7)]


def _row(seed, V=9, K=4):
    g = np.random.default_rng(seed)
    t = g.standard_normal(V) * 2
    idx = np.argsort(-t)[:K]
    return g.standard_normal(V) * 1.5, t, idx


@pytest.mark.parametrize("with_lse,tau", CASES)
def test_gradient_is_the_difference_quotient_of_the_loss(with_lse, tau):
    s, t, idx = _row(3)
    lse = math.log(np.exp(t / tau).sum()) if with_lse else None
    _, grad, _ = O.distill_row(s, t[idx], idx, lse, 0.75, tau)
    h = 1e-5
    for v in range(s.size):
        d = np.zeros(s.size)
        d[v] = h
        diff = (O.distill_row(s + d, t[idx], idx, lse, 0.75, tau)[0] - O.distill_row(s - d, t[idx], idx, lse, 0.75, tau)[0]) / (2 * h)
        assert abs(diff - grad[v]) < 1e-9 / tau ** 3 + 2e-11 / h * 1e-4      # h^2 f''' / 6 and rounding / h


@pytest.mark.parametrize("tau", [1.0, 3.0])
def test_a_student_that_is_its_teacher_has_loss_and_gradient_zero(tau):
    _, t, idx = _row(5)
    lse = math.log(np.exp(t / tau).sum())
    loss, grad, _ = O.distill_row(t, t[idx], idx, lse, 1.0, tau)
    assert abs(loss) < 1e-14 and np.abs(grad).max() < 1e-15
    loss, grad, _ = O.distill_row(t, t, np.arange(t.size), None, 1.0, tau)        # the whole vocabulary listed
    assert abs(loss) < 1e-14 and np.abs(grad).max() < 1e-15


def test_whole_vocabulary_listed_is_the_plain_divergence():
    s, t, _ = _row(7)
    loss, grad, _ = O.distill_row(s, t, np.arange(t.size), None, 1.0, 1.0)
    q, p = np.exp(t) / np.exp(t).sum(), np.exp(s) / np.exp(s).sum()
    assert abs(loss - (q * np.log(q / p)).sum()) < 1e-12
    np.testing.assert_allclose(grad, p - q, atol=1e-14)
    same, _, _ = O.distill_row(s, t, np.arange(t.size), math.log(np.exp(t).sum()), 1.0, 1.0)
    assert abs(same - loss) < 1e-12


def test_repeated_and_empty_slots():
    s, t, idx = _row(11)
    lse = math.log(np.exp(t).sum())
    for norm in (None, lse):
        want = O.distill_row(s, t[idx], idx, norm, 1.0, 1.0)
        got = O.distill_row(s, np.r_[np.nan, t[idx], 50.0, 3.0], np.r_[-1, idx, idx[0], s.size], norm, 1.0, 1.0)
        assert got[0] == want[0] and np.array_equal(got[1], want[1])
        assert O.distill_row(s, t[idx], np.full(4, -1), norm, 1.0, 1.0)[0] == 0
        assert O.distill_row(np.full(9, np.nan), t[idx], idx, norm, 0.0, 1.0)[0] == 0
