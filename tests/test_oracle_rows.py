"""Pins of the oracle of the operators on token rows: closed forms, differences, and independent ways to the same numbers."""
import numpy as np
import pytest

from oracle import flop_oracle as O
from oracle import rows as R


def test_embedding_is_a_product_with_one_hot_rows():
    g = np.random.default_rng(0)
    E, dY = g.standard_normal((7, 5)), g.standard_normal((20, 5))
    ids = g.integers(-2, 9, 20)
    hot = (ids[:, None] == np.arange(7)).astype(float)
    np.testing.assert_allclose(R.embedding_fwd(ids, E, 3.0), 3.0 * hot @ E)
    dE, size, count = R.embedding_bwd(dY, ids, 7, -2.0)
    np.testing.assert_allclose(dE, -2.0 * hot.T @ dY)
    np.testing.assert_allclose(size, 2.0 * hot.T @ np.abs(dY))
    assert np.array_equal(count, hot.sum(0))


def test_mask_draws_other_numbers_than_the_gates_and_the_right_share():
    p, T, d = 0.3, 400, 200
    keep, s = R.dropout_mask(T, d, p, seed=11, offset=0)
    q = 1 - int(np.floor(p * 65536 + 0.5)) / 65536
    assert s == 1 / q
    assert abs(keep.mean() - q) < 5 * np.sqrt(q * (1 - q) / keep.size)
    assert abs((keep[:, :-1] & keep[:, 1:]).mean() - q * q) < 6 * np.sqrt(q * q * (1 - q * q) / keep.size)
    u = O.gate_uniforms(T * d, 11, 0).reshape(T, d)
    assert abs(np.corrcoef(u.ravel(), keep.ravel())[0, 1]) < 5 / np.sqrt(keep.size)


def test_mask_of_single_groups():
    """Group g of row t is one block of the generator, at offset + t ceil(d / 8) + g, for rows of any width and offsets beyond 32 bits."""
    for d, offset in ((8, 0), (13, 2 ** 32 - 2), (1, 2 ** 64 - 2)):
        T, groups, seed = 5, (d + 7) // 8, (77 << 32) + 5
        keep, _ = R.dropout_mask(T, d, 0.5, seed, offset)
        for t in range(T):
            for k in range(d):
                n = (offset + t * groups + k // 8) % 2 ** 64
                word = int(O.philox4x32_10([n & 0xFFFFFFFF], [n >> 32], [1], [0], 5, 77)[k % 8 // 2][0])
                assert keep[t, k] == (((word >> 16) if k % 2 else (word & 0xFFFF)) >= 32768)


@pytest.mark.parametrize("p,threshold", [(0.0, 0), (2.0 ** -17, 1), (0.99999, 65535), (0.25, 16384)])
def test_threshold(p, threshold):
    assert R.dropout_mask(1, 8, p, 0, 0)[1] == 65536 / (65536 - threshold)


def test_layer_norm_closed_form():
    Y, mean, rstd = R.layer_norm_fwd([[1.0, 3.0]], np.array([2.0, 2.0]), np.array([0.5, 0.5]), 0.0)
    np.testing.assert_allclose(Y, [[-1.5, 2.5]])
    assert mean[0, 0] == 2 and rstd[0, 0] == 1


def test_layer_norm_gradient_by_differences():
    g = np.random.default_rng(3)
    S, dY, dS, w, b = g.standard_normal((3, 7)), g.standard_normal((3, 7)), g.standard_normal((3, 7)), g.standard_normal(7), g.standard_normal(7)
    f = lambda s, ww, bb: (R.layer_norm_fwd(s, ww, bb, 1e-3)[0] * dY).sum() + (s * dS).sum()  # noqa: E731
    got = R.layer_norm_bwd(dY, S, w, 1e-3, dS)
    h = 1e-6
    for which, (base, want) in enumerate(zip((S, w, b), got)):
        for at in np.ndindex(base.shape):
            up, down = [S, w, b], [S, w, b]
            up[which], down[which] = base.copy(), base.copy()
            up[which][at] += h
            down[which][at] -= h
            assert abs((f(*up) - f(*down)) / (2 * h) - want[at]) < 1e-7


def test_bounds_hold_for_a_32_bit_evaluation_and_not_for_a_wrong_one():
    g = np.random.default_rng(5)
    S, dY = (4 + 3 * g.standard_normal((40, 300))).astype(np.float32), g.standard_normal((40, 300)).astype(np.float32)
    w, b = g.standard_normal(300).astype(np.float32), g.standard_normal(300).astype(np.float32)
    eps = np.float32(1e-5)
    mean = S.mean(1, keepdims=True, dtype=np.float32)
    rstd = 1 / np.sqrt(((S - mean) ** 2).mean(1, keepdims=True, dtype=np.float32) + eps)
    x = (S - mean) * rstd
    want, _, _ = R.layer_norm_fwd(S, w, b, 1e-5)
    bound = R.layer_norm_fwd_bound(S, w, b, 1e-5, "f32")
    assert np.all(np.abs(x * w + b - want) <= bound)
    assert not np.all(np.abs(x * w * (1 + 1e-4) + b - want) <= bound)
    a = dY * w
    grad = rstd * (a - a.mean(1, keepdims=True) - x * (a * x).mean(1, keepdims=True))
    for got, exact, bd in zip((grad, (dY * x).sum(0), dY.sum(0)), R.layer_norm_bwd(dY, S, w, 1e-5), R.layer_norm_bwd_bound(dY, S, w, 1e-5, "f32")):
        assert np.all(np.abs(got - exact) <= bd)
        assert not np.all(np.abs(got * (1 + 1e-3) - exact) <= bd)
