"""Teachers whose list sums to more than one, or to less with every word on it (logits and normalisers kept in 16 bits): the loss has the slope
(sum q + r) p - q there, against the oracle and against differences of the library's own losses.  Bounds: `Case.check` (tests/test_gpu_distill.py)."""
import numpy as np
import pytest
import torch

from tests.test_gpu_distill import BF, F, FORMS, Case, b  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("shift", [-0.02, -0.4, 0.3])
@pytest.mark.parametrize("T,V,K", [(3, 40, 40), (3, 40, 39), (6, 205, 30), (3600, 205, 16), (3600, 12, 12), (5, 5000, 60), (90, 6000, 30), (80, 20000, 100), (90, 40000, 64), (80, 70000, 20)])
def test_lists_that_do_not_sum_to_one(b, form, dtype, shift, T, V, K):  # noqa: F811
    c = Case(T, V, K, dtype, 1.0, True)
    c.lse += np.float32(shift)
    c.check(b, form, rows=np.unique([0, 1, T // 2, T - 1]))


@pytest.mark.parametrize("K,shift", [(8, -0.5), (39, -0.1), (40, -0.3), (40, 0.3)])
def test_gradient_is_the_difference_of_the_losses(b, K, shift):  # noqa: F811
    """Central differences, h = 2^-4: the rounding of two losses (2^-21 each) over 2 h is 2^-17, and the third derivative of (sum q + r) log sum exp
    (below 2 at a sum of 2) gives h^2 / 3 at most."""
    V = 40
    c = Case(1, V, K, F, 1.0, True, weighted=False)
    c.lse += np.float32(shift)
    h, many = 2.0 ** -4, Case(2 * V, V, K, F, 1.0, True, weighted=False)
    many.t[:], many.idx[:], many.lse[:] = c.t[0], c.idx[0], c.lse[0]
    many.S.copy_(c.S.expand(2 * V, V))
    many.S[:V] += h * torch.eye(V, device="cuda")
    many.S[V:] -= h * torch.eye(V, device="cuda")
    loss, _ = many.run(b, "fwd")
    diff = (loss[:V] - loss[V:]) / (2 * h)
    for form in ("bwd", "both"):
        _, dS = c.run(b, form)
        assert torch.all((diff - dS[0]).abs() < 1.3e-3 + 2.0 ** -17)
