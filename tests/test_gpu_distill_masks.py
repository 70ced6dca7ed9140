"""A student that rules out every word on the teacher's list, the logits of all others far below zero: the sums on the list are 0, and no
reference may turn that into NaN, in rows that are held as in rows that are walked.

Bounds: `Case.check` (tests/test_gpu_distill.py) for rows that the oracle gives a finite loss; where the teacher gives a ruled-out word
something the loss is infinite and its gradient, p - q with p = 0 on the list, is finite and checked with the same terms."""
import math

import numpy as np
import pytest
import torch

from oracle import operators as O
from tests.test_gpu_distill import BF, F, FORMS, STORE, U, Case, b  # noqa: F401

pytestmark = pytest.mark.gpu


# few rows (held by clusters) and many: one pass, two passes, blocks of 128, 256 and 512 threads, both types
@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("rest", [True, False])
@pytest.mark.parametrize("dtype,T,V", [(BF, 6, 700), (BF, 6, 40000), (F, 80, 9000), (BF, 80, 9000), (BF, 80, 17000), (F, 80, 40000), (BF, 80, 70000), (BF, 700, 5000)])
@pytest.mark.parametrize("level", [-300.0, -95.0, 250.0])
def test_every_listed_word_is_masked(b, form, rest, dtype, T, V, level):  # noqa: F811
    c = Case(T, V, 12, dtype, 1.0, rest)
    c.S.sub_(c.S.mean(1, keepdim=True)).add_(level)
    listed = torch.from_numpy(c.idx.astype(np.int64)).cuda()
    c.S.scatter_(1, listed, float("-inf"))
    ruled = np.arange(T) % 2 == 0                    # the teacher gives these words nothing either
    c.t[ruled] = -np.inf
    pick = np.array([0, 2, T - 2 - T % 2])
    loss, dS = c.check(b, form, rows=pick)
    assert torch.isfinite(loss[::2]).all() and torch.all(loss[1::2] == math.inf)
    if dS is None:
        return
    assert torch.isfinite(dS).all()
    for i in (1, 3, T - 1 - T % 2):
        S = c.S[i].cpu().double().numpy()
        _, grad, f = O.distill_row(S, c.t[i], c.idx[i], float(c.lse[i]) if rest else None, float(c.weight[i]), 1.0)
        size = (abs(level) + 20 + np.abs(c.t[i]).max()) / math.log(2) + (abs(float(c.lse[i])) / math.log(2) if rest else 0)
        e = (V / 32 + 64) * U + 8 * U + 2 * U * size
        allowed = float(c.weight[i]) * (2 * e * (f["p"] + f["q"]) + 2 * (e + e * f["r"]) * f["pull"]) + np.abs(grad) * (STORE[dtype] + 3 * U) + 1e-38
        assert np.all(np.abs(dS[i].cpu().double().numpy() - grad) <= allowed), i
