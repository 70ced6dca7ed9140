"""Wide rows against the fp64 oracle with the bound of the sums as the kernels take them.

A thread of the walking kernel has at least 96 companions (224 where a row has more than 1024 pieces of 16 bytes), adds the elements of a piece to one
another and the pieces' sums in turn: V / (8 * 224) roundings for bf16, V / (4 * 224) for fp32, doubled for the two packed halves that are added
last.  Held rows and clusters add at most 64 elements in turn.  Beside that, 64 roundings for the reductions over lanes, warps and blocks, the changes of
reference and the logarithms; a probability 2^(x c - m) has 2^-24 |x c| each for c, the product and the reference, and 2^-22 for the exponential.
At 128000 words that is 2e-5, a tenth of V / 32 roundings."""
import math

import numpy as np
import pytest
import torch

from oracle import operators as O
from tests.test_gpu_distill import BF, F, FORMS, STORE, U, Case, b  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("rest", [True, False])
@pytest.mark.parametrize("dtype,T,V,K", [(BF, 80, 9000, 40), (BF, 80, 40000, 64), (BF, 80, 128000, 64), (BF, 80, 300001, 20), (F, 80, 40000, 32), (F, 80, 128000, 64), (BF, 3, 128000, 64),
                                         (F, 3, 50001, 100)])
def test_wide_rows(b, form, rest, dtype, T, V, K):  # noqa: F811
    c = Case(T, V, K, dtype, 1.0, rest)
    loss, dS = c.run(b, form)
    per = 8 if dtype == BF else 4
    chain = 2 * V / (per * (224 if V > 1024 * per else 96)) + 64
    for i in (0, 1, T - 1):
        S = c.S[i].cpu().double().numpy()
        want, grad, f = O.distill_row(S, c.t[i], c.idx[i], float(c.lse[i]) if rest else None, float(c.weight[i]), 1.0)
        size = (np.abs(S).max() + np.abs(c.t[i]).max() + (abs(float(c.lse[i])) if rest else 0)) / math.log(2)
        e = (chain + 64 + 8 + 3 * size) * U
        w = float(c.weight[i])
        bound = w * (2 * e * (1 + f["terms"]) + (2 * e * (1 + f["log_r"]) if rest else 0)) + abs(want) * 2 * U
        assert abs(loss[i].item() - want) <= bound, (i, loss[i].item(), want, bound)
        if dS is None:
            continue
        allowed = w * (2 * e * (f["p"] + f["q"]) + 2 * (e + e * f["r"]) * f["pull"]) + np.abs(grad) * (STORE[dtype] + 3 * U) + 1e-38
        off = np.abs(dS[i].cpu().double().numpy() - grad)
        assert np.all(off <= allowed), (i, int(np.argmax(off / allowed)), float(np.max(off / allowed)))
