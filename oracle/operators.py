"""fp64 oracle of the 8-bit products and of distillation from top logits, written from their formulas in plain numpy (rows in a loop,
nothing shared with the library)."""
from __future__ import annotations

import math

import numpy as np


def quantize_rows(x):
    """(8-bit integers, fp32 scale) of each row of x (values that fp32 holds): 127 x / max|x| rounded half to even in fp64, which is on
    a border only where the exact quotient is."""
    x = np.asarray(x, dtype=np.float64)
    q, scale = np.zeros(x.shape, dtype=np.int64), np.zeros(x.shape[0], dtype=np.float32)
    for i, row in enumerate(x):
        if row.size == 0:
            continue
        if not np.all(np.isfinite(row)):
            scale[i] = np.nan
            continue
        amax = np.abs(row).max()
        if amax > 0:
            q[i] = np.rint(127.0 * row / amax).astype(np.int64)
            scale[i] = np.float32(amax) / np.float32(127)
    return q, scale


def gemm_i8(a, b, a_scale, b_scale):
    acc = np.asarray(a, dtype=np.float64) @ np.asarray(b, dtype=np.float64).T          # integers below 2^53: exact
    return acc * np.asarray(a_scale, dtype=np.float64)[:, None] * np.asarray(b_scale, dtype=np.float64)


def compact_fwd_i8(x, qq, q_scale, pq, p_scale):
    """(Y, the intermediate's integers).  The token's scale is common to a row of H and leaves its integers alone; a row of H that is not
    finite (a channel whose scale is not) has none."""
    xq, x_scale = quantize_rows(x)
    with np.errstate(invalid="ignore"):                      # 0 times infinity
        h = (xq.astype(np.float64) @ np.asarray(qq, dtype=np.float64).T) * np.asarray(q_scale, dtype=np.float64)
    hq, h_scale = np.zeros(h.shape, dtype=np.int64), np.zeros(h.shape[0])
    for i, row in enumerate(h):
        amax = np.abs(row).max()
        if not np.isfinite(amax):
            h_scale[i] = np.nan
            continue
        if amax > 0:
            hq[i] = np.rint(127.0 * row / amax).astype(np.int64)
        h_scale[i] = float(x_scale[i]) * amax / 127.0
    return gemm_i8(hq, pq, h_scale, p_scale), hq


def _log_sum_exp(v):
    m = max(v, default=-math.inf)
    if m == -math.inf:
        return -math.inf
    return m + math.log(math.fsum(math.exp(u - m) for u in v))


def distill_row(s, t_logits, t_idx, t_lse, weight, tau):
    """(loss, gradient, facts) of one token: `facts` are the sizes a bound on fp32 errors is made of (how the results move with p, q and
    with r, also where r is 0 here and a rounding above it there)."""
    s = np.asarray(s, dtype=np.float64) / tau
    V = s.size
    zero = 0.0, np.zeros(V), None
    listed, t = [], []
    for v, u in zip(t_idx, t_logits):
        if 0 <= v < V and int(v) not in listed:
            listed.append(int(v))
            t.append(float(u) / tau)
    if weight == 0 or not listed:
        return zero
    norm = t_lse if t_lse is not None else _log_sum_exp(t)
    if norm == -math.inf:
        return zero
    outside = np.ones(V, dtype=bool)
    outside[listed] = False
    lse, rest = _log_sum_exp(list(s)), _log_sum_exp(list(s[outside]))
    q = np.array([math.exp(u - norm) for u in t])
    log_p = s[listed] - lse
    terms = [a * (u - norm - b) for a, u, b in zip(q, t, log_p) if a > 0]
    r = max(0.0, 1.0 - math.fsum(q)) if t_lse is not None and len(listed) < V else 0.0
    if r > 0:
        terms.append(r * (math.log(r) - (rest - lse)))
    p = np.exp(s - lse)
    if t_lse is not None:
        p = p * (math.fsum(q) + r)                           # every term holds a -log p of its own weight
    grad = p.copy()
    grad[listed] -= q
    pull, log_r = np.zeros(V), 0.0
    if t_lse is not None and rest > -math.inf:
        pull[outside] = np.exp(s[outside] - rest)
        grad -= r * pull
        log_r = abs(math.log(max(r, 2.0 ** -24))) + abs(rest - lse)
    qv = np.zeros(V)
    qv[listed] = q
    return weight * math.fsum(terms), weight / tau * grad, dict(p=p, q=qv, pull=pull, r=r, terms=math.fsum(abs(x) for x in terms), log_r=log_r)


def distill_topk(S, t_logits, t_idx, t_lse, weight, tau):
    """(loss[T], gradient[T, V], facts[T])."""
    T = S.shape[0]
    out = [distill_row(S[i], t_logits[i], t_idx[i], None if t_lse is None else float(t_lse[i]), 1.0 if weight is None else float(weight[i]), tau) for i in range(T)]
    return np.array([o[0] for o in out]), np.stack([o[1] for o in out]), [o[2] for o in out]
