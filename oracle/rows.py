"""fp64 oracle of the operators on token rows (embedding lookup and its gradient, dropout, layer norm), written from their formulas in
plain numpy, and bounds on what a 32-bit evaluation of them in any order may be off by."""
from __future__ import annotations

import numpy as np

from .flop_oracle import philox4x32_10

U = 2.0 ** -24                                   # half a step of fp32, relative
HALF_STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
# Additions that a value passes through in the sum over a row: a thread's own columns (8 for each of its groups), 5 steps within a warp,
# one for each warp.  128 covers 12 groups a thread and 16 warps, or 8 groups and 32 warps.
ROW_ADDS = 128


def embedding_fwd(ids, E, scale):
    ids = np.asarray(ids)
    Y = np.zeros((ids.size, E.shape[1]))
    for t, v in enumerate(ids.reshape(-1)):
        if 0 <= v < E.shape[0]:
            Y[t] = scale * np.asarray(E[v], dtype=np.float64)
    return Y


def embedding_bwd(dY, ids, n_rows, scale):
    """(dE, the sums of magnitudes, tokens of each word)."""
    dE, size, count = np.zeros((n_rows, dY.shape[1])), np.zeros((n_rows, dY.shape[1])), np.zeros(n_rows, dtype=np.int64)
    for t, v in enumerate(np.asarray(ids).reshape(-1)):
        if 0 <= v < n_rows:
            dE[v] += dY[t]
            size[v] += np.abs(dY[t])
            count[v] += 1
    return scale * dE, abs(scale) * size, count


def dropout_mask(T, d, p, seed, offset):
    """(keep[T, d], the factor of what is kept)."""
    groups = (d + 7) // 8
    threshold = min(int(np.floor(p * 65536 + 0.5)), 65535)
    keep = np.zeros((T, groups * 8), dtype=bool)
    with np.errstate(over="ignore"):
        n = np.uint64(offset % 2 ** 64) + np.arange(T * groups, dtype=np.uint64)
    words = philox4x32_10(n & np.uint64(0xFFFFFFFF), n >> np.uint64(32), np.ones_like(n), np.zeros_like(n), seed & 0xFFFFFFFF, (seed >> 32) & 0xFFFFFFFF)
    for j in range(8):
        h = (words[j // 2] >> np.uint32(16)) if j % 2 else (words[j // 2] & np.uint32(0xFFFF))
        keep[:, j::8] = (h >= threshold).reshape(T, groups)
    return keep[:, :d], 65536.0 / (65536 - threshold)


def dropout(X, p, seed, offset, R=None):
    keep, s = dropout_mask(*X.shape, p, seed, offset)
    Y = np.where(keep, np.asarray(X, dtype=np.float64) * s, 0.0)
    return Y if R is None else Y + R


def layer_norm_fwd(S, weight, bias, eps):
    """(Y, mean, rstd) of rows S."""
    S = np.asarray(S, dtype=np.float64)
    mean = S.mean(1, keepdims=True)
    rstd = 1.0 / np.sqrt(((S - mean) ** 2).mean(1, keepdims=True) + eps)
    Y = (S - mean) * rstd
    Y = Y * (1.0 if weight is None else weight) + (0.0 if bias is None else bias)
    return Y, mean, rstd


def layer_norm_bwd(dY, S, weight, eps, dS=None):
    """(g, dweight, dbias): g is the gradient that arrives at S."""
    S, dY = np.asarray(S, dtype=np.float64), np.asarray(dY, dtype=np.float64)
    _, mean, rstd = layer_norm_fwd(S, None, None, eps)
    x = (S - mean) * rstd
    a = dY if weight is None else dY * weight
    g = rstd * (a - a.mean(1, keepdims=True) - x * (a * x).mean(1, keepdims=True))
    if dS is not None:
        g = g + dS
    return g, (dY * x).sum(0), dY.sum(0)


# ------------------------------------------------------------------------------------------------ bounds
def _x_error(S, eps):
    """(x, its error, rstd, rstd's relative error) in fp32: the mean is off by at most ROW_ADDS + 1 roundings of the magnitudes' mean; the
    squared differences' sum by as many of itself (and by the square of the mean's error); the reciprocal root halves that and is off by
    two steps itself; differences and products round once each."""
    S = np.asarray(S, dtype=np.float64)
    _, mean, rstd = layer_norm_fwd(S, None, None, eps)
    x = (S - mean) * rstd
    d_mean = (ROW_ADDS + 1) * U * np.abs(S).mean(1, keepdims=True)
    rel = (ROW_ADDS + 5) / 2 * U + 4 * U + 0.5 * (d_mean * rstd) ** 2 + d_mean * rstd * U
    return x, rstd * d_mean + np.abs(x) * (rel + 3 * U), rstd, rel


def layer_norm_fwd_bound(S, weight, bias, eps, kind):
    x, e, _, _ = _x_error(S, eps)
    w = 1.0 if weight is None else np.abs(weight)
    Y, _, _ = layer_norm_fwd(S, weight, bias, eps)
    return w * e + U * (np.abs(x) * w + np.abs(Y)) + HALF_STEP[kind] * np.abs(Y) * (1 + 2 ** -7) + 1e-38


def layer_norm_bwd_bound(dY, S, weight, eps, kind, dS=None):
    """Bounds of (g, dweight, dbias); the sums over rows pass through at most T additions."""
    dY = np.asarray(dY, dtype=np.float64)
    x, e, rstd, rel = _x_error(S, eps)
    a = np.abs(dY if weight is None else dY * weight)
    c1, c2 = np.abs((dY if weight is None else dY * weight).mean(1, keepdims=True)), np.abs(((dY if weight is None else dY * weight) * x).mean(1, keepdims=True))
    h = ROW_ADDS + 4
    e1, e2 = h * U * a.mean(1, keepdims=True), h * U * (a * np.abs(x)).mean(1, keepdims=True) + (a * e).mean(1, keepdims=True)
    terms = a + c1 + np.abs(x) * c2
    g, _, _ = layer_norm_bwd(dY, S, weight, eps, dS)
    bound = rstd * (5 * U * terms + rel * terms + e1 + np.abs(x) * e2 + c2 * e) + (0 if dS is None else U * np.abs(g))
    T = dY.shape[0]
    dw = (T + 2) * U * (np.abs(dY) * np.abs(x)).sum(0) + (np.abs(dY) * e).sum(0)
    db = (T + 1) * U * np.abs(dY).sum(0)
    return bound + HALF_STEP[kind] * np.abs(g) * (1 + 2 ** -7) + 1e-38, dw + 1e-38, db + 1e-38
