"""The operators on logits from their definitions, in 64 bits with numpy, one row at a time; test infrastructure only."""
from __future__ import annotations

import numpy as np

NINF = -np.inf


def log_softmax(z: np.ndarray, scale: float):
    """(largest logit, ln sum exp(scale (z - largest)), log probabilities) of one row of float64."""
    if z.size == 0 or np.all(np.isneginf(z)):
        return NINF, NINF, np.full(z.size, NINF)
    if np.any(np.isnan(z)) or np.any(np.isposinf(z)):
        return (np.nan if np.any(np.isnan(z)) else np.inf), np.nan, np.full(z.size, np.nan)
    m = z.max()
    y = scale * (z - m)
    ls = np.log(np.exp(y).sum())
    return m, ls, y - ls


def entropy(lq: np.ndarray) -> float:
    if np.any(np.isnan(lq)):
        return np.nan
    with np.errstate(invalid="ignore"):
        return float(-np.where(np.isneginf(lq), 0.0, np.exp(lq) * lq).sum())


def top(z: np.ndarray, k: int) -> np.ndarray:
    """Columns of the k largest, the lower one first among equals, NaN before all."""
    v = np.where(np.isnan(z), np.inf, z)
    order = sorted(range(z.size), key=lambda j: (not np.isnan(z[j]), -v[j], j))
    return np.array(order[:k], dtype=np.int64)


def score_grad(z, scale, targets, g, gh):
    """Gradient, and the sum of the sizes of its terms (what its error is measured by)."""
    _, ls, lq = log_softmax(z, scale)
    if np.isneginf(ls):
        return np.zeros(z.size), np.zeros(z.size)
    q, lqf = np.exp(lq), np.where(np.isneginf(lq), 0.0, lq)
    h = entropy(lq)
    dz, size = np.zeros(z.size), np.zeros(z.size)
    for t, w in zip(targets, g):
        if 0 <= t < z.size:
            dz -= w * q
            dz[t] += w
            size += abs(w) * q
            size[t] += abs(w)
    dz -= gh * q * (lqf + h)
    size += abs(gh) * q * (np.abs(lqf) + h)
    return scale * dz, scale * size


def distill(z, scale, ids, v, teacher_scale, tail: bool):
    """(loss, d loss / dz, sizes of the loss's terms, sizes of the gradient's, ln of the sum off the list)."""
    n = z.size
    m, ls, lq = log_softmax(z, scale)
    there = (ids >= 0) & (ids < n)
    v = v.astype(np.float64)
    if tail:
        p = np.where(there, np.exp(v), 0.0)
        rest = max(0.0, 1.0 - p.sum())
    else:
        x = np.where(there, teacher_scale * v, NINF)
        p = np.zeros(len(ids)) if np.all(np.isneginf(x)) else np.exp(x - x.max())
        p = p / p.sum() if p.sum() > 0 else p
        rest = 0.0
    off = np.ones(n, dtype=bool)
    off[ids[there]] = False
    if np.isneginf(ls):
        asked = np.any(p > 0) or rest > 0
        return (np.inf if asked else 0.0), np.zeros(n), 1.0, np.zeros(n), (NINF if tail else 0.0)
    q = np.exp(lq)
    loss, size, dz, dsize = 0.0, 0.0, np.zeros(n), np.zeros(n)
    total = p.sum() + rest
    for k in np.flatnonzero(there):
        if p[k] > 0:
            loss += p[k] * (np.log(p[k]) - lq[ids[k]])
            size += p[k] * (abs(np.log(p[k])) + (0 if np.isinf(lq[ids[k]]) else abs(lq[ids[k]])))
        dz[ids[k]] -= p[k]
        dsize[ids[k]] += p[k]
    dz += total * q
    dsize += total * q
    lr = 0.0
    if tail:
        y = scale * (z[off] - m)
        lr = NINF if y.size == 0 or np.all(np.isneginf(y)) else float(np.log(np.exp(y - y.max()).sum()) + y.max())
        if rest > 0 and not (np.isneginf(lr) and rest < 1e-5):
            loss += rest * (np.log(rest) - (lr - ls))
            size += rest * (abs(np.log(rest)) + (0 if np.isinf(lr) else abs(lr - ls)))
        if not np.isneginf(lr):
            r = np.where(off, np.exp(np.where(off, scale * (z - m) - lr, NINF)), 0.0)
            dz -= rest * r
            dsize += rest * r
    return loss, scale * dz, size, scale * dsize, lr
