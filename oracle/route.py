"""Routing to experts in 64 bits, written from its definition (test infrastructure)."""
import numpy as np


def scores(logits, score):
    """Scores [T, E] of logits (float64, -inf: none); a row without any logit has none."""
    if score == "sigmoid":
        return np.exp(-np.logaddexp(0.0, -logits))
    top = logits.max(axis=1, keepdims=True)
    e = np.where(logits > -np.inf, np.exp(logits - np.where(top > -np.inf, top, 0.0)), 0.0)
    return e / np.maximum(e.sum(axis=1, keepdims=True), 1e-300)


def cleaned(logits):
    """NaN counts as -inf, +inf as the largest fp32 number."""
    l = np.asarray(logits, np.float64)
    return np.where(l > -np.inf, np.minimum(l, float(np.finfo(np.float32).max)), -np.inf)


def choose(logits, top, score, bias=None, groups=1, kept=1, best=2, renormalise=True, scale=1.0):
    """Experts [T, top] (-1: none) and weights [T, top]."""
    l = cleaned(logits)
    T, E = l.shape
    s = scores(l, score)
    with np.errstate(invalid="ignore"):
        c = s + (0.0 if bias is None else np.asarray(bias, np.float64))
    c = np.where((l > -np.inf) & (c > -np.inf), c, -np.inf)
    expert, weight = np.full((T, top), -1, np.int64), np.zeros((T, top))
    for t in range(T):
        key = c[t]
        if groups > 1:
            of = -np.sort(-key.reshape(groups, -1), axis=1)[:, :best]
            total = np.where(of[:, 0] > -np.inf, np.where(of > -np.inf, of, 0.0).sum(axis=1), -np.inf)
            stay = np.argsort(-total, kind="stable")[:kept]
            mask = np.zeros(groups, bool)
            mask[stay] = total[stay] > -np.inf
            key = np.where(np.repeat(mask, E // groups), key, -np.inf)
        order = np.lexsort((np.arange(E), -l[t], -key))
        order = order[key[order] > -np.inf][:top]
        expert[t, :len(order)] = order
        if not len(order):
            continue
        if renormalise:   # the logarithms first: a common factor does not count
            logs = l[t, order] if score == "softmax" else -np.logaddexp(0.0, -l[t, order])
            w = np.exp(logs - logs.max())
            weight[t, :len(order)] = w / w.sum()
        else:
            weight[t, :len(order)] = s[t, order]
    return expert, weight * scale


def routes(expert, E):
    """(token [R], offset [E + 1], row [T, top]) of the choices."""
    T, top = expert.shape
    flat = expert.reshape(-1)
    there = np.flatnonzero(flat >= 0)
    order = there[np.argsort(flat[there], kind="stable")]
    token, row = np.full(T * top, -1, np.int64), np.full(T * top, -1, np.int64)
    token[:len(order)] = order // top
    row[order] = np.arange(len(order))
    return token, np.concatenate([[0], np.bincount(flat[there], minlength=E).cumsum()]), row.reshape(T, top)


def combine(y, weight, row, add=None):
    """(sums [T, N], sums of their terms' magnitudes)."""
    T, N = row.shape[0], y.shape[1]
    out = np.zeros((T, N)) if add is None else np.array(add, np.float64)
    size = np.abs(out)
    for j in range(row.shape[1]):
        live = (row[:, j] >= 0) & (row[:, j] < y.shape[0])
        part = y[row[live, j]] * np.asarray(weight, np.float64)[live, j][:, None]
        out[live] += part
        size[live] += np.abs(part)
    return out, size
