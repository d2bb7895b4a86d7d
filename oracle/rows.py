"""Definitions of the row operators in 64 bits (numpy): layer normalisation, the product in 8-bit integers, log-probabilities.

Test infrastructure: plain formulas over a matrix of rows, shares nothing with the library."""
from __future__ import annotations

import numpy as np


def layernorm(x, gamma, beta, eps):
    x = np.asarray(x, np.float64)
    mu = x.mean(axis=1, keepdims=True)
    var = ((x - mu) ** 2).mean(axis=1, keepdims=True)
    return (x - mu) / np.sqrt(var + eps) * np.asarray(gamma, np.float64) + np.asarray(beta, np.float64)


def quantise_rows(x):
    """(whole numbers, scales): round(127 x / a), halves to even, a = max |x|; scale a / 127, NaN for a row that is not finite."""
    x = np.asarray(x, np.float64)
    ok = np.isfinite(x).all(axis=1)
    a = np.where(ok, np.abs(np.where(np.isfinite(x), x, 0)).max(axis=1), 0)
    q = np.rint(127.0 * np.where(ok[:, None], x, 0) / np.where(a > 0, a, 1)[:, None])
    return np.where(a[:, None] > 0, q, 0), np.where(ok, a / 127.0, np.nan)


def qmatmul(x, weight, scale, bias, act):
    """act(sx * scale * (q @ weight.T) + bias); act: 0 none, 1 ReLU, 2 ReLU6."""
    q, sx = quantise_rows(x)
    y = (q @ np.asarray(weight, np.float64).T) * sx[:, None] * np.asarray(scale, np.float64)
    if bias is not None:
        y = y + np.asarray(bias, np.float64)
    if act >= 1:
        y = np.where(y < 0, 0, y)
    if act == 2:
        y = np.where(y > 6, 6, y)
    return y


def logprob(x, labels, top):
    """(log-probabilities of the labels, entropy, ids of the best, their log-probabilities), row by row from the definition."""
    x = np.asarray(x, np.float64)
    rows, n = x.shape
    n_labels = 0 if labels is None else labels.shape[1]
    lp, ent = np.zeros((rows, n_labels)), np.zeros((rows, 1))
    ids, tops = np.full((rows, top), -1, np.int64), np.full((rows, top), -np.inf)
    for r in range(rows):
        v = x[r]
        order = np.argsort(-np.where(np.isnan(v), -np.inf, v), kind="stable")
        order = order[(v[order] > -np.inf)][:top]        # (NaN > -inf is false)
        ids[r, :len(order)] = order
        if np.isnan(v).any() or np.isposinf(v).any():
            logp, ent[r] = np.full(n, np.nan), np.nan
            tops[r] = np.nan
        elif np.isneginf(v).all():
            logp = np.full(n, -np.inf)
        else:
            m = v.max()
            logp = v - m - np.log(np.exp(v - m).sum())
            p = np.exp(logp)
            ent[r] = -(p[p > 0] * logp[p > 0]).sum()
            tops[r, :len(order)] = logp[order]
        for j in range(n_labels):
            lab = labels[r, j]
            lp[r, j] = 0.0 if lab == -1 else logp[lab] if 0 <= lab < n else np.nan
    return lp, ent, ids, tops
