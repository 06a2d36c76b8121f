"""fp64 oracle of the logit operators, row by row from the definitions: log
probabilities with entropy and top alternatives, and distillation from a
teacher's top logits. Rows are given as a list of one-dimensional arrays;
indices count from 0 in each row (`first`, per row, is added to what comes out)."""
from __future__ import annotations

import numpy as np


def _log_softmax(z):
    """log p, or None for a row with nothing left."""
    m = z.max() if z.size else -np.inf
    if m == -np.inf:
        return None
    return z - m - np.log(np.exp(z - m).sum())


def top_order(x):
    """Highest first, equal values by index, NaN after every number."""
    x = np.asarray(x, np.float64)
    return np.lexsort((np.arange(x.size), -np.nan_to_num(x, nan=0.0, posinf=np.inf, neginf=-np.inf), np.isnan(x)))


def logprobs(rows, tokens, K, temperature=1.0, first=None):
    n = len(rows)
    first = np.zeros(n, np.int64) if first is None else first
    o = dict(logp=np.full(n, np.nan), entropy=np.zeros(n), top=np.full((n, K), -1, np.int64),
             top_logp=np.full((n, K), -np.inf))
    for r, x in enumerate(rows):
        x = np.asarray(x, np.float64)
        masked = np.where(np.isnan(x), -np.inf, x)
        lp = _log_softmax(masked / temperature)
        if lp is None:
            lp = np.full(x.size, -np.inf)
        else:
            p = np.exp(lp)
            o["entropy"][r] = -(p[p > 0] * lp[p > 0]).sum()
        if tokens is not None and 0 <= tokens[r] - first[r] < x.size:
            o["logp"][r] = lp[tokens[r] - first[r]]
        idx = top_order(x)[:K]
        o["top"][r, :idx.size] = idx + first[r]
        o["top_logp"][r, :idx.size] = lp[idx]
    return o


def distill(rows, top, teacher, weight=None, temperature=1.0, first=None):
    """-> dict(loss [n], grad: list of rows)"""
    n = len(rows)
    first = np.zeros(n, np.int64) if first is None else first
    loss, grad = np.zeros(n), []
    for r, x in enumerate(rows):
        x = np.asarray(x, np.float64)
        g = np.zeros(x.size)
        grad.append(g)
        at = top[r].astype(np.int64) - first[r]
        have = (top[r] >= 0) & (at >= 0) & (at < x.size)
        lq = _log_softmax(np.asarray(teacher[r], np.float64)[have] / temperature)
        lp = _log_softmax(x / temperature)
        if lq is None or lp is None:
            continue
        q, i = np.exp(lq), at[have]
        loss[r] = sum(q[k] * (lq[k] - lp[i[k]]) for k in range(q.size) if q[k] > 0)
        g += np.exp(lp)
        np.subtract.at(g, i, q)
        g *= (1.0 if weight is None else float(weight[r])) / temperature
    return dict(loss=loss, grad=grad)
