"""fp64 oracle of layer norm and the gated delta rule with their gradients, row by row
and token by token from the definitions.

Layer norm also gives, under "bound", how far fp32 arithmetic of the same formulas may be off, element by
element and to first order. The delta rule's sequences are packed: sequence i is rows offs[i] .. offs[i+1]-1.
"""
from __future__ import annotations

import numpy as np

EPS = 2.0 ** -24  # one fp32 rounding
SUM = 64          # roundings on the longest way through a sum over a row: 32 entries of a thread, the rest joined by halves


def layer_norm(x, w=None, b=None, eps=1e-5):
    """-> dict(y, bound)"""
    x, w, b, h, r, e = _norm(x, w, b, eps)
    y = h * w + b
    return dict(y=y, bound=np.abs(w) * e["h"] + 2 * EPS * (np.abs(h * w) + np.abs(b)))


def _norm(x, w, b, eps):
    """h, r and the errors of both in fp32: the mean's is SUM roundings of the mean absolute value; the
    variance's is relative: SUM + 16 roundings, and that of the means of parts whose differences it
    sums; r has half of it."""
    x = np.asarray(x, np.float64)
    C = x.shape[1]
    w = np.ones(C) if w is None else np.asarray(w, np.float64)
    b = np.zeros(C) if b is None else np.asarray(b, np.float64)
    m = x.mean(1, keepdims=True)
    var = ((x - m) ** 2).mean(1, keepdims=True)
    r = 1.0 / np.sqrt(var + eps)
    h = (x - m) * r
    em = SUM * EPS * np.abs(x).mean(1, keepdims=True)
    sd = np.sqrt(var)
    ev = (SUM + 16) * EPS * var + 4 * em * sd + 4 * em ** 2
    er = 0.5 * ev / (var + eps) + 4 * EPS
    return x, w, b, h, r, dict(h=r * em + np.abs(h) * (er + 4 * EPS), r=er)


def layer_norm_backward(x, w, dy, eps=1e-5):
    """-> dict(dx, dw, db, bound: dict of the same)"""
    x, w, _, h, r, e = _norm(x, w, None, eps)
    dy = np.asarray(dy, np.float64)
    g = dy * w
    mean = lambda a: a.mean(1, keepdims=True)
    mg, mgh = mean(g), mean(g * h)
    emg = SUM * EPS * mean(np.abs(g))
    emgh = mean(np.abs(g) * e["h"]) + (SUM + 4) * EPS * mean(np.abs(g * h))
    dx = r * (g - mg - h * mgh)
    terms = np.abs(g) + np.abs(mg) + np.abs(h * mgh)
    bx = r * (emg + np.abs(h) * emgh + e["h"] * np.abs(mgh) + terms * (e["r"] + 4 * EPS))
    chain = len(x) + 40
    bw = (np.abs(dy) * e["h"]).sum(0) + chain * EPS * np.abs(dy * h).sum(0)
    return dict(dx=dx, dw=(dy * h).sum(0), db=dy.sum(0),
                bound=dict(dx=bx, dw=bw, db=chain * EPS * np.abs(dy).sum(0)))


def _delta(q, k, v, g, beta, offs, scale, state):
    q, k, v, g, beta = (np.asarray(a, np.float64) for a in (q, k, v, g, beta))
    T, H, Dv = v.shape
    share = H // q.shape[1]
    q, k = np.repeat(q, share, 1), np.repeat(k, share, 1)
    Dk = q.shape[2]
    n = len(offs) - 1
    start = np.zeros((n, H, Dk, Dv)) if state is None else np.asarray(state, np.float64)
    return q, k, v, np.exp(g), beta, start, Dk ** -0.5 if scale is None else scale, share


def delta_rule(q, k, v, g, beta, offs, scale=None, state=None):
    """S <- e^g S, u = beta (v - S^T k), S <- S + k u^T, o = scale S^T q. -> dict(o, end)"""
    q, k, v, a, beta, start, scale, _ = _delta(q, k, v, g, beta, offs, scale, state)
    o, end = np.zeros_like(v), start.copy()
    for i in range(len(offs) - 1):
        S = end[i]
        for t in range(offs[i], offs[i + 1]):
            S *= a[t][:, None, None]
            u = beta[t][:, None] * (v[t] - (S * k[t][:, :, None]).sum(1))
            S += k[t][:, :, None] * u[:, None, :]
            o[t] = scale * (S * q[t][:, :, None]).sum(1)
    return dict(o=o, end=end)


def delta_rule_backward(q, k, v, g, beta, do, offs, scale=None, state=None, dend=None):
    """-> dict(dq, dk, dv, dg, dbeta, dstate)"""
    q, k, v, a, beta, start, scale, share = _delta(q, k, v, g, beta, offs, scale, state)
    do = np.asarray(do, np.float64)
    T, H, Dk = q.shape
    dq, dk, dv, dg, dbeta = (np.zeros_like(x) for x in (q, k, v, a, beta))
    dstate = np.zeros_like(start)
    for i in range(len(offs) - 1):
        S, before, us = start[i].copy(), [], []
        for t in range(offs[i], offs[i + 1]):
            before.append(S.copy())
            S = S * a[t][:, None, None]
            us.append(v[t] - (S * k[t][:, :, None]).sum(1))
            S = S + k[t][:, :, None] * (beta[t][:, None] * us[-1])[:, None, :]
        G = np.zeros_like(S) if dend is None else np.asarray(dend[i], np.float64).copy()
        for t in reversed(range(offs[i], offs[i + 1])):
            D = before[t - offs[i]] * a[t][:, None, None]
            u = us[t - offs[i]]
            S = D + k[t][:, :, None] * (beta[t][:, None] * u)[:, None, :]
            dq[t] = scale * (S * do[t][:, None, :]).sum(2)
            G = G + scale * q[t][:, :, None] * do[t][:, None, :]
            du = (G * k[t][:, :, None]).sum(1)
            dbeta[t] = (du * u).sum(1)
            du = du * beta[t][:, None]
            dv[t] = du
            dk[t] = (G * (beta[t][:, None] * u)[:, None, :]).sum(2) - (D * du[:, None, :]).sum(2)
            G = G - k[t][:, :, None] * du[:, None, :]
            dg[t] = (G * D).sum((1, 2))
            G = G * a[t][:, None, None]
        dstate[i] = G
    sum_heads = lambda x: x.reshape(T, H // share, share, Dk).sum(2)
    return dict(dq=sum_heads(dq), dk=sum_heads(dk), dv=dv, dg=dg, dbeta=dbeta, dstate=dstate)
