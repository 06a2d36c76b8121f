"""fp64 oracle of the sequence operators: the causal convolution + SiLU and the
selective scan with carried states, and their gradients (sections 5.2 and 6 of the
paper's Mamba block, token by token from the definitions).

Sequences are packed: sequence i is rows offs[i] .. offs[i+1]-1. `state` holds one
start state per sequence (None: zeros); end states are returned per sequence.

Every function also returns, under "bound", how far fp32 arithmetic of the
same formulas may be off, element by element: the sums of the absolute values
of everything that enters a result, times the relative error of one path
through the formula (see EPS_*).
"""
from __future__ import annotations

import numpy as np

EPS = 2.0 ** -24        # one fp32 rounding
EPS_ACT = 4e-6          # SiLU, sigmoid and softplus in fp32, relative


def sigmoid(x):
    return 1.0 / (1.0 + np.exp(-x))


def softplus(x):
    return np.log1p(np.exp(-np.abs(x))) + np.maximum(x, 0.0)


def _f64(*arrays):
    return [None if a is None else np.asarray(a, np.float64) for a in arrays]


def conv(x, w, b, offs, state=None):
    """-> dict(u, end, bound)"""
    x, w, b, state = _f64(x, w, b, state)
    E, K = w.shape
    b = np.zeros(E) if b is None else b
    u, bound = np.zeros_like(x), np.zeros_like(x)
    end = np.zeros((len(offs) - 1, K - 1, E))
    for i in range(len(offs) - 1):
        lo, hi = offs[i], offs[i + 1]
        ext = np.concatenate([np.zeros((K - 1, E)) if state is None else state[i], x[lo:hi]])
        for t in range(hi - lo):
            win = ext[t:t + K]
            pre = b + (w.T * win).sum(0)
            u[lo + t] = pre * sigmoid(pre)
            size = np.abs(b) + (np.abs(w.T) * np.abs(win)).sum(0)
            # K + 1 roundings of partial sums; |SiLU'| <= 1.1
            bound[lo + t] = 1.1 * (K + 1) * EPS * size + EPS_ACT * np.abs(u[lo + t])
        end[i] = ext[hi - lo:]
    return dict(u=u, end=end, bound=bound)


def conv_backward(x, w, b, du, offs, state=None, dend=None):
    """-> dict(dx, dw, db, dstate, bound: dict of the same)"""
    x, w, b, du, state, dend = _f64(x, w, b, du, state, dend)
    E, K = w.shape
    b = np.zeros(E) if b is None else b
    dx, dw, db = np.zeros_like(x), np.zeros_like(w), np.zeros(E)
    bx, bw, bb = np.zeros_like(x), np.zeros_like(w), np.zeros(E)
    n = len(offs) - 1
    ds, bs = np.zeros((n, K - 1, E)), np.zeros((n, K - 1, E))
    for i in range(n):
        lo, hi = offs[i], offs[i + 1]
        L = hi - lo
        ext = np.concatenate([np.zeros((K - 1, E)) if state is None else state[i], x[lo:hi]])
        g_ext, g_abs = np.zeros_like(ext), np.zeros_like(ext)
        if dend is not None:
            g_ext[L:] += dend[i]
            g_abs[L:] += np.abs(dend[i]) * EPS
        for t in range(L):
            win = ext[t:t + K]
            pre = b + (w.T * win).sum(0)
            s = sigmoid(pre)
            d1 = s * (1 + pre * (1 - s))
            g = du[lo + t] * d1
            size = np.abs(b) + (np.abs(w.T) * np.abs(win)).sum(0)
            # SiLU' is off by |SiLU''| <= 0.5 times pre's error, and by its own
            e = np.abs(du[lo + t]) * (0.5 * (K + 1) * EPS * size + EPS_ACT * (1 + np.abs(pre)) * s + 4 * EPS)
            g_ext[t:t + K] += w.T * g
            g_abs[t:t + K] += np.abs(w.T) * (e + (K + 1) * EPS * np.abs(g))
            dw += (g * win).T
            bw += (np.abs(win) * (e + (len(x) + 2) * EPS * np.abs(g))).T
            db += g
            bb += e + (len(x) + 2) * EPS * np.abs(g)
        dx[lo:hi], bx[lo:hi] = g_ext[K - 1:], g_abs[K - 1:]
        ds[i], bs[i] = g_ext[:K - 1], g_abs[:K - 1]
    return dict(dx=dx, dw=dw, db=db, dstate=ds, bound=dict(dx=bx, dw=bw, db=bb, dstate=bs))


def scan(u, dt, A_log, B, C, offs, D=None, z=None, b_dt=None, state=None):
    """-> dict(y, end, bound: dict(y, end))"""
    u, dt, A_log, B, C, D, z, b_dt, state = _f64(u, dt, A_log, B, C, D, z, b_dt, state)
    T, E = u.shape
    N = A_log.shape[1]
    A = -np.exp(A_log)
    D = np.zeros(E) if D is None else D
    v = dt if b_dt is None else dt + b_dt
    d = softplus(v)
    n = len(offs) - 1
    y, end = np.zeros_like(u), np.zeros((n, E, N))
    by, be = np.zeros_like(u), np.zeros((n, E, N))
    gate = np.ones_like(u) if z is None else z * sigmoid(z)
    for i in range(n):
        s = np.zeros((E, N)) if state is None else state[i].copy()
        err = np.zeros((E, N))
        for t in range(offs[i], offs[i + 1]):
            dA = d[t][:, None] * A
            a = np.exp(dA)
            new = a * s + (d[t] * u[t])[:, None] * B[t]
            # dt + b_dt rounds once (|softplus'| <= 1), softplus is off by EPS_ACT; the exponent
            # by that and three roundings (A, its product, log2 e), exp by one
            rel = EPS_ACT + (EPS * np.abs(v[t]) / d[t])
            err = a * err + np.abs(a * s) * (np.abs(dA) * (rel[:, None] + 4 * EPS) + 3 * EPS)
            err += np.abs((d[t] * u[t])[:, None] * B[t]) * (rel[:, None] + 3 * EPS) + np.abs(new) * EPS
            s = new
            full = (s * C[t]).sum(1) + D * u[t]
            size = (np.abs(s * C[t])).sum(1) + np.abs(D * u[t])
            y[t] = full * gate[t]
            by[t] = ((np.abs(C[t]) * err).sum(1) + (N + 2) * EPS * size) * np.abs(gate[t]) + EPS_ACT * np.abs(y[t])
        end[i], be[i] = s, err
    return dict(y=y, end=end, bound=dict(y=by, end=be))


def scan_backward(u, dt, A_log, B, C, dy, offs, D=None, z=None, b_dt=None, state=None, dend=None):
    """-> dict(du, ddt, dz, dB, dC, dA_log, dD, db_dt, dstate, bound: dict of the same)"""
    u, dt, A_log, B, C, dy, D, z, b_dt, state, dend = _f64(u, dt, A_log, B, C, dy, D, z, b_dt, state, dend)
    T, E = u.shape
    N = A_log.shape[1]
    A = -np.exp(A_log)
    D = np.zeros(E) if D is None else D
    v = dt if b_dt is None else dt + b_dt
    d, sv = softplus(v), sigmoid(v)
    sz = None if z is None else sigmoid(z)
    gate = np.ones_like(u) if z is None else z * sz
    dgate = None if z is None else sz * (1 + z * (1 - sz))
    n = len(offs) - 1
    o = dict(du=np.zeros((T, E)), ddt=np.zeros((T, E)), dz=np.zeros((T, E)), dB=np.zeros((T, N)), dC=np.zeros((T, N)),
             dA_log=np.zeros((E, N)), dD=np.zeros(E), db_dt=np.zeros(E), dstate=np.zeros((n, E, N)))
    m = {k: np.zeros_like(a) for k, a in o.items()}  # the same with every term's absolute value
    longest = 0.0
    for i in range(n):
        lo, hi = offs[i], offs[i + 1]
        S = [np.zeros((E, N)) if state is None else state[i]]
        M = [np.abs(S[0])]
        total = np.zeros((E, N))
        for t in range(lo, hi):
            a = np.exp(d[t][:, None] * A)
            S.append(a * S[-1] + (d[t] * u[t])[:, None] * B[t])
            M.append(a * M[-1] + np.abs((d[t] * u[t])[:, None] * B[t]))
            total += np.abs(d[t][:, None] * A)
        longest = max(longest, total.max() if hi > lo else 0.0)
        g = np.zeros((E, N)) if dend is None else dend[i].copy()
        ga = np.abs(g)
        for t in reversed(range(lo, hi)):
            k = t - lo
            a = np.exp(d[t][:, None] * A)
            q = dy[t] * gate[t]
            full, size = (S[k + 1] * C[t]).sum(1) + D * u[t], (M[k + 1] * np.abs(C[t])).sum(1) + np.abs(D * u[t])
            if z is not None:
                o["dz"][t] = dy[t] * full * dgate[t]
                m["dz"][t] = np.abs(dy[t]) * size * sz[t] * (1 + np.abs(z[t]))
            g = g + q[:, None] * C[t]
            ga = ga + np.abs(q[:, None] * C[t])
            o["dC"][t] = (q[:, None] * S[k + 1]).sum(0)
            m["dC"][t] = (np.abs(q)[:, None] * M[k + 1]).sum(0)
            o["dB"][t] = (g * (d[t] * u[t])[:, None]).sum(0)
            m["dB"][t] = (ga * np.abs(d[t] * u[t])[:, None]).sum(0)
            gB, gBa = (g * B[t]).sum(1), (ga * np.abs(B[t])).sum(1)
            gs, gsa = g * a * S[k], ga * a * M[k]
            o["du"][t] = D * q + d[t] * gB
            m["du"][t] = np.abs(D * q) + d[t] * gBa
            o["ddt"][t] = ((gs * A).sum(1) + u[t] * gB) * sv[t]
            m["ddt"][t] = ((gsa * -A).sum(1) + np.abs(u[t]) * gBa) * sv[t]
            o["dA_log"] += gs * d[t][:, None] * A
            m["dA_log"] += gsa * d[t][:, None] * -A
            o["dD"] += q * u[t]
            m["dD"] += np.abs(q * u[t])
            o["db_dt"] += o["ddt"][t]
            m["db_dt"] += m["ddt"][t]
            g, ga = g * a, ga * a
        o["dstate"][i], m["dstate"][i] = g, ga
    # One path: a product of decays, whose exponents sum to `longest` at most and are off by d's
    # error and four roundings each (|x e^-x| and the decays' own factor aside, an overestimate),
    # its L factors' roundings forwards and back, the activations, and sums of N or, for dB,
    # dC and the parameters, of E or T terms.
    L = int(max(np.diff(offs), default=0))
    rel_v = (EPS * np.abs(v) / d).max() if T else 0.0
    path = (longest + 4) * (EPS_ACT + rel_v + 4 * EPS) + (4 * L + N + 16) * EPS
    long_sum = dict(dB=E, dC=E, dA_log=T, dD=T, db_dt=T)
    return dict(o, bound={k: a * (path + long_sum.get(k, 0) * EPS) for k, a in m.items()})
