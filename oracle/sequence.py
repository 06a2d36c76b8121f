"""fp64 oracle of the sequence operators: the causal convolution + SiLU and the
selective scan with carried states, and their gradients (sections 5.2 and 6 of the
paper's Mamba block, token by token from the definitions).

Sequences are packed: sequence i is rows offs[i] .. offs[i+1]-1. `state` holds one
start state per sequence (None: zeros); end states are returned per sequence.

Every function also returns, under "bound", how far fp32 arithmetic of the
same formulas may be off, element by element: every term's absolute value times
the relative error with which it is formed (see EPS_*), to first order.
"""
from __future__ import annotations

import numpy as np

EPS = 2.0 ** -24        # one fp32 rounding
EPS_ACT = 4e-6          # SiLU, sigmoid and softplus in fp32, relative
TINY = 2.0 ** -126      # a decay below it, or a product of decays, may be zero in fp32


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


def conv_backward(x, w, b, du, offs, state=None, dend=None, chain=None):
    """-> dict(dx, dw, db, dstate, bound: dict of the same); chain: the most additions that a
    term of dw or db passes through (None: one for every token)"""
    x, w, b, du, state, dend = _f64(x, w, b, du, state, dend)
    E, K = w.shape
    b = np.zeros(E) if b is None else b
    chain = len(x) if chain is None else chain
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
            bw += (np.abs(win) * (e + (chain + 2) * EPS * np.abs(g))).T
            db += g
            bb += e + (chain + 2) * EPS * np.abs(g)
        dx[lo:hi], bx[lo:hi] = g_ext[K - 1:], g_abs[K - 1:]
        ds[i], bs[i] = g_ext[:K - 1], g_abs[:K - 1]
    return dict(dx=dx, dw=dw, db=db, dstate=ds, bound=dict(dx=bx, dw=bw, db=bb, dstate=bs))


def _steps(dt, b_dt):
    """v = dt + b_dt, d = softplus(v), sigmoid(v), and the relative error of d in fp32: v rounds
    once, which moves d by softplus'(v) = sigmoid(v) as much, and softplus is off by EPS_ACT."""
    v = dt if b_dt is None else dt + b_dt
    d, sv = softplus(v), sigmoid(v)
    return v, d, sv, EPS_ACT + EPS * np.abs(v) * sv / d


def _decay(d, rel, A, A_log, length):
    """One token's decays exp(d A) [E, N] and their error: TINY and, relative, the exponent's own (d; A,
    whose exponent A_log rounds twice, and three roundings more; the product; where decays are multiplied
    by adding up their steps, a rounding per token of the sequence) times the exponent, and six
    roundings: exp2 (one unit, two roundings), the product with a state, the sum that it enters, and as
    many again where a sequence's parts are joined."""
    x = d[:, None] * A
    a = np.exp(x)
    return a, a * (np.abs(x) * (rel[:, None] + (2 * np.abs(A_log) + 5 + length) * EPS) + 6 * EPS) + TINY


def scan(u, dt, A_log, B, C, offs, D=None, z=None, b_dt=None, state=None):
    """-> dict(y, end, bound: dict(y, end))

    The states' bound runs along with them: a step passes on the error that is there and adds
    the decay's and the input's errors, times what these multiply with every term's
    absolute value (as parts of a sequence may be summed apart)."""
    u, dt, A_log, B, C, D, z, b_dt, state = _f64(u, dt, A_log, B, C, D, z, b_dt, state)
    T, E = u.shape
    N = A_log.shape[1]
    A = -np.exp(A_log)
    D = np.zeros(E) if D is None else D
    _, d, _, rel = _steps(dt, b_dt)
    n = len(offs) - 1
    y, end = np.zeros_like(u), np.zeros((n, E, N))
    by, be = np.zeros_like(u), np.zeros((n, E, N))
    gate = np.ones_like(u) if z is None else z * sigmoid(z)
    for i in range(n):
        s = np.zeros((E, N)) if state is None else state[i].copy()
        size, err = np.abs(s), np.zeros((E, N))
        for t in range(offs[i], offs[i + 1]):
            a, ea = _decay(d[t], rel[t], A, A_log, offs[i + 1] - offs[i])
            x = (d[t] * u[t])[:, None] * B[t]
            err = a * err + ea * size + np.abs(x) * (rel[t][:, None] + 4 * EPS)
            s, size = a * s + x, a * size + np.abs(x)
            err += 2 * EPS * size
            full = (s * C[t]).sum(1) + D * u[t]
            terms = (np.abs(s * C[t])).sum(1) + np.abs(D * u[t])
            y[t] = full * gate[t]
            by[t] = ((np.abs(C[t]) * err).sum(1) + (N + 2) * EPS * terms) * np.abs(gate[t]) + EPS_ACT * np.abs(y[t])
        end[i], be[i] = s, err
    return dict(y=y, end=end, bound=dict(y=by, end=be))


def scan_backward(u, dt, A_log, B, C, dy, offs, D=None, z=None, b_dt=None, state=None, dend=None):
    """-> dict(du, ddt, dz, dB, dC, dA_log, dD, db_dt, dstate, bound: dict of the same)

    The bound of every element is a sum over what enters it: states S and adjoints g each with an
    error of their own (eS, eg, propagated as in scan), and every product with the relative errors of
    its factors, on sums of absolute values (M for S, ga for g)."""
    u, dt, A_log, B, C, dy, D, z, b_dt, state, dend = _f64(u, dt, A_log, B, C, dy, D, z, b_dt, state, dend)
    T, E = u.shape
    N = A_log.shape[1]
    A = -np.exp(A_log)
    absA, eA = -A, (2 * np.abs(A_log) + 4) * EPS
    D = np.zeros(E) if D is None else D
    v, d, sv, rel = _steps(dt, b_dt)
    e_sv = EPS_ACT + EPS * np.abs(v) * (1 - sv)  # sigmoid' / sigmoid = 1 - sigmoid
    sz = None if z is None else sigmoid(z)
    gate = np.ones_like(u) if z is None else z * sz
    dgate = None if z is None else sz * (1 + z * (1 - sz))
    e_gate = (0.0 if z is None else EPS_ACT) + 2 * EPS
    n = len(offs) - 1
    names = dict(du=(T, E), ddt=(T, E), dz=(T, E), dB=(T, N), dC=(T, N), dA_log=(E, N), dD=(E,), db_dt=(E,),
                 dstate=(n, E, N))
    o = {k: np.zeros(s) for k, s in names.items()}
    b = {k: np.zeros(s) for k, s in names.items()}

    def add(k, t, terms, errors, axis=None):
        """Terms of a sum over all channels (axis 0 of them) or all tokens, with their errors, and
        a rounding for each of the sum's additions."""
        more = errors + ((E if axis == 0 else T) + 2) * EPS * np.abs(terms)
        o[k][t] += terms if axis is None else terms.sum(axis)
        b[k][t] += more if axis is None else more.sum(axis)

    for i in range(n):
        lo, hi = offs[i], offs[i + 1]
        S = [np.zeros((E, N)) if state is None else state[i]]
        M, eS = [np.abs(S[0])], [np.zeros((E, N))]
        decays = []
        for t in range(lo, hi):
            a, ea = _decay(d[t], rel[t], A, A_log, hi - lo)
            x = (d[t] * u[t])[:, None] * B[t]
            S.append(a * S[-1] + x)
            M.append(a * M[-1] + np.abs(x))
            eS.append(a * eS[-1] + ea * M[-2] + np.abs(x) * (rel[t][:, None] + 4 * EPS) + 2 * EPS * M[-1])
            decays.append((a, ea))
        g = np.zeros((E, N)) if dend is None else dend[i].copy()
        ga, eg = np.abs(g), np.zeros((E, N))
        for t in reversed(range(lo, hi)):
            k = t - lo
            a, ea = decays[k]
            q = dy[t] * gate[t]
            aq, aC, aB, au = np.abs(q), np.abs(C[t]), np.abs(B[t]), np.abs(u[t])
            if z is not None:
                full, terms = (S[k + 1] * C[t]).sum(1) + D * u[t], (M[k + 1] * aC).sum(1) + np.abs(D * u[t])
                o["dz"][t] = dy[t] * full * dgate[t]
                # SiLU' = sg (1 + z (1 - sg)): sg's relative error on both
                b["dz"][t] = np.abs(dy[t]) * (((eS[k + 1] * aC).sum(1) + (N + 4) * EPS * terms) * np.abs(dgate[t]) +
                                              terms * (EPS_ACT * sz[t] * (1 + np.abs(z[t])) + 4 * EPS))
            x = q[:, None] * C[t]
            g, ga, eg = g + x, ga + np.abs(x), eg + np.abs(x) * (e_gate + EPS)
            eg = eg + EPS * ga
            step = (d[t] * u[t])[:, None]
            add("dC", t, q[:, None] * S[k + 1], aq[:, None] * (eS[k + 1] + M[k + 1] * (e_gate + EPS)), 0)
            add("dB", t, g * step, (eg + ga * (rel[t][:, None] + 3 * EPS)) * np.abs(step), 0)
            gB, gBa = (g * B[t]).sum(1), (ga * aB).sum(1)
            egB = (eg * aB).sum(1) + (N + 1) * EPS * gBa
            gs, gsa = g * a * S[k], ga * a * M[k]
            egs = a * (eg * M[k] + ga * eS[k]) + ga * M[k] * ea + 2 * EPS * gsa
            o["du"][t] = D * q + d[t] * gB
            b["du"][t] = np.abs(D * q) * (e_gate + 2 * EPS) + d[t] * (egB + gBa * (rel[t] + 3 * EPS))
            dd, dda = (gs * A).sum(1) + u[t] * gB, (gsa * absA).sum(1) + au * gBa
            edd = ((egs + gsa * (eA + (N + 2) * EPS)) * absA).sum(1) + au * egB + 3 * EPS * dda
            ddt, eddt = dd * sv[t], edd * sv[t] + dda * sv[t] * (e_sv[t] + 2 * EPS)
            o["ddt"][t], b["ddt"][t] = ddt, eddt
            add("dA_log", slice(None), gs * d[t][:, None] * A,
                (egs + gsa * (rel[t][:, None] + eA + 3 * EPS)) * d[t][:, None] * absA)
            add("dD", slice(None), q * u[t], aq * au * (e_gate + EPS))
            add("db_dt", slice(None), ddt, eddt)
            g, ga, eg = g * a, ga * a, a * eg + ga * ea
        o["dstate"][i], b["dstate"][i] = g, eg
    return dict(o, bound=b)
