"""fp64 oracle of beam search's selection and of the reordering of states, from the definitions."""
from __future__ import annotations

import numpy as np


def beam_select(logits, score, K, ended=None, temperature=1.0):
    """logits [G W, V], score [G, W]: the K best (beam, token) of each group by score + log p, highest
    first, equal ones by lower beam, a beam's own by logit, then by lower token. -> dict(parent, token, score) [G, K]"""
    logits, score = np.asarray(logits, np.float64), np.asarray(score, np.float64)
    G, W = score.shape
    parent, token = np.full((G, K), -1, np.int64), np.full((G, K), -1, np.int64)
    out = np.full((G, K), -np.inf)
    for g in range(G):
        cand = []
        for w in range(W):
            s = score[g, w]
            if not s > -np.inf:
                continue
            if ended is not None and ended[g, w] >= 0:
                cand.append((-s, w, 0, int(ended[g, w])))
                continue
            x = logits[g * W + w]
            x = np.where(np.isnan(x), -np.inf, x)
            m = x.max()
            if not np.isfinite(m):
                continue
            z = (x - m) / temperature
            lp = z - np.log(np.exp(z).sum())
            best = np.lexsort((np.arange(lp.size), -x))[:K]
            cand += [(-(s + lp[v]), w, i, int(v)) for i, v in enumerate(best) if lp[v] > -np.inf]
        for i, (s, w, _, v) in enumerate(sorted(cand)[:K]):
            parent[g, i], token[g, i], out[g, i] = g * W + w, v, -s
    return dict(parent=parent, token=token, score=out)


def beam_reorder(parent, slots, n_slots, pools):
    """-> (slots [G, W], the pools afterwards)"""
    G, W = parent.shape
    new, pools = np.full((G, W), -1, np.int64), [p.copy() for p in pools]
    for g in range(G):
        p = [x - g * W if g * W <= x < (g + 1) * W else None for x in parent[g]]
        free = [slots[g, w] for w in range(W) if w not in p]
        for i in range(W):
            if p[i] is not None and p[i] not in p[:i]:
                new[g, i] = slots[g, p[i]]
                continue
            new[g, i] = free.pop(0)
            if p[i] is not None and 0 <= new[g, i] < n_slots and 0 <= slots[g, p[i]] < n_slots:
                for pool in pools:
                    pool[new[g, i]] = pool[slots[g, p[i]]]
    return new, pools
