"""fp64 oracle of drawing under limits (temperature, top-k, top-p, min-p), one row and one tree at a time."""
from __future__ import annotations

import numpy as np


def kept(z, temperature, top_k=0, top_p=1.0, min_p=0.0):
    """(weights, ids that stay in falling order, margin) of a row; temperature > 0.  margin: how far, as a share of the
    mass, the decisions about top-p and min-p are from their borders (inf where an exact number decides)."""
    z = np.asarray(z, dtype=np.float64)
    x = (z - z.max()) / temperature
    w = np.where(x < -1000 * np.log(2.0), 0.0, np.exp(x))
    ids = np.argsort(-z, kind="stable")          # equal ones: the lowest id first
    ids = ids[z[ids] > -np.inf]
    if top_k > 0:
        ids = ids[:top_k]
    margin = np.inf
    if top_p < 1:
        sums = np.cumsum(w[ids])
        goal = top_p * sums[-1]
        n = max(1, int(np.searchsorted(sums, goal, side="left")) + 1)
        gaps = np.abs(sums - goal)[max(0, n - 2):n] / sums[-1]
        # (sums of equal weights of 1 are whole numbers: exact on both sides)
        margin = min(margin, gaps.min()) if not np.all(w[ids] == 1.0) else margin
        ids = ids[:n]
    if min_p > 0:
        p = min(max(min_p, 0.0), 1.0)
        n = max(1, int(np.searchsorted(-w[ids], -p, side="right")))
        if p < 1:
            margin = min(margin, np.abs(w[ids] - p).min())
        ids = ids[:n]
    return w, ids, margin


def sound(z, temperature, top_p=1.0, min_p=0.0):
    z = np.asarray(z, dtype=np.float64)
    return bool(0 <= temperature < np.inf and not np.isnan([top_p, min_p]).any()
                and not np.isnan(z).any() and not np.isposinf(z).any() and not np.isneginf(z).all())


def draw(p, u):
    """(the first id whose cumulative sum passes u times the whole, distance of that decision as a share of the mass)."""
    sums = np.cumsum(p)
    aim = u * sums[-1]
    v = min(int(np.searchsorted(sums, aim, side="right")), len(p) - 1)
    gap = abs(sums[v] - aim)
    if v and aim > 0:
        gap = min(gap, abs(aim - sums[v - 1]))
    return v, gap / sums[-1]


def sample(z, temperature, u, top_k=0, top_p=1.0, min_p=0.0):
    """(token, log-probability, how many stay, margin)."""
    if not sound(z, temperature, top_p, min_p):
        return -1, 0.0, 0, np.inf
    if temperature == 0:
        return int(np.argmax(z)), 0.0, 1, np.inf
    w, ids, margin = kept(z, temperature, top_k, top_p, min_p)
    p = np.zeros(len(w))
    p[ids] = w[ids]
    v, gap = draw(p, min(max(u, 0.0), 1 - 2.0 ** -24))
    return v, float(np.log(p[v] / p.sum())), len(ids), min(margin, gap)


def verify(parent, token, rows, target, temperature, u_node, u_bonus, D, d2t=None, top_k=0, top_p=1.0, min_p=0.0):
    """One tree, as decode_oracle.verify, under limits."""
    cur, row, path, ids, margin = -1, 0, [], [], np.inf
    while True:
        z = np.asarray(target[row], dtype=np.float64)
        if not sound(z, temperature, top_p, min_p):
            return path, ids, -1, margin
        if temperature == 0:
            best = int(np.argmax(z))
        else:
            w, stay, m = kept(z, temperature, top_k, top_p, min_p)
            margin = min(margin, m)
            p = np.zeros(len(w))
            p[stay] = w[stay] / w[stay].sum()
        mass, nxt = 1.0, None
        for n in [n for n in range(len(parent)) if parent[n] == cur]:
            x = int(token[n]) if d2t is None else int(d2t[token[n]])
            if temperature == 0:
                if x == best:
                    nxt = n
                    break
                continue
            margin = min(margin, abs(u_node[n] * mass - p[x])) if p[x] > 0 else margin
            if u_node[n] * mass < p[x]:
                nxt = n
                break
            mass -= p[x]
            p[x] = 0.0
        if nxt is None:
            if temperature == 0:
                return path, ids, best, margin
            v, gap = draw(p, u_bonus)
            return path, ids, v, min(margin, gap)
        path.append(nxt)
        ids.append(int(token[nxt]) if d2t is None else int(d2t[token[nxt]]))
        cur, row = nxt, int(rows[nxt])
        if row < 0:
            return path, ids, -1, margin
