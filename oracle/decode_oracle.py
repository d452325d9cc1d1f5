"""Plain fp64 definitions of the decoding step over a draft tree (numpy, loops, CPU).

Shares no code with the CUDA path.  Arrays follow include/gto.h: a batch is a dict with q_start, kv_len,
page_table and, with trees, node_mask (bool [S, g, g]: node n sees node a), node_depth, n_nodes.
"""
from __future__ import annotations

import numpy as np


def chunks(batch, g=0):
    """(first token, tokens, entries, base, nodes, lead) of every sequence."""
    out = []
    for s in range(len(batch["kv_len"])):
        q0, q1, L = int(batch["q_start"][s]), int(batch["q_start"][s + 1]), int(batch["kv_len"][s])
        n = q1 - q0
        nodes = 0
        if n and ("node_mask" in batch or "node_depth" in batch):
            nodes = int(batch["n_nodes"][s]) if batch.get("n_nodes") is not None else g
        out.append((q0, n, L, L - n, nodes, n - nodes))
    return out


def slots(batch, s, entries, page_size):
    """(page, place) of the entries of sequence s."""
    e = np.asarray(entries)
    return np.asarray(batch["page_table"])[s][e // page_size], e % page_size


def rotate(x, position, inv_freq, interleaved=False, weight=None, eps=1e-6):
    """x [..., head_dim] at one position: optional norm, then rotation of the leading 2*len(inv_freq) dims."""
    x = np.array(x, dtype=np.float64)
    if weight is not None:
        x = x / np.sqrt(np.mean(x * x, -1, keepdims=True) + eps) * weight
    r = 2 * len(inv_freq)
    y = x.copy()
    for i, f in enumerate(inv_freq):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + r // 2)
        c, s = np.cos(position * f), np.sin(position * f)
        y[..., a] = x[..., a] * c - x[..., b] * s
        y[..., b] = x[..., b] * c + x[..., a] * s
    return y


def append(batch, q, k, v, k_cache, v_cache, page_size, inv_freq, g=0, interleaved=False, q_norm=None, k_norm=None,
           eps=1e-6):
    """Returns (q rotated, k cache, v cache); rows and entries that the batch does not name stay as they are."""
    q2 = None if q is None else np.array(q, dtype=np.float64)
    k_cache, v_cache = np.array(k_cache, dtype=np.float64), np.array(v_cache, dtype=np.float64)
    for s, (q0, n, L, base, nodes, lead) in enumerate(chunks(batch, g)):
        for i in range(n):
            pos = base + i if i < lead else base + lead - 1 + int(batch["node_depth"][s][i - lead])
            page, place = slots(batch, s, base + i, page_size)
            k_cache[page, place] = rotate(k[q0 + i], pos, inv_freq, interleaved, k_norm, eps)
            v_cache[page, place] = v[q0 + i]
            if q is not None:
                q2[q0 + i] = rotate(q[q0 + i], pos, inv_freq, interleaved, q_norm, eps)
    return q2, k_cache, v_cache


def attention(batch, q, k_cache, v_cache, page_size, scale, g=0):
    """(out, lse, spread) for the batch's tokens; spread[t, h, :] = sum_e p_e |v_e|, for error bounds.  Only visible
    entries are looked at.  Rows of other tokens are NaN."""
    T, hq, dh = q.shape
    hkv = k_cache.shape[2]
    out, spread = np.full((T, hq, dh), np.nan), np.full((T, hq, dh), np.nan)
    lse = np.full((T, hq), np.nan)
    for s, (q0, n, L, base, nodes, lead) in enumerate(chunks(batch, g)):
        for i in range(n):
            if i < lead:
                seen = np.arange(base + i + 1)
            else:
                row = np.asarray(batch["node_mask"])[s][i - lead][:nodes]
                seen = np.concatenate([np.arange(base + lead), base + lead + np.nonzero(row)[0]])
            page, place = slots(batch, s, seen.astype(np.int64), page_size)
            for h in range(hq):
                kv = h // (hq // hkv)
                x = scale * (k_cache[page, place, kv].astype(np.float64) @ q[q0 + i, h].astype(np.float64))
                if len(x) == 0:
                    out[q0 + i, h] = spread[q0 + i, h] = 0.0
                    lse[q0 + i, h] = -np.inf
                    continue
                top = x.max()
                w = np.exp(x - top)
                vv = v_cache[page, place, kv].astype(np.float64)
                out[q0 + i, h] = (w @ vv) / w.sum()
                spread[q0 + i, h] = (w @ np.abs(vv)) / w.sum()
                lse[q0 + i, h] = top + np.log(w.sum())
    return out, lse, spread


def verify(parent, token, rows, target, temperature, u_node, u_bonus, D, d2t=None):
    """One tree.  rows[n]: the target row after node n (-1: none); row 0 follows the root.  Returns (accepted nodes,
    their target ids, last token or -1, margin): margin is the distance of the closest decision from its border, as a
    probability."""
    cur, row, path, ids, margin = -1, 0, [], [], np.inf
    while True:
        z = np.asarray(target[row], dtype=np.float64)
        if np.isnan(z).any() or np.isposinf(z).any() or np.isneginf(z).all() or not 0 <= temperature < np.inf:
            return path, ids, -1, margin
        kids = [n for n in range(len(parent)) if parent[n] == cur]
        if temperature == 0:
            best = int(np.argmax(z))
        else:
            p = np.exp((z - z.max()) / temperature)
            p /= p.sum()
        mass, nxt = 1.0, None
        for n in kids:
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
            sums = np.cumsum(p)
            aim = u_bonus * sums[-1]
            v = int(np.searchsorted(sums, aim, side="right"))
            v = min(v, len(p) - 1)
            margin = min(margin, abs(sums[v] - aim), abs(aim - (sums[v - 1] if v else 0.0)) if aim > 0 else np.inf)
            return path, ids, v, margin
        path.append(nxt)
        ids.append(int(token[nxt]) if d2t is None else int(d2t[token[nxt]]))
        cur, row = nxt, int(rows[nxt])
        if row < 0:
            return path, ids, -1, margin
