"""How far an attention's results may be from fp64, entry by entry, so that a coarser kernel or a lost entry does not pass.

The errors counted (e: cache entry, d: dimension, half: half a step of the type, relative):
  score       a sum of dh products in fp32.  Roundings are 2^-24 of partial sums (a tensor core may cut, 2^-23), which are about
              sqrt(sum_d (q_d k_d)^2); dh of them add up like a random walk: sigma below sqrt(dh) 2^-24 of that, 8 sigma are
              allowed.  And 2^-22 |score| for the rounding of its product with the scale, and of the exponential's argument.
  weight      the exponential errs by 2^-22, the sums (of tens to hundreds of partial sums) by less than 2^-21: 2^-20 in all.
  16 bits     weights are rounded to the type, independently: |error| <= half p_e, and the sum of n independent errors passes
              7 half sqrt(sum (p_e v_e)^2) with probability 2 exp(-49/2) = 5e-11 (Hoeffding); half sum p_e |v_e| at most.
  result      rounded once: half |out|, and where the type's numbers are subnormal half of their step (fp16: numbers below 2^-14
              lie 2^-24 apart, whatever their size, so that rounding one errs by up to 2^-25).
A first-order change of scores by s_e changes out by sum_e p_e s_e (v_e - out) and the log-sum-exp by sum_e p_e s_e.

Over all results the root mean square is held too: the terms but the last are at least 4 standard deviations each, and
a rounding's is half |out| / sqrt(3)."""
from __future__ import annotations

import numpy as np
import torch

import decode_cases as dc


def expected(c, scale, device="cpu", drop=None, weights=None, dtype=None):
    """fp64 attention of the batch with its bounds: dict of out, lse, tol, lse_tol, rest (tol without the last rounding).
    drop(s, L) names entries that are left out, weights maps unnormalised weights to what they are rounded to, dtype
    rounds queries, keys and values: for results as a wrong kernel would give them."""
    load = lambda x: torch.from_numpy(np.nan_to_num(x) if dtype is None else dc.round_to(np.nan_to_num(x), dtype)).to(device)
    q, k, v = load(c.q), load(c.k), load(c.v)
    half = dc.HALF_STEP[c.dtype]
    h, rep = c.host, c.hq // c.hkv
    r = {n: [] for n in ("out", "lse", "rest", "lse_tol")}
    for s in range(c.S):
        q0, q1, L = int(h["q_start"][s]), int(h["q_start"][s + 1]), int(h["kv_len"][s])
        n = q1 - q0
        if n == 0:
            continue
        nodes = 0 if not c.g else int(h["n_nodes"][s]) if "n_nodes" in h else c.g
        e = torch.arange(L, device=device)
        table = torch.from_numpy(h["page_table"][s]).to(device).long()
        see = e[None] <= (L - n + torch.arange(n, device=device))[:, None]
        if nodes:
            see[n - nodes:, L - nodes:] = torch.from_numpy(h["node_mask"][s][:nodes, :nodes]).to(device)
        if drop is not None:
            see[:, torch.as_tensor(drop(s, L), dtype=torch.long, device=device)] = False
        kk = k[table[e // c.page], e % c.page].repeat_interleave(rep, 1).permute(1, 2, 0)     # [hq, dh, L]
        vv = v[table[e // c.page], e % c.page].repeat_interleave(rep, 1).permute(1, 0, 2)     # [hq, L, dh]
        qq = q[q0:q1].permute(1, 0, 2)
        x = (qq @ kk * scale).masked_fill(~see, float("-inf"))
        top = x.amax(2, keepdim=True)
        top = torch.where(torch.isinf(top), 0.0, top)
        w = torch.exp(x - top)
        total = w.sum(2, keepdim=True)
        lse = torch.where(total > 0, top + total.log(), float("-inf"))[..., 0]
        inv = torch.where(total > 0, 1 / total, 0.0)
        p = w * inv
        out = ((w if weights is None else weights(w)) @ vv) * inv
        step = 8 * c.dh ** 0.5 * 2.0 ** -24 * scale * ((qq * qq) @ (kk * kk)).sqrt() + 2.0 ** -22 * torch.where(see, x, 0.0).abs()
        spread = p @ vv.abs()
        rest = (p * step) @ vv.abs() + (p * step).sum(2, keepdim=True) * out.abs() + 2.0 ** -20 * spread
        if c.dtype != "f32":
            rest = rest + torch.minimum(half * spread, 7 * half * ((p * p) @ (vv * vv)).sqrt())
        r["out"].append(out.permute(1, 0, 2))
        r["rest"].append(rest.permute(1, 0, 2))
        r["lse"].append(lse.T)
        r["lse_tol"].append((p * step).sum(2).T + 2.0 ** -19 + 2.0 ** -22 * torch.where(torch.isinf(lse), 0.0, lse.abs()).T)
    r = {n: torch.cat(x).cpu().numpy() for n, x in r.items()}
    r["half"], r["subnormal"] = half, 2.0 ** -25 if c.dtype == "f16" else 1e-30
    return r


def misses(want, out, lse):
    """What is wrong with results out [n, hq, dh] and lse [n, hq] (fp64 numpy): a list of texts, empty where nothing is."""
    bad = []
    err = np.abs(out - want["out"])
    tol = want["rest"] + want["half"] * np.abs(want["out"]) + want["subnormal"]
    if not np.all(err <= tol):                                     # (NaN too)
        part = np.nan_to_num(err / tol, nan=np.inf)
        bad.append("out: %.3g of its tolerance at %s" % (part.max(), np.unravel_index(np.argmax(part), part.shape)))
    limit = np.sqrt(np.mean((want["half"] * np.abs(want["out"]) / 3 ** 0.5) ** 2 + (want["rest"] / 4) ** 2))
    rms = np.sqrt(np.mean(err ** 2))
    if not rms <= limit:
        bad.append("out: rms error %.3g, limit %.3g" % (rms, limit))
    empty = np.isneginf(want["lse"])
    if not np.array_equal(np.isneginf(lse), empty):
        bad.append("lse: rows that see nothing")
    err = np.abs(lse[~empty] - want["lse"][~empty])
    if not np.all(err <= want["lse_tol"][~empty]):
        bad.append("lse: %.3g of its tolerance" % np.nan_to_num(err / want["lse_tol"][~empty], nan=np.inf).max())
    return bad
