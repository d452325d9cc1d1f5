"""Random batches for the decoding-step tests: shuffled pages, ragged chunks, draft trees, unused memory poisoned with NaN."""
from __future__ import annotations

import numpy as np
import torch

TORCH = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
HALF_STEP = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}   # half a step, relative


def round_to(x, dtype):
    """Values a tensor of that type can hold, as fp64."""
    return torch.tensor(np.asarray(x)).to(TORCH[dtype]).double().numpy()


def random_tree(rng, g, D):
    """(parent, depth, mask): parents before children, depth at most D."""
    parent, depth = np.full(g, -1, np.int32), np.ones(g, np.int32)
    mask = np.eye(g, dtype=bool)
    for n in range(1, g):
        a = int(rng.integers(-1, n))
        if a >= 0 and depth[a] < D:
            parent[n], depth[n] = a, depth[a] + 1
            mask[n] |= mask[a]
    return parent, depth, mask


def words(mask):
    """bool [S, g, g] -> int64 words [S, g, W]."""
    S, g, _ = mask.shape
    W = (g + 63) // 64
    out = np.zeros((S, g, W), np.uint64)
    for a in range(g):
        out[:, :, a // 64] |= mask[:, :, a].astype(np.uint64) << np.uint64(a % 64)
    return out.view(np.int64)


class Case:
    """One batch on the host (fp64 values that the type can hold) and on the device."""

    def __init__(self, q_lens, kv_lens, hq, hkv, dh, page, dtype, g=0, D=1, n_nodes=None, seed=0, spare=3, device="cuda:0",
                 head_major=False, poison=float("nan"), scale=1.0):
        rng = self.rng = np.random.default_rng(seed)
        S = len(q_lens)
        self.S, self.g, self.D, self.page, self.dtype = S, g, D, page, dtype
        self.hq, self.hkv, self.dh = hq, hkv, dh
        start = np.concatenate([[0], np.cumsum(q_lens)]).astype(np.int32)
        self.n = int(start[-1])
        self.T = self.n + spare
        need = [-(-L // page) for L in kv_lens]
        self.max_pages = max(max(need), 1) + 1
        self.n_pages = sum(need) + 2
        table = np.full((S, self.max_pages), 2 ** 30, np.int32)     # never to be followed
        order = rng.permutation(self.n_pages).astype(np.int32)
        at = 0
        for s in range(S):
            table[s, :need[s]] = order[at:at + need[s]]
            at += need[s]
        self.host = dict(q_start=start, kv_len=np.array(kv_lens, np.int32), page_table=table)
        dev = dict(q_start=start, kv_len=self.host["kv_len"], page_table=table)
        if g:
            trees = [random_tree(rng, g, D) for _ in range(S)]
            self.parent = np.stack([t[0] for t in trees])
            self.host["node_depth"] = np.stack([t[1] for t in trees])
            self.host["node_mask"] = np.stack([t[2] for t in trees])
            dev["node_depth"], dev["node_mask"] = self.host["node_depth"], words(self.host["node_mask"])
            if n_nodes is not None:
                self.host["n_nodes"] = dev["n_nodes"] = np.array(n_nodes, np.int32)
        self.batch = {k: torch.from_numpy(np.ascontiguousarray(v)).to(device) for k, v in dev.items()}
        self.q = round_to(rng.normal(size=(self.T, hq, dh)) * scale, dtype)
        pool = (self.n_pages, page, hkv, dh)
        self.k, self.v = round_to(rng.normal(size=pool) * scale, dtype), round_to(rng.normal(size=pool), dtype)
        # memory that belongs to no entry
        used = np.zeros((self.n_pages, page), bool)
        for s in range(S):
            e = np.arange(kv_lens[s])
            used[table[s][e // page], e % page] = True
        self.used = used
        if poison is not None:
            self.k[~used] = poison
            self.v[~used] = poison
        self.device, self.head_major = device, head_major
        self.dq = self.tensor(self.q)
        self.dk, self.dv = self.pool(self.k), self.pool(self.v)

    def tensor(self, x):
        return torch.from_numpy(np.ascontiguousarray(x)).to(self.device).to(TORCH[self.dtype])

    def pool(self, x):
        t = self.tensor(x)
        if self.head_major:     # [n_pages, heads, page, dh] in memory
            return t.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3)
        return t

    def ctx(self, gto, **kw):
        cfg = gto.make_decode_config(S=self.S, T=self.T, n_q_heads=self.hq, n_kv_heads=self.hkv, head_dim=self.dh,
                                     page_size=self.page, n_pages=self.n_pages, max_pages=self.max_pages, dtype=self.dtype,
                                     g=self.g, D=self.D, **kw)
        return gto.gto_decode_create(cfg, torch.device(self.device).index)

    def attention_on_device(self, scale):
        """What oracle.decode_oracle.attention gives, in fp64 on the device (for batches too long for its loops)."""
        q, k, v = (torch.from_numpy(x).to(self.device) for x in (self.q, self.k, self.v))
        out = torch.full((self.T, self.hq, self.dh), float("nan"), dtype=torch.float64, device=self.device)
        spread, lse = out.clone(), out[:, :, 0].clone()
        h = self.host
        for s in range(self.S):
            q0, q1, L = int(h["q_start"][s]), int(h["q_start"][s + 1]), int(h["kv_len"][s])
            n = q1 - q0
            if n == 0:
                continue
            nodes = 0 if not self.g else int(h["n_nodes"][s]) if "n_nodes" in h else self.g
            e = torch.arange(L, device=self.device)
            table = torch.from_numpy(h["page_table"][s]).to(self.device).long()
            see = e[None] <= (L - n + torch.arange(n, device=self.device))[:, None]
            if nodes:
                see[n - nodes:, L - nodes:] = torch.from_numpy(h["node_mask"][s][:nodes, :nodes]).to(self.device)
            rep = self.hq // self.hkv
            kk = k[table[e // self.page], e % self.page].repeat_interleave(rep, 1).permute(1, 2, 0)
            vv = v[table[e // self.page], e % self.page].repeat_interleave(rep, 1).permute(1, 0, 2)
            x = (q[q0:q1].permute(1, 0, 2) @ kk * scale).masked_fill(~see, float("-inf"))
            z = torch.logsumexp(x, 2)
            w = torch.where(torch.isinf(z)[:, :, None], 0.0, torch.exp(x - z[:, :, None]))
            out[q0:q1] = (w @ vv).permute(1, 0, 2)
            spread[q0:q1] = (w @ vv.abs()).permute(1, 0, 2)
            lse[q0:q1] = z.T
        return out.cpu().numpy(), lse.cpu().numpy(), spread.cpu().numpy()
