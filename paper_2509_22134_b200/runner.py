"""Convenience drivers: one full training pass (build tree -> reward -> surrogate gradient), and the
decoding step that a trained draft serves (append -> attention in every layer -> verify -> commit).

Each owns a library context and the caller-side buffers; every step is one C-ABI call.
"""
from __future__ import annotations

import numpy as np
import torch

from . import binding as gto
from . import synth


class GtoPass:
    def __init__(self, w: synth.Workload, device="cuda:0", reward_agg=gto.GTO_AGG_LSE, flags=0):
        self.w = w
        self.device = torch.device(device)
        idx = self.device.index if self.device.index is not None else torch.cuda.current_device()
        self.cfg = gto.make_config(w.B, w.D, w.k, w.g, w.m, w.V_draft, w.V_target, w.dtype, G=w.G,
                                   eta=w.eta, clip_eps=w.clip_eps, std_delta=w.std_delta,
                                   grad_scale=w.grad_scale, reward_agg=reward_agg, flags=flags)
        self.ctx = gto.gto_create(self.cfg, idx)
        self.tree = gto.alloc_tree(self.cfg, self.device)
        self.reward = gto.alloc_reward(self.cfg, self.device)
        self.stats = gto.alloc_grad_stats(self.cfg, self.device)
        self.grad = torch.empty((w.B, w.D, w.V_draft), dtype=w.torch_dtype, device=self.device)
        self.old_logp = torch.zeros((w.B, w.D), dtype=torch.float32, device=self.device)

    def close(self):
        if self.ctx is not None:
            gto.gto_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # ---- the three entry points
    def build_tree(self, draft, stream=None):
        gto.gto_build_tree(self.ctx, draft, self.tree, stream)

    def tree_reward(self, target, d2t, stream=None):
        gto.gto_tree_reward(self.ctx, self.tree, target, d2t, self.reward, stream)

    def tree_reward_host(self, target_host, target_dev, d2t, stream=None) -> int:
        return gto.gto_tree_reward_host(self.ctx, self.tree, target_host, target_dev, d2t, self.reward,
                                        stream)

    def surrogate_grad(self, draft, stream=None):
        gto.gto_group_surrogate_grad(self.ctx, draft, self.tree, self.reward, self.old_logp,
                                     self.grad, self.stats, stream)

    def set_old_logp_from_path(self, b0: int = 0):
        """Old-policy log-probabilities of the accepted paths (an input of the gradient
        call): the reported path log-probabilities plus the seeded perturbation."""
        r = self.reward
        old = synth.old_logp_from_path(self.w, r["path_logp"].cpu().numpy().astype(np.float64),
                                       r["path_row"].cpu().numpy(), r["path_token"].cpu().numpy(),
                                       r["path_len"].cpu().numpy(), b0=b0)
        self.old_logp.copy_(torch.from_numpy(old).to(torch.float32))

    def step(self, draft, target, d2t, stream=None):
        """One pass with the current old_logp buffer."""
        self.build_tree(draft, stream)
        self.tree_reward(target, d2t, stream)
        self.surrogate_grad(draft, stream)

    def token_loss(self, draft, target, d2t, weight: float = 1.0, stream=None):
        """Token-level loss on the root rows; allocates its outputs on first use."""
        if not hasattr(self, "token_stats"):
            self.token_stats = gto.alloc_token_stats(self.cfg, self.device)
            self.grad_root = torch.empty((self.w.B, self.w.V_draft), dtype=self.w.torch_dtype,
                                         device=self.device)
        gto.gto_token_loss(self.ctx, draft, target, d2t, self.tree, weight, self.grad_root,
                           self.token_stats, stream)

    def token_loss_accumulate(self, draft, target, d2t, weight: float = 1.0, stream=None):
        """Token-level loss added into slice [b, 0, :] of the surrogate gradient buffer."""
        if not hasattr(self, "token_stats"):
            self.token_stats = gto.alloc_token_stats(self.cfg, self.device)
        gto.gto_token_loss_accumulate(self.ctx, draft, target, d2t, self.tree, self.reward, self.stats,
                                      weight, self.grad, self.token_stats, stream)

    def status(self) -> int:
        return gto.gto_device_status(self.ctx)

    def launches(self) -> int:
        return gto.gto_launch_count(self.ctx)


def draft_trees(tree: dict, b0: int = 0, b1: int | None = None, t: int = 0) -> dict:
    """The decoding arrays of trees [b0, b1) that gto_build_tree made (t = 0: the current draft's), as views."""
    return {n: tree[n][t, b0:b1] for n in ("node_token", "node_parent", "node_depth", "node_slot", "node_mask")}


class DecodeStep:
    """Decoding with draft trees: S sequences over a paged cache of n_layers layers.

    A step is begin(), attend() for every layer, verify() and commit(), all on the current stream; nothing
    waits for the device, and a step can be captured into a CUDA graph.  kv_len holds the cached entries of
    every sequence; page_table is the caller's to fill (a page may be added between steps).
    """

    def __init__(self, cfg: gto.gto_decode_config, n_layers: int, inv_freq, device="cuda:0"):
        self.cfg, self.device = cfg, torch.device(device)
        idx = self.device.index if self.device.index is not None else torch.cuda.current_device()
        self.ctx = gto.gto_decode_create(cfg, idx)
        dtype = {gto.GTO_BF16: torch.bfloat16, gto.GTO_F16: torch.float16,
                 gto.GTO_F32: torch.float32}[cfg.kv_dtype]
        pool = (n_layers, cfg.n_pages, cfg.page_size, cfg.n_kv_heads, cfg.head_dim)
        self.k_cache = torch.zeros(pool, dtype=dtype, device=self.device)
        self.v_cache = torch.zeros(pool, dtype=dtype, device=self.device)
        self.page_table = torch.full((cfg.S, cfg.max_pages), -1, dtype=torch.int32, device=self.device)
        self.kv_len = torch.zeros(cfg.S, dtype=torch.int32, device=self.device)
        self.inv_freq = torch.as_tensor(inv_freq, dtype=torch.float64, device=self.device)
        self.verdict = gto.alloc_verdict(cfg, self.device)
        self.q_rotated = torch.empty((cfg.T, cfg.n_q_heads, cfg.head_dim), dtype=dtype, device=self.device)
        self.batch = None
        self.tokens = None  # rows that this step's layers were given, the fewest

    def close(self):
        if self.ctx is not None:
            gto.gto_decode_destroy(self.ctx)
            self.ctx = None

    def begin(self, q_start, trees: dict | None = None):
        """The tokens of this step: chunk s is q_start[s] .. q_start[s+1], what comes before the draft tree (a
        prompt, or the last step's token) and then the tree's nodes."""
        self.batch = {"q_start": q_start, "kv_len": self.kv_len + torch.diff(q_start), "page_table": self.page_table}
        self.tokens = None
        if trees is not None:
            self.batch.update({n: trees[n] for n in ("node_mask", "node_depth", "n_nodes") if n in trees})

    def attend(self, layer: int, q, k, v, out, lse=None, q_norm=None, k_norm=None):
        """Keys and values of one layer into its cache, then the attention of the step's tokens over it."""
        rotated = self.q_rotated[:q.shape[0]]
        self.tokens = q.shape[0] if self.tokens is None else min(self.tokens, q.shape[0])
        gto.gto_kv_append(self.ctx, self.batch, q, k, v, rotated, self.k_cache[layer], self.v_cache[layer],
                          self.inv_freq, q_norm, k_norm)
        gto.gto_tree_attention(self.ctx, self.batch, rotated, self.k_cache[layer], self.v_cache[layer], out, lse)

    def verify(self, trees: dict, target, d2t, temperature, u_node, u_bonus) -> dict:
        gto.gto_verify_tree(self.ctx, trees, target, d2t, temperature, u_node, u_bonus, self.verdict)
        return self.verdict

    def commit(self):
        """Keeps the accepted nodes' entries in all layers; kv_len then counts them.  A sequence that the other calls
        skipped keeps its kv_len."""
        gto.gto_kv_commit(self.ctx, self.batch, self.verdict, self.k_cache, self.v_cache, self.kv_len, tokens=self.tokens)

    def status(self) -> int:
        return gto.gto_decode_status(self.ctx)

    def launches(self) -> int:
        return gto.gto_decode_launch_count(self.ctx)
