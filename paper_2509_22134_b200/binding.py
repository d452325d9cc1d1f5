"""Binding of libgto.so: argument marshalling only, through ctypes, and through the extension _gto_decode
for the calls of a decoding step, where microseconds count.

The functions carry the names of the C entry points (include/gto.h) and take torch
tensors for device buffers; PyTorch supplies device memory and streams, every step of
the pass runs in the library's kernels.  Importing this module loads the library and
raises if it has not been built - there is no fallback path.  The extension is loaded by the
first decoding context (gto_decode_create), which raises if it has not been built for this
Python and PyTorch; the training pass does without it.
"""
from __future__ import annotations

import ctypes
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libgto.so")

GTO_OK = 0
GTO_F32, GTO_BF16, GTO_F16 = 0, 1, 2
GTO_AGG_LSE, GTO_AGG_MAX, GTO_AGG_MEAN = 0, 1, 2
GTO_FLAG_STD_UNBIASED, GTO_FLAG_NO_DEBIAS, GTO_FLAG_GRAD_LIVE_ROWS, GTO_FLAG_SEQ_ALL_NODES = 1, 2, 4, 8
GTO_FLAG_FORCE_ROW_SPLIT = 16
GTO_FLAG_PATH_MAX_EXPECTED = 32

if not os.path.exists(LIB_PATH):
    raise RuntimeError(
        f"{LIB_PATH} is missing: build it with `python -m paper_2509_22134_b200.build` "
        "(the GTO pass has no CPU or PyTorch fallback)")
_lib = ctypes.CDLL(LIB_PATH)
_native = None  # the extension, from the first decoding context on


def _load_native():
    global _native
    if _native is None:
        from .build import extension_key
        advice = "build it with `python -m paper_2509_22134_b200.build`"
        try:
            from . import _gto_decode
        except ImportError as e:
            raise RuntimeError(f"_gto_decode.so is missing or cannot be loaded ({e}): {advice}") from e
        if _gto_decode.built_for != extension_key():
            raise RuntimeError(f"_gto_decode.so was built for {_gto_decode.built_for}, this is {extension_key()}: {advice}")
        _native = _gto_decode
    return _native


class gto_config(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in
                ("B", "G", "D", "k", "g", "m", "V_draft", "V_target", "logit_dtype", "reward_agg")] + \
               [(n, ctypes.c_float) for n in ("eta", "clip_eps", "std_delta", "grad_scale")] + \
               [("flags", ctypes.c_uint32)]


_TREE_FIELDS = [("node_token", torch.int32), ("node_parent", torch.int32), ("node_depth", torch.int32),
                ("node_ctx_row", torch.int32), ("node_slot", torch.int32), ("node_pool", torch.int32),
                ("node_logp", torch.float32), ("node_score", torch.float64),
                ("node_mask", torch.int64), ("row_lse", torch.float64)]
_REWARD_FIELDS = [("reward", torch.float64), ("etree", torch.float64), ("n_leaves", torch.int32),
                  ("node_ptarget", torch.float32), ("node_pathprod", torch.float32),
                  ("node_L", torch.float32), ("row_lse_t", torch.float64),
                  ("row_argmax_t", torch.int32), ("path_len", torch.int32),
                  ("path_node", torch.int32), ("path_row", torch.int32),
                  ("path_token", torch.int32), ("path_logp", torch.float32)]
_TOKEN_FIELDS = [("loss", torch.float64), ("lse_t", torch.float64)]
_STATS_FIELDS = [("R", torch.float64), ("adv", torch.float64), ("ratio", torch.float64),
                 ("coeff", torch.float64), ("active", torch.int32), ("loss", torch.float64)]


def _struct(name, fields):
    return type(name, (ctypes.Structure,), {"_fields_": [(n, ctypes.c_void_p) for n, _ in fields]})


gto_tree = _struct("gto_tree", _TREE_FIELDS)
gto_reward = _struct("gto_reward", _REWARD_FIELDS)
gto_grad_stats = _struct("gto_grad_stats", _STATS_FIELDS)
gto_token_stats = _struct("gto_token_stats", _TOKEN_FIELDS)

_vp = ctypes.c_void_p
_lib.gto_create.argtypes = [ctypes.POINTER(_vp), ctypes.POINTER(gto_config), ctypes.c_int]
_lib.gto_destroy.argtypes = [_vp]
_lib.gto_build_tree.argtypes = [_vp, _vp, ctypes.POINTER(gto_tree), _vp]
_lib.gto_build_tree_noalloc.argtypes = [ctypes.POINTER(gto_config), ctypes.c_int, _vp,
                                        ctypes.POINTER(gto_tree), _vp]
_lib.gto_build_tree_noalloc.restype = ctypes.c_int
_lib.gto_tree_reward.argtypes = [_vp, ctypes.POINTER(gto_tree), _vp, _vp, ctypes.POINTER(gto_reward), _vp]
_lib.gto_tree_reward_host.argtypes = [_vp, ctypes.POINTER(gto_tree), _vp, _vp, _vp,
                                      ctypes.POINTER(gto_reward), _vp, ctypes.POINTER(ctypes.c_int64)]
_lib.gto_tree_reward_host.restype = ctypes.c_int
_lib.gto_group_surrogate_grad.argtypes = [_vp, _vp, ctypes.POINTER(gto_tree), ctypes.POINTER(gto_reward),
                                          _vp, _vp, ctypes.POINTER(gto_grad_stats), _vp]
_lib.gto_token_loss.argtypes = [_vp, _vp, _vp, _vp, ctypes.POINTER(gto_tree), ctypes.c_float, _vp,
                                ctypes.POINTER(gto_token_stats), _vp]
_lib.gto_token_loss.restype = ctypes.c_int
_lib.gto_token_loss_accumulate.argtypes = [_vp, _vp, _vp, _vp, ctypes.POINTER(gto_tree),
                                           ctypes.POINTER(gto_reward), ctypes.POINTER(gto_grad_stats),
                                           ctypes.c_float, _vp, ctypes.POINTER(gto_token_stats), _vp]
_lib.gto_token_loss_accumulate.restype = ctypes.c_int
_lib.gto_sample_groups.argtypes = [ctypes.c_int32, ctypes.c_int32, ctypes.c_int32,
                                   ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_int32)]
_lib.gto_sample_groups.restype = ctypes.c_int
_lib.gto_device_status.argtypes = [_vp, _vp, ctypes.POINTER(ctypes.c_int32)]
_lib.gto_launch_count.argtypes = [_vp]
_lib.gto_launch_count.restype = ctypes.c_int64
_lib.gto_kernel_timing.argtypes = [_vp, ctypes.c_int]
_lib.gto_kernel_times.argtypes = [_vp, _vp, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_int64)]
_lib.gto_status_string.argtypes = [ctypes.c_int]
_lib.gto_status_string.restype = ctypes.c_char_p
for _f in ("gto_create", "gto_destroy", "gto_build_tree", "gto_tree_reward",
           "gto_group_surrogate_grad", "gto_device_status", "gto_kernel_timing", "gto_kernel_times"):
    getattr(_lib, _f).restype = ctypes.c_int


GTO_DECODE_ROPE_INTERLEAVED, GTO_DECODE_CONTEXT_ROWS = 1, 2


class gto_decode_config(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in
                ("S", "T", "g", "D", "k", "n_q_heads", "n_kv_heads", "head_dim", "page_size", "n_pages",
                 "max_pages", "kv_dtype", "rope_dims", "V_draft", "V_target", "logit_dtype")] + \
               [(n, ctypes.c_float) for n in ("softmax_scale", "norm_eps")] + \
               [("flags", ctypes.c_uint32)]


class gto_batch(ctypes.Structure):
    _fields_ = [("S", ctypes.c_int32), ("T", ctypes.c_int32)] + \
               [(n, ctypes.c_void_p) for n in
                ("q_start", "kv_len", "page_table", "n_nodes", "node_mask", "node_depth")]


class gto_kv_cache(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p)] + \
               [(n, ctypes.c_int64) for n in ("k_page", "k_entry", "k_head", "k_layer",
                                              "v_page", "v_entry", "v_head", "v_layer")] + \
               [("n_layers", ctypes.c_int32)]


class gto_draft_tree(ctypes.Structure):
    _fields_ = [("S", ctypes.c_int32)] + \
               [(n, ctypes.c_void_p) for n in
                ("node_token", "node_parent", "node_depth", "node_slot", "n_nodes")]


class gto_verdict(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("accept_len", "path_node", "token")]


_lib.gto_decode_create.argtypes = [ctypes.POINTER(_vp), ctypes.POINTER(gto_decode_config), ctypes.c_int]
_lib.gto_decode_destroy.argtypes = [_vp]
_lib.gto_decode_status.argtypes = [_vp, _vp, ctypes.POINTER(ctypes.c_int32)]
_lib.gto_decode_launch_count.argtypes = [_vp]
_lib.gto_decode_launch_count.restype = ctypes.c_int64
for _f in ("gto_decode_create", "gto_decode_destroy", "gto_decode_status"):
    getattr(_lib, _f).restype = ctypes.c_int


class GtoError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where}: {gto_status_string(code)} (status {code})")


def gto_status_string(code: int) -> str:
    return _lib.gto_status_string(code).decode()


def _check(code: int, where: str):
    if code != GTO_OK:
        raise GtoError(code, where)


def _stream_ptr(stream) -> int:
    if stream is None:
        stream = torch.cuda.current_stream()
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _fill(struct_type, fields, bufs: dict):
    s = struct_type()
    for name, dtype in fields:
        t = bufs[name]
        assert t.is_cuda and t.is_contiguous() and t.dtype == dtype, name
        setattr(s, name, t.data_ptr())
    return s


def make_config(B, D, k, g, m, V_draft, V_target, dtype, G=2, eta=1.0, clip_eps=0.2,
                std_delta=1e-6, grad_scale=1.0, reward_agg=GTO_AGG_LSE, flags=0) -> gto_config:
    code = {torch.bfloat16: GTO_BF16, torch.float32: GTO_F32, torch.float16: GTO_F16,
            "bf16": GTO_BF16, "f32": GTO_F32, "f16": GTO_F16}[dtype]
    return gto_config(B, G, D, k, g, m, V_draft, V_target, code, reward_agg,
                      eta, clip_eps, std_delta, grad_scale, flags)


def gto_create(cfg: gto_config, device: int = 0) -> int:
    h = _vp()
    _check(_lib.gto_create(ctypes.byref(h), ctypes.byref(cfg), device), "gto_create")
    return h.value


def gto_destroy(ctx: int):
    _check(_lib.gto_destroy(ctx), "gto_destroy")


def alloc_tree(cfg: gto_config, device) -> dict:
    G, B, g, R = cfg.G, cfg.B, cfg.g, 1 + (cfg.D - 1) * cfg.k
    W = (g + 63) // 64
    shapes = {"node_mask": (G, B, g, W), "row_lse": (G, B, R)}
    return {n: torch.empty(shapes.get(n, (G, B, g)), dtype=dt, device=device) for n, dt in _TREE_FIELDS}


def alloc_reward(cfg: gto_config, device) -> dict:
    G, B, g, D, R = cfg.G, cfg.B, cfg.g, cfg.D, 1 + (cfg.D - 1) * cfg.k
    shapes = {"reward": (G, B), "etree": (G, B), "n_leaves": (G, B), "row_lse_t": (G, B, R),
              "row_argmax_t": (G, B, R), "path_len": (B,), "path_node": (B, D), "path_row": (B, D),
              "path_token": (B, D), "path_logp": (B, D)}
    return {n: torch.empty(shapes.get(n, (G, B, g)), dtype=dt, device=device) for n, dt in _REWARD_FIELDS}


def alloc_grad_stats(cfg: gto_config, device) -> dict:
    B = cfg.B
    return {n: torch.empty((B // cfg.m,) if n == "loss" else (B,), dtype=dt, device=device)
            for n, dt in _STATS_FIELDS}


def gto_build_tree(ctx: int, draft: torch.Tensor, tree: dict, stream=None):
    assert draft.is_cuda and draft.is_contiguous()
    t = _fill(gto_tree, _TREE_FIELDS, tree)
    _check(_lib.gto_build_tree(ctx, draft.data_ptr(), ctypes.byref(t), _stream_ptr(stream)),
           "gto_build_tree")


GTO_NOALLOC_MAX_ENTRIES = 1 << 20


def gto_build_tree_noalloc(cfg: gto_config, device: int, draft: torch.Tensor, tree: dict, stream=None):
    """gto_build_tree without a context and without any device allocation: for callers
    that must keep every device byte under their own allocator.  Raises GtoError(7) when
    G*B*R*k exceeds GTO_NOALLOC_MAX_ENTRIES."""
    assert draft.is_cuda and draft.is_contiguous()
    t = _fill(gto_tree, _TREE_FIELDS, tree)
    _check(_lib.gto_build_tree_noalloc(ctypes.byref(cfg), device, draft.data_ptr(), ctypes.byref(t),
                                       _stream_ptr(stream)), "gto_build_tree_noalloc")


def gto_tree_reward(ctx: int, tree: dict, target: torch.Tensor, d2t, reward: dict, stream=None):
    assert target.is_cuda and target.is_contiguous()
    if d2t is not None:
        assert d2t.is_cuda and d2t.dtype == torch.int32 and d2t.is_contiguous()
    t = _fill(gto_tree, _TREE_FIELDS, tree)
    r = _fill(gto_reward, _REWARD_FIELDS, reward)
    _check(_lib.gto_tree_reward(ctx, ctypes.byref(t), target.data_ptr(),
                                None if d2t is None else d2t.data_ptr(), ctypes.byref(r),
                                _stream_ptr(stream)), "gto_tree_reward")


def gto_tree_reward_host(ctx: int, tree: dict, target_host: torch.Tensor, target_dev: torch.Tensor,
                         d2t, reward: dict, stream=None) -> int:
    """gto_tree_reward with the target logits in (pinned) host memory: copies only the
    needed rows into target_dev.  Returns the number of rows copied."""
    assert not target_host.is_cuda and target_host.is_contiguous()
    assert target_dev.is_cuda and target_dev.is_contiguous()
    assert target_host.shape == target_dev.shape and target_host.dtype == target_dev.dtype
    if d2t is not None:
        assert d2t.is_cuda and d2t.dtype == torch.int32 and d2t.is_contiguous()
    t = _fill(gto_tree, _TREE_FIELDS, tree)
    r = _fill(gto_reward, _REWARD_FIELDS, reward)
    n = ctypes.c_int64(0)
    _check(_lib.gto_tree_reward_host(ctx, ctypes.byref(t), target_host.data_ptr(), target_dev.data_ptr(),
                                     None if d2t is None else d2t.data_ptr(), ctypes.byref(r),
                                     _stream_ptr(stream), ctypes.byref(n)), "gto_tree_reward_host")
    return int(n.value)


def gto_group_surrogate_grad(ctx: int, draft: torch.Tensor, tree: dict, reward: dict,
                             old_logp: torch.Tensor, grad: torch.Tensor, stats: dict, stream=None):
    assert old_logp.is_cuda and old_logp.dtype == torch.float32 and old_logp.is_contiguous()
    assert grad.is_cuda and grad.is_contiguous() and grad.dtype == draft.dtype
    t = _fill(gto_tree, _TREE_FIELDS, tree)
    r = _fill(gto_reward, _REWARD_FIELDS, reward)
    s = _fill(gto_grad_stats, _STATS_FIELDS, stats)
    _check(_lib.gto_group_surrogate_grad(ctx, draft.data_ptr(), ctypes.byref(t), ctypes.byref(r),
                                         old_logp.data_ptr(), grad.data_ptr(), ctypes.byref(s),
                                         _stream_ptr(stream)), "gto_group_surrogate_grad")


def alloc_token_stats(cfg: gto_config, device) -> dict:
    return {n: torch.empty((cfg.B,), dtype=dt, device=device) for n, dt in _TOKEN_FIELDS}


def gto_token_loss(ctx: int, draft: torch.Tensor, target: torch.Tensor, d2t, tree: dict, weight: float,
                   grad_root: torch.Tensor, stats: dict, stream=None):
    assert draft.is_cuda and draft.is_contiguous() and target.is_cuda and target.is_contiguous()
    assert grad_root.is_cuda and grad_root.is_contiguous() and grad_root.dtype == draft.dtype
    if d2t is not None:
        assert d2t.is_cuda and d2t.dtype == torch.int32 and d2t.is_contiguous()
    t = _fill(gto_tree, _TREE_FIELDS, tree)
    s = _fill(gto_token_stats, _TOKEN_FIELDS, stats)
    _check(_lib.gto_token_loss(ctx, draft.data_ptr(), target.data_ptr(),
                               None if d2t is None else d2t.data_ptr(), ctypes.byref(t),
                               ctypes.c_float(weight), grad_root.data_ptr(), ctypes.byref(s),
                               _stream_ptr(stream)), "gto_token_loss")


def gto_token_loss_accumulate(ctx: int, draft: torch.Tensor, target: torch.Tensor, d2t, tree: dict,
                              reward: dict, stats: dict, weight: float, grad: torch.Tensor,
                              token_stats: dict, stream=None):
    """gto_token_loss into slice [b, 0, :] of the surrogate's gradient buffer [B, D, V_draft]."""
    assert draft.is_cuda and draft.is_contiguous() and target.is_cuda and target.is_contiguous()
    assert grad.is_cuda and grad.is_contiguous() and grad.dtype == draft.dtype and grad.dim() == 3
    if d2t is not None:
        assert d2t.is_cuda and d2t.dtype == torch.int32 and d2t.is_contiguous()
    t = _fill(gto_tree, _TREE_FIELDS, tree)
    r = _fill(gto_reward, _REWARD_FIELDS, reward)
    g = _fill(gto_grad_stats, _STATS_FIELDS, stats)
    s = _fill(gto_token_stats, _TOKEN_FIELDS, token_stats)
    _check(_lib.gto_token_loss_accumulate(ctx, draft.data_ptr(), target.data_ptr(),
                                          None if d2t is None else d2t.data_ptr(), ctypes.byref(t),
                                          ctypes.byref(r), ctypes.byref(g), ctypes.c_float(weight),
                                          grad.data_ptr(), ctypes.byref(s), _stream_ptr(stream)),
           "gto_token_loss_accumulate")


def gto_sample_groups(s: int, m: int, K: int, u) -> list:
    """Start indices (1-based) of K non-overlapping groups of m adjacent positions (host only)."""
    uu = (ctypes.c_double * max(K, 1))(*[float(x) for x in list(u)[:K]])
    out = (ctypes.c_int32 * max(K, 1))()
    _check(_lib.gto_sample_groups(s, m, K, uu, out), "gto_sample_groups")
    return [int(out[i]) for i in range(K)]


def gto_device_status(ctx: int, stream=None) -> int:
    code = ctypes.c_int32(0)
    _check(_lib.gto_device_status(ctx, _stream_ptr(stream), ctypes.byref(code)), "gto_device_status")
    return code.value


def gto_launch_count(ctx: int) -> int:
    return int(_lib.gto_launch_count(ctx))


KERNEL_NAMES = ["draft_rows", "tree_build", "reward_plan", "target_rows", "tree_reward",
                "group_stats", "grad_rows", "token_loss"]   # GTO_K_* order


def gto_kernel_timing(ctx: int, enable: bool):
    _check(_lib.gto_kernel_timing(ctx, int(bool(enable))), "gto_kernel_timing")


def gto_kernel_times(ctx: int, stream=None) -> dict:
    """{kernel name: (total device ms, launches)} since the last call; synchronises."""
    n = len(KERNEL_NAMES)
    ms = (ctypes.c_double * n)()
    cnt = (ctypes.c_int64 * n)()
    _check(_lib.gto_kernel_times(ctx, _stream_ptr(stream), ms, cnt), "gto_kernel_times")
    return {name: (ms[i], cnt[i]) for i, name in enumerate(KERNEL_NAMES)}


# ---- one decoding step over a draft tree

_DTYPE_CODE = {torch.bfloat16: GTO_BF16, torch.float32: GTO_F32, torch.float16: GTO_F16,
               "bf16": GTO_BF16, "f32": GTO_F32, "f16": GTO_F16}


def make_decode_config(S, T=0, n_q_heads=0, n_kv_heads=0, head_dim=0, page_size=0, n_pages=0, max_pages=0,
                       dtype="bf16", g=0, D=1, k=0, V_draft=0, V_target=0, logit_dtype="bf16", softmax_scale=None,
                       rope_dims=None, norm_eps=1e-6, flags=0) -> gto_decode_config:
    """softmax_scale defaults to head_dim ** -0.5, rope_dims to the whole head."""
    if softmax_scale is None:
        softmax_scale = head_dim ** -0.5 if head_dim > 0 else 1.0
    if rope_dims is None:
        rope_dims = head_dim
    return gto_decode_config(S, T, g, D, k, n_q_heads, n_kv_heads, head_dim, page_size, n_pages, max_pages,
                             _DTYPE_CODE[dtype], rope_dims, V_draft, V_target, _DTYPE_CODE[logit_dtype], softmax_scale,
                             norm_eps, flags)


class DecodeCtx:
    """A decoding context: the library's handle and the configuration it was made with, which the
    calls below check their tensors against.  gto_decode_destroy (or the end of the object) frees it."""

    def __init__(self, handle: int, cfg: gto_decode_config, device: int):
        self.handle, self.cfg, self.index = handle, cfg, device
        self.native = _native.make(handle, bytes(cfg), device)

    def __del__(self):
        if self.handle and _lib is not None:
            _lib.gto_decode_destroy(self.handle)
            self.handle = self.native = None


def _stream_of(ctx: DecodeCtx, stream) -> int:
    """The given stream, else the current one of the context's device (which need not be the current device)."""
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(ctx.index)
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def gto_decode_create(cfg: gto_decode_config, device: int = 0) -> DecodeCtx:
    _load_native()
    h = _vp()
    _check(_lib.gto_decode_create(ctypes.byref(h), ctypes.byref(cfg), device), "gto_decode_create")
    return DecodeCtx(h.value, gto_decode_config.from_buffer_copy(cfg), device)


def gto_decode_destroy(ctx: DecodeCtx):
    handle, ctx.handle, ctx.native = ctx.handle, None, None
    _check(_lib.gto_decode_destroy(handle), "gto_decode_destroy")


# Tensors that do not fit the context (type, shape, strides, device) raise ValueError.

def gto_kv_append(ctx: DecodeCtx, batch: dict, q, k, v, q_out, k_cache, v_cache, inv_freq, q_norm=None, k_norm=None,
                  stream=None):
    """batch: dict of device tensors q_start [S+1], kv_len [S], page_table [S, max_pages] (int32) and, with trees,
    node_mask (int64), node_depth, optionally n_nodes.  q, k, v: [T, heads, head_dim], the last two dimensions dense;
    q and q_out may be None.  k_cache, v_cache: [n_pages, page_size, n_kv_heads, head_dim], any strides with dense heads."""
    code = _native.kv_append(ctx.native, batch, q, k, v, q_out, k_cache, v_cache, inv_freq, q_norm, k_norm,
                             _stream_of(ctx, stream))
    if code:
        raise GtoError(code, "gto_kv_append")


def gto_tree_attention(ctx: DecodeCtx, batch: dict, q, k_cache, v_cache, out, lse=None, stream=None):
    code = _native.tree_attention(ctx.native, batch, q, k_cache, v_cache, out, lse, _stream_of(ctx, stream))
    if code:
        raise GtoError(code, "gto_tree_attention")


_VERDICT_FIELDS = ("accept_len", "path_node", "token")


def alloc_verdict(cfg: gto_decode_config, device, S=None) -> dict:
    S = cfg.S if S is None else S
    shapes = {"accept_len": (S,), "path_node": (S, cfg.D), "token": (S, cfg.D + 1)}
    return {n: torch.empty(shapes[n], dtype=torch.int32, device=device) for n in _VERDICT_FIELDS}


def gto_verify_tree(ctx: DecodeCtx, tree: dict, target, d2t, temperature, u_node, u_bonus, verdict: dict, stream=None):
    """tree: dict of [S, g] int32 tensors node_token and node_parent (with GTO_DECODE_CONTEXT_ROWS also node_depth and
    node_slot), optionally n_nodes [S]; target: [S, 1+g, V_target] or [S, R, V_target]."""
    code = _native.verify_tree(ctx.native, tree, target, d2t, temperature, u_node, u_bonus, verdict, _stream_of(ctx, stream))
    if code:
        raise GtoError(code, "gto_verify_tree")


def gto_kv_commit(ctx: DecodeCtx, batch: dict, verdict: dict, k_cache, v_cache, kv_len_out, stream=None, tokens=None):
    """k_cache, v_cache: [n_pages, ...] of one layer or [n_layers, n_pages, ...] of all.  tokens: rows of the q, k and v that
    the step's other calls were given, by which they judged the batch (default: the context's T, which skips nothing that
    ends behind those rows)."""
    code = _native.kv_commit(ctx.native, batch, verdict, k_cache, v_cache, kv_len_out, tokens, _stream_of(ctx, stream))
    if code:
        raise GtoError(code, "gto_kv_commit")


def gto_decode_status(ctx: DecodeCtx, stream=None) -> int:
    code = ctypes.c_int32(0)
    _check(_lib.gto_decode_status(ctx.handle, _stream_of(ctx, stream), ctypes.byref(code)), "gto_decode_status")
    return code.value


def gto_decode_launch_count(ctx: DecodeCtx) -> int:
    return int(_lib.gto_decode_launch_count(ctx.handle))


EXPORTS = ["gto_create", "gto_destroy", "gto_build_tree", "gto_tree_reward",
           "gto_group_surrogate_grad", "gto_device_status", "gto_launch_count", "gto_status_string",
           "gto_kernel_timing", "gto_kernel_times", "gto_build_tree_noalloc", "gto_token_loss", "gto_sample_groups", "gto_tree_reward_host",
           "gto_token_loss_accumulate", "gto_decode_create", "gto_decode_destroy", "gto_kv_append",
           "gto_tree_attention", "gto_verify_tree", "gto_kv_commit", "gto_decode_status", "gto_decode_launch_count"]
