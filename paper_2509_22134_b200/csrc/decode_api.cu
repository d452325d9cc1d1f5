// C ABI of the decoding step: contexts, argument checks, launch sequencing.
#include <cmath>
#include <initializer_list>
#include <new>

#include <nvtx3/nvToolsExt.h>

#include "decode_internal.h"
#include "gto_common.cuh"

struct gto_decode_ctx {
  gto_decode_config cfg;
  int device;
  int sms;
  char* ws;          // one allocation
  int32_t* status;
  char* attn_ws;     // parts of blocks that were cut, null where the tensor-core kernel does not serve
  int64_t launches;
};

namespace {

struct DeviceGuard {
  int prev = -1;
  bool ok = true;
  explicit DeviceGuard(int dev) {
    ok = cudaGetDevice(&prev) == cudaSuccess && (prev == dev || cudaSetDevice(dev) == cudaSuccess);
    dev_ = dev;
  }
  ~DeviceGuard() {
    if (prev >= 0 && prev != dev_) cudaSetDevice(prev);
  }
  int dev_;
};

struct CallRange {
  explicit CallRange(const char* name) { nvtxRangePushA(name); }
  ~CallRange() { nvtxRangePop(); }
};

bool aligned(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
bool table(const void* p, size_t n) { return p != nullptr && aligned(p, n); }

bool overlap(const void* a, size_t na, const void* b, size_t nb) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x < y + nb && y < x + na;
}

// Whether an output lies over one of several arrays.
struct Array {
  const void* p;
  size_t bytes;
};
bool over_any(Array out, std::initializer_list<Array> in) {
  for (const Array& x : in)
    if (x.p && x.bytes && overlap(out.p, out.bytes, x.p, x.bytes)) return true;
  return false;
}

// Bytes a token array of T rows spans.
size_t span(int T, int64_t stride, int64_t row) {
  return T <= 0 ? 0 : static_cast<size_t>(T - 1) * stride + row;
}

gto_status batch_args(const gto_decode_ctx* ctx, const gto_batch* in, bool needs_depth, bool needs_mask,
                      gto::BatchArgs* out) {
  const gto_decode_config& c = ctx->cfg;
  if (!in || in->S < 0 || in->T < 0) return GTO_ERR_INVALID_ARG;
  if (in->S > c.S || in->T > c.T || c.n_kv_heads == 0) return GTO_ERR_INVALID_ARG;
  out->S = in->S;
  out->T = in->T;
  if (in->S == 0) return GTO_OK;  // its arrays have no elements and may have no address
  if (!table(in->q_start, 4) || !table(in->kv_len, 4) || !table(in->page_table, 4)) return GTO_ERR_INVALID_ARG;
  if (in->n_nodes && !aligned(in->n_nodes, 4)) return GTO_ERR_INVALID_ARG;
  if (in->node_mask && !aligned(in->node_mask, 8)) return GTO_ERR_INVALID_ARG;
  if (in->node_depth && !aligned(in->node_depth, 4)) return GTO_ERR_INVALID_ARG;
  // a batch has trees for all calls or for none
  const bool tree = in->node_mask != nullptr || in->node_depth != nullptr;
  if (tree && c.g == 0) return GTO_ERR_INVALID_ARG;
  if (!tree && in->n_nodes) return GTO_ERR_INVALID_ARG;
  if (tree && needs_depth && !in->node_depth) return GTO_ERR_INVALID_ARG;
  if (tree && needs_mask && !in->node_mask) return GTO_ERR_INVALID_ARG;
  out->g = c.g;
  out->W = (c.g + 63) / 64;
  out->page_size = c.page_size;
  out->n_pages = c.n_pages;
  out->max_pages = c.max_pages;
  out->q_start = in->q_start;
  out->kv_len = in->kv_len;
  out->page_table = in->page_table;
  out->n_nodes = in->n_nodes;
  out->node_mask = in->node_mask;
  out->node_depth = in->node_depth;
  out->tree = tree;
  out->status = ctx->status;
  return GTO_OK;
}

gto_status cache_args(const gto_decode_ctx* ctx, const gto_kv_cache* in, gto::CacheArgs* out) {
  const gto_decode_config& c = ctx->cfg;
  if (!in || !table(in->k, 16) || !table(in->v, 16) || in->n_layers < 1 || in->n_layers > 65535)
    return GTO_ERR_INVALID_ARG;
  const int64_t e = gto::elem_bytes(c.kv_dtype);
  const int64_t* from[8] = {&in->k_page, &in->k_entry, &in->k_head, &in->k_layer,
                            &in->v_page, &in->v_entry, &in->v_head, &in->v_layer};
  int64_t* to[8] = {&out->k_page, &out->k_entry, &out->k_head, &out->k_layer,
                    &out->v_page, &out->v_entry, &out->v_head, &out->v_layer};
  for (int i = 0; i < 8; ++i) {
    if (*from[i] < 0 || *from[i] >= (1ll << 40) || (*from[i] * e) % 16) return GTO_ERR_INVALID_ARG;
    *to[i] = *from[i] * e;
  }
  out->k = static_cast<char*>(in->k);
  out->v = static_cast<char*>(in->v);
  out->n_layers = in->n_layers;
  out->n_kv_heads = c.n_kv_heads;
  out->head_dim = c.head_dim;
  out->dtype = c.kv_dtype;
  return GTO_OK;
}

}  // namespace

extern "C" {

gto_status gto_decode_create(gto_decode_ctx** out, const gto_decode_config* c, int device) {
  if (!out || !c) return GTO_ERR_INVALID_ARG;
  *out = nullptr;
  if (c->S <= 0 || c->T < 0 || c->g < 0 || c->D < 1 || c->n_kv_heads < 0 || c->V_target < 0)
    return GTO_ERR_INVALID_ARG;
  if (c->flags & ~static_cast<uint32_t>(GTO_DECODE_ROPE_INTERLEAVED | GTO_DECODE_CONTEXT_ROWS))
    return GTO_ERR_INVALID_ARG;
  if (c->n_kv_heads == 0 && c->V_target == 0) return GTO_ERR_INVALID_ARG;
  if (c->g > gto::kMaxNodes || c->D > gto::kMaxDepth) return GTO_ERR_UNSUPPORTED;
  if (c->n_kv_heads > 0) {
    if (c->n_q_heads <= 0 || c->n_q_heads % c->n_kv_heads || c->head_dim <= 0 || c->page_size <= 0 ||
        c->n_pages <= 0 || c->max_pages <= 0 || c->rope_dims < 0 || c->rope_dims > c->head_dim)
      return GTO_ERR_INVALID_ARG;
    if (!gto::valid_dtype(c->kv_dtype)) return GTO_ERR_INVALID_ARG;
    if (!std::isfinite(c->softmax_scale) || !(c->softmax_scale > 0.f) || !(c->norm_eps >= 0.f))
      return GTO_ERR_INVALID_ARG;
    if (c->n_q_heads / c->n_kv_heads > gto::kMaxGroup || c->head_dim % 16 || c->head_dim > gto::kMaxHeadDim ||
        c->rope_dims % 16 || c->n_kv_heads > 65535)
      return GTO_ERR_UNSUPPORTED;
    if (static_cast<int64_t>(c->max_pages) * c->page_size > (1ll << 31) - 256) return GTO_ERR_UNSUPPORTED;
    // work units of a call are counted in 32 bits
    if (static_cast<int64_t>(c->T) * c->n_q_heads + c->S >= (1ll << 30)) return GTO_ERR_UNSUPPORTED;
  }
  if (c->V_target > 0) {
    if (!gto::valid_dtype(c->logit_dtype)) return GTO_ERR_INVALID_ARG;
    if (c->V_draft <= 0 || c->V_draft > c->V_target || c->g > c->V_draft) return GTO_ERR_INVALID_ARG;
    const int64_t row = static_cast<int64_t>(c->V_target) * gto::elem_bytes(c->logit_dtype);
    if (row % 16 || row > static_cast<int64_t>(gto::kMaxTargetRow)) return GTO_ERR_UNSUPPORTED;
    if ((c->flags & GTO_DECODE_CONTEXT_ROWS) && c->k <= 0) return GTO_ERR_INVALID_ARG;
    if ((c->flags & GTO_DECODE_CONTEXT_ROWS) && c->k > gto::kMaxTopK) return GTO_ERR_UNSUPPORTED;
    if (c->S > (1 << 27)) return GTO_ERR_UNSUPPORTED;  // eight CTAs a sequence
  }
  DeviceGuard guard(device);
  if (!guard.ok) {
    cudaGetLastError();
    return GTO_ERR_CUDA;
  }
  gto_decode_ctx* ctx = new (std::nothrow) gto_decode_ctx();
  if (!ctx) return GTO_ERR_WORKSPACE;
  ctx->cfg = *c;
  ctx->device = device;
  ctx->launches = 0;
  if (cudaDeviceGetAttribute(&ctx->sms, cudaDevAttrMultiProcessorCount, device) != cudaSuccess) {
    cudaGetLastError();
    delete ctx;
    return GTO_ERR_CUDA;
  }
  const bool tc = c->n_kv_heads > 0 && gto::attention_tc_serves(*c);
  if (cudaMalloc(&ctx->ws, 256 + (tc ? gto::attention_tc_workspace(*c, ctx->sms) : 0)) != cudaSuccess) {
    cudaGetLastError();
    delete ctx;
    return GTO_ERR_WORKSPACE;
  }
  ctx->status = reinterpret_cast<int32_t*>(ctx->ws);
  ctx->attn_ws = tc ? ctx->ws + 256 : nullptr;
  // (waited for: the first call may come on a stream that the default one does not order)
  if (cudaMemset(ctx->ws, 0, 256) != cudaSuccess || cudaStreamSynchronize(nullptr) != cudaSuccess) {
    cudaGetLastError();
    cudaFree(ctx->ws);
    delete ctx;
    return GTO_ERR_WORKSPACE;
  }
  *out = ctx;
  return GTO_OK;
}

gto_status gto_decode_destroy(gto_decode_ctx* ctx) {
  if (!ctx) return GTO_ERR_INVALID_ARG;
  DeviceGuard guard(ctx->device);
  const cudaError_t e = cudaFree(ctx->ws);
  delete ctx;
  return e == cudaSuccess ? GTO_OK : GTO_ERR_CUDA;
}

gto_status gto_kv_append(gto_decode_ctx* ctx, const gto_batch* batch, const gto_kv_cache* cache,
                         const void* q, int64_t q_stride, const void* k, int64_t k_stride, const void* v,
                         int64_t v_stride, void* q_out, const double* inv_freq, const void* q_norm,
                         const void* k_norm, void* stream) {
  if (!ctx) return GTO_ERR_INVALID_ARG;
  CallRange range("gto_kv_append");
  const gto_decode_config& c = ctx->cfg;
  gto::AppendArgs a{};
  gto_status st = batch_args(ctx, batch, true, false, &a.b);
  if (st != GTO_OK) return st;
  st = cache_args(ctx, cache, &a.c);
  if (st != GTO_OK) return st;
  if (a.b.S == 0 || a.b.T == 0) return GTO_OK;
  const int64_t e = gto::elem_bytes(c.kv_dtype);
  const int64_t q_row = c.n_q_heads * static_cast<int64_t>(c.head_dim) * e;
  const int64_t kv_row = c.n_kv_heads * static_cast<int64_t>(c.head_dim) * e;
  if (!table(k, 16) || !table(v, 16) || (k_stride * e) % 16 || (v_stride * e) % 16 || k_stride * e < kv_row ||
      v_stride * e < kv_row)
    return GTO_ERR_INVALID_ARG;
  if ((q == nullptr) != (q_out == nullptr) || (!q && q_norm)) return GTO_ERR_INVALID_ARG;
  if (q) {
    if (!table(q, 16) || !table(q_out, 16) || (q_stride * e) % 16 || q_stride * e < q_row) return GTO_ERR_INVALID_ARG;
    const bool in_place = q == q_out && q_stride * e == q_row;
    if (!in_place && overlap(q, span(a.b.T, q_stride * e, q_row), q_out, static_cast<size_t>(a.b.T) * q_row))
      return GTO_ERR_INVALID_ARG;
    if (overlap(k, span(a.b.T, k_stride * e, kv_row), q_out, static_cast<size_t>(a.b.T) * q_row) ||
        overlap(v, span(a.b.T, v_stride * e, kv_row), q_out, static_cast<size_t>(a.b.T) * q_row))
      return GTO_ERR_INVALID_ARG;
  }
  if (c.rope_dims > 0 && !table(inv_freq, 8)) return GTO_ERR_INVALID_ARG;
  if ((q_norm && !aligned(q_norm, 16)) || (k_norm && !aligned(k_norm, 16))) return GTO_ERR_INVALID_ARG;
  a.q = static_cast<const char*>(q);
  a.k = static_cast<const char*>(k);
  a.v = static_cast<const char*>(v);
  a.q_stride = q_stride * e;
  a.k_stride = k_stride * e;
  a.v_stride = v_stride * e;
  a.q_out = static_cast<char*>(q_out);
  a.inv_freq = inv_freq;
  a.q_norm = static_cast<const char*>(q_norm);
  a.k_norm = static_cast<const char*>(k_norm);
  a.n_q_heads = c.n_q_heads;
  a.rope_dims = c.rope_dims;
  a.norm_eps = c.norm_eps;
  a.interleaved = (c.flags & GTO_DECODE_ROPE_INTERLEAVED) != 0;
  DeviceGuard guard(ctx->device);
  if (!guard.ok) return GTO_ERR_CUDA;
  if (gto::launch_kv_append(a, static_cast<cudaStream_t>(stream), &ctx->launches) != cudaSuccess)
    return GTO_ERR_CUDA;
  return GTO_OK;
}

gto_status gto_tree_attention(gto_decode_ctx* ctx, const gto_batch* batch, const gto_kv_cache* cache,
                              const void* q, int64_t q_stride, void* out, float* lse, void* stream) {
  if (!ctx) return GTO_ERR_INVALID_ARG;
  CallRange range("gto_tree_attention");
  const gto_decode_config& c = ctx->cfg;
  gto::AttnArgs a{};
  gto_status st = batch_args(ctx, batch, false, true, &a.b);
  if (st != GTO_OK) return st;
  st = cache_args(ctx, cache, &a.c);
  if (st != GTO_OK) return st;
  if (a.b.S == 0 || a.b.T == 0) return GTO_OK;
  const int64_t e = gto::elem_bytes(c.kv_dtype);
  const int64_t q_row = c.n_q_heads * static_cast<int64_t>(c.head_dim) * e;
  if (!table(q, 16) || !table(out, 16) || (q_stride * e) % 16 || q_stride * e < q_row || (lse && !aligned(lse, 4)))
    return GTO_ERR_INVALID_ARG;
  const Array rows{q, span(a.b.T, q_stride * e, q_row)}, outs{out, static_cast<size_t>(a.b.T) * q_row};
  if (over_any(outs, {rows})) return GTO_ERR_INVALID_ARG;
  if (lse && over_any({lse, sizeof(float) * a.b.T * c.n_q_heads}, {rows, outs})) return GTO_ERR_INVALID_ARG;
  a.q = static_cast<const char*>(q);
  a.q_stride = q_stride * e;
  a.out = static_cast<char*>(out);
  a.lse = lse;
  a.n_q_heads = c.n_q_heads;
  a.scale = c.softmax_scale;
  DeviceGuard guard(ctx->device);
  if (!guard.ok) return GTO_ERR_CUDA;
  // a tensor map takes strides above 0 and below 2^40 bytes
  const int64_t strides[6] = {a.c.k_page, a.c.k_entry, a.c.k_head, a.c.v_page, a.c.v_entry, a.c.v_head};
  bool tc = ctx->attn_ws != nullptr;
  for (int64_t x : strides) tc = tc && x > 0 && x < (1ll << 40);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const cudaError_t err = tc ? gto::launch_attention_tc(a, ctx->attn_ws, ctx->sms, s, &ctx->launches)
                           : gto::launch_attention_simt(a, ctx->sms, s, &ctx->launches);
  if (err != cudaSuccess) return GTO_ERR_CUDA;
  return GTO_OK;
}

gto_status gto_verify_tree(gto_decode_ctx* ctx, const gto_draft_tree* tree, const void* target,
                           const int32_t* d2t, const float* temperature, const float* u_node,
                           const float* u_bonus, const gto_verdict* out, void* stream) {
  if (!ctx) return GTO_ERR_INVALID_ARG;
  CallRange range("gto_verify_tree");
  const gto_decode_config& c = ctx->cfg;
  if (!tree || !out || c.V_target == 0 || tree->S < 0 || tree->S > c.S) return GTO_ERR_INVALID_ARG;
  if (tree->S == 0) return GTO_OK;
  if (!table(target, 16) || !table(temperature, 4) || !table(u_bonus, 4) || !table(out->accept_len, 4) ||
      !table(out->path_node, 4) || !table(out->token, 4) || (d2t && !aligned(d2t, 4)))
    return GTO_ERR_INVALID_ARG;
  if (c.g > 0 && (!table(tree->node_token, 4) || !table(tree->node_parent, 4) || !table(u_node, 4)))
    return GTO_ERR_INVALID_ARG;
  if (tree->n_nodes && !aligned(tree->n_nodes, 4)) return GTO_ERR_INVALID_ARG;
  if (!d2t && c.V_draft != c.V_target) return GTO_ERR_INVALID_ARG;
  const bool ctx_rows = (c.flags & GTO_DECODE_CONTEXT_ROWS) != 0;
  if (ctx_rows && c.g > 0 && (!table(tree->node_depth, 4) || !table(tree->node_slot, 4)))
    return GTO_ERR_INVALID_ARG;
  const size_t S = tree->S, word = sizeof(int32_t), nodes = word * S * c.g;
  const size_t target_rows = ctx_rows ? 1 + static_cast<size_t>(c.D - 1) * c.k : 1 + static_cast<size_t>(c.g);
  const Array outs[3] = {{out->accept_len, word * S}, {out->path_node, word * S * c.D}, {out->token, word * S * (c.D + 1)}};
  for (int i = 0; i < 3; ++i)
    if (over_any(outs[i], {outs[(i + 1) % 3], {tree->node_token, nodes}, {tree->node_parent, nodes},
                           {ctx_rows ? tree->node_depth : nullptr, nodes}, {ctx_rows ? tree->node_slot : nullptr, nodes},
                           {tree->n_nodes, word * S}, {target, S * target_rows * c.V_target * gto::elem_bytes(c.logit_dtype)},
                           {d2t, word * c.V_draft}, {temperature, word * S}, {u_node, nodes}, {u_bonus, word * S}}))
      return GTO_ERR_INVALID_ARG;
  gto::VerifyArgs a{};
  a.S = tree->S;
  a.g = c.g;
  a.D = c.D;
  a.k = c.k;
  a.V_draft = c.V_draft;
  a.V_target = c.V_target;
  a.dtype = c.logit_dtype;
  a.context_rows = ctx_rows;
  a.rows = ctx_rows ? 1 + (c.D - 1) * c.k : 1 + c.g;
  a.node_token = tree->node_token;
  a.node_parent = tree->node_parent;
  a.node_depth = tree->node_depth;
  a.node_slot = tree->node_slot;
  a.n_nodes = tree->n_nodes;
  a.target = static_cast<const char*>(target);
  a.d2t = d2t;
  a.temperature = temperature;
  a.u_node = u_node;
  a.u_bonus = u_bonus;
  a.accept_len = out->accept_len;
  a.path_node = out->path_node;
  a.token = out->token;
  a.status = ctx->status;
  DeviceGuard guard(ctx->device);
  if (!guard.ok) return GTO_ERR_CUDA;
  if (gto::launch_verify_tree(a, ctx->sms, static_cast<cudaStream_t>(stream), &ctx->launches) != cudaSuccess)
    return GTO_ERR_CUDA;
  return GTO_OK;
}

gto_status gto_kv_commit(gto_decode_ctx* ctx, const gto_batch* batch, const gto_verdict* verdict,
                         const gto_kv_cache* cache, int32_t* kv_len_out, void* stream) {
  if (!ctx) return GTO_ERR_INVALID_ARG;
  CallRange range("gto_kv_commit");
  gto::CommitArgs a{};
  gto_status st = batch_args(ctx, batch, false, false, &a.b);
  if (st != GTO_OK) return st;
  st = cache_args(ctx, cache, &a.c);
  if (st != GTO_OK) return st;
  if (a.b.S == 0) return GTO_OK;
  if (!verdict || !table(verdict->accept_len, 4) || !table(verdict->path_node, 4) || !table(kv_len_out, 4))
    return GTO_ERR_INVALID_ARG;
  const size_t word = sizeof(int32_t), S = a.b.S;
  if (over_any({kv_len_out, word * S}, {{batch->kv_len, word * S}, {batch->q_start, word * (S + 1)}, {batch->n_nodes, word * S},
                                        {batch->page_table, word * S * ctx->cfg.max_pages}, {verdict->accept_len, word * S},
                                        {verdict->path_node, word * S * ctx->cfg.D}}))
    return GTO_ERR_INVALID_ARG;
  a.accept_len = verdict->accept_len;
  a.path_node = verdict->path_node;
  a.D = ctx->cfg.D;
  a.kv_len_out = kv_len_out;
  DeviceGuard guard(ctx->device);
  if (!guard.ok) return GTO_ERR_CUDA;
  if (gto::launch_kv_commit(a, static_cast<cudaStream_t>(stream), &ctx->launches) != cudaSuccess)
    return GTO_ERR_CUDA;
  return GTO_OK;
}

gto_status gto_decode_status(gto_decode_ctx* ctx, void* stream, int32_t* host_code) {
  if (!ctx || !host_code) return GTO_ERR_INVALID_ARG;
  DeviceGuard guard(ctx->device);
  if (!guard.ok) return GTO_ERR_CUDA;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  int32_t word = 0;
  if (cudaMemcpyAsync(&word, ctx->status, sizeof(word), cudaMemcpyDeviceToHost, s) != cudaSuccess ||
      cudaMemsetAsync(ctx->status, 0, sizeof(word), s) != cudaSuccess ||
      cudaStreamSynchronize(s) != cudaSuccess)
    return GTO_ERR_CUDA;
  *host_code = (word & gto::kStatusTimeout)     ? GTO_ERR_TIMEOUT
               : (word & gto::kStatusBadIndex)  ? GTO_ERR_BAD_INDEX
               : (word & gto::kStatusNonFinite) ? GTO_ERR_NONFINITE
                                                : GTO_OK;
  return GTO_OK;
}

int64_t gto_decode_launch_count(const gto_decode_ctx* ctx) { return ctx ? ctx->launches : 0; }

}  // extern "C"
