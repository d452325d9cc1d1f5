// Host-side declarations shared by the translation units of the decoding step (not part of the ABI).
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "gto_internal.h"

namespace gto {

constexpr int kMaxHeadDim = 256;
constexpr int kMaxGroup = 128;          // query heads per key head
constexpr size_t kMaxTargetRow = 1536u << 10;  // bytes of a target row gto_verify_tree takes

// A batch as the kernels see it.
struct BatchArgs {
  int S, T, g, W, page_size, n_pages, max_pages;
  const int32_t* q_start;
  const int32_t* kv_len;
  const int32_t* page_table;
  const int32_t* n_nodes;      // or null
  const uint64_t* node_mask;   // or null
  const int32_t* node_depth;   // or null
  bool tree;                   // chunks end in tree nodes
  int32_t* status;
};

struct CacheArgs {
  char* k;
  char* v;
  // bytes
  int64_t k_page, k_entry, k_head, k_layer;
  int64_t v_page, v_entry, v_head, v_layer;
  int n_layers, n_kv_heads, head_dim, dtype;
};

struct AppendArgs {
  BatchArgs b;
  CacheArgs c;
  const char* q;
  const char* k;
  const char* v;
  int64_t q_stride, k_stride, v_stride;  // bytes between tokens
  char* q_out;
  const double* inv_freq;
  const char* q_norm;
  const char* k_norm;
  int n_q_heads, rope_dims;
  float norm_eps;
  bool interleaved;
};
cudaError_t launch_kv_append(const AppendArgs& a, cudaStream_t stream, int64_t* launches);

struct CommitArgs {
  BatchArgs b;
  CacheArgs c;
  const int32_t* accept_len;
  const int32_t* path_node;
  int D;
  int32_t* kv_len_out;
};
cudaError_t launch_kv_commit(const CommitArgs& a, cudaStream_t stream, int64_t* launches);

struct VerifyArgs {
  int S, g, D, k, V_draft, V_target, dtype, rows;  // rows of a sequence's target block
  bool context_rows;
  const int32_t* node_token;
  const int32_t* node_parent;
  const int32_t* node_depth;
  const int32_t* node_slot;
  const int32_t* n_nodes;
  const char* target;
  const int32_t* d2t;
  const float* temperature;
  const float* u_node;
  const float* u_bonus;
  int32_t* accept_len;
  int32_t* path_node;
  int32_t* token;
  int32_t* status;
};
cudaError_t launch_verify_tree(const VerifyArgs& a, int sms, cudaStream_t stream, int64_t* launches);

constexpr int kMaxLeft = 4096;  // rows that gto_sample_tokens can list for its second kernel,
constexpr int kLeftRows = 64;   // from this word of their workspace on

// Rows to draw from, or trees to verify, under limits.
struct LimitedArgs {
  int N, V, dtype;       // sequences; length of a row
  const char* logits;
  int64_t row_stride;    // bytes
  const float* temperature;
  const int32_t* top_k;  // or null, as the next two
  const float* top_p;
  const float* min_p;
  const float* u;        // of the drawn token
  int32_t* token;        // [N], with trees [N, D+1]
  int32_t* status;
  // rows
  const int32_t* rows;   // or null: row s
  int n_rows;
  float* logp;           // or null, as the next one
  int32_t* n_kept;
  int32_t* left;         // workspace: their count, the CTAs that have read it (both 0 between calls), the rows
  // trees
  int g, D, k, V_draft, rows_of_tree;
  bool context_rows;
  const int32_t* node_token;
  const int32_t* node_parent;
  const int32_t* node_depth;
  const int32_t* node_slot;
  const int32_t* n_nodes;
  const int32_t* d2t;
  const float* u_node;
  int32_t* accept_len;
  int32_t* path_node;
};
cudaError_t launch_limited_bf16(const LimitedArgs& a, bool tree, int sms, cudaStream_t stream, int64_t* launches);
cudaError_t launch_limited_f16(const LimitedArgs& a, bool tree, int sms, cudaStream_t stream, int64_t* launches);
cudaError_t launch_limited_f32(const LimitedArgs& a, bool tree, int sms, cudaStream_t stream, int64_t* launches);
inline cudaError_t launch_limited(const LimitedArgs& a, bool tree, int sms, cudaStream_t stream, int64_t* launches) {
  if (a.dtype == GTO_BF16) return launch_limited_bf16(a, tree, sms, stream, launches);
  if (a.dtype == GTO_F16) return launch_limited_f16(a, tree, sms, stream, launches);
  return launch_limited_f32(a, tree, sms, stream, launches);
}

// Pages of the cache and the tables that name them.
struct PoolArgs {
  int S, page_size, n_pages, max_pages;
  int32_t* page_table;
  int32_t* kv_len;
  int32_t* held;
  int32_t* ref_count;
  int32_t* status;
};
size_t pages_workspace(const gto_decode_config& c);
cudaError_t launch_pages_fork(const PoolArgs& p, const int32_t* parent, void* ws, cudaStream_t stream, int64_t* launches);
cudaError_t launch_pages_resize(const PoolArgs& p, const int32_t* want, const CacheArgs& c, void* ws, int sms,
                                cudaStream_t stream, int64_t* launches);
cudaError_t launch_pages_compact(const PoolArgs& p, const CacheArgs& c, int32_t* table_out, int32_t* ref_out, int32_t* n_used,
                                 void* ws, int sms, cudaStream_t stream, int64_t* launches);

struct AttnArgs {
  BatchArgs b;
  CacheArgs c;
  const char* q;
  int64_t q_stride;  // bytes between tokens
  char* out;
  float* lse;        // or null
  int n_q_heads;
  float scale;
};
// Tensor-core kernel: whether it takes a configuration, what workspace it needs.
bool attention_tc_serves(const gto_decode_config& c);
size_t attention_tc_workspace(const gto_decode_config& c, int sms);
cudaError_t launch_attention_tc(const AttnArgs& a, void* workspace, int sms, cudaStream_t stream,
                                int64_t* launches);
cudaError_t launch_attention_simt(const AttnArgs& a, int sms, cudaStream_t stream, int64_t* launches);

}  // namespace gto
