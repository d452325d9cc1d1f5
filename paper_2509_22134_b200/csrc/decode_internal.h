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
