// Device helpers shared by the kernels of the decoding step.
#pragma once

#include "decode_internal.h"
#include "gto_common.cuh"

namespace gto {

// One sequence's chunk.  `ok` is false where its tables contradict one another.
struct Chunk {
  int q0, n, len, base, nodes, lead;
  bool ok;
};

__device__ __forceinline__ Chunk load_chunk(const BatchArgs& b, int s) {
  Chunk c;
  c.q0 = b.q_start[s];
  c.n = b.q_start[s + 1] - c.q0;
  c.len = b.kv_len[s];
  c.nodes = 0;
  if (b.tree && c.n != 0) c.nodes = b.n_nodes ? b.n_nodes[s] : b.g;
  c.base = c.len - c.n;
  c.lead = c.n - c.nodes;
  // q0 <= T and n <= T - q0 are tested so that no sum can wrap
  c.ok = c.q0 >= 0 && c.q0 <= b.T && c.n >= 0 && c.n <= b.T - c.q0 && c.len >= c.n &&
         c.len <= static_cast<int64_t>(b.max_pages) * b.page_size && c.nodes >= 0 &&
         c.nodes <= b.g && c.lead >= 0;
  return c;
}

// Whether q_start decreases over sequence s.  That sequence and all behind it are skipped: load_chunk looks at
// one sequence alone, and only where q_start has not decreased are the tokens of two sequences apart.
__device__ __forceinline__ bool falls(const BatchArgs& b, int s) { return b.q_start[s + 1] < b.q_start[s]; }

// Page of cache entry t (t inside the sequence); -1 if the table names none.
__device__ __forceinline__ int page_of(const BatchArgs& b, int s, int t) {
  const int p = b.page_table[static_cast<int64_t>(s) * b.max_pages + t / b.page_size];
  return p >= 0 && p < b.n_pages ? p : -1;
}

// Whether token i of a chunk sees cache entry e of its sequence (e < len).
__device__ __forceinline__ bool sees(const BatchArgs& b, int s, const Chunk& c, int i, int e) {
  if (i < c.lead) return e <= c.base + i;
  const int a = e - c.base - c.lead;
  if (a < 0) return true;
  if (a >= c.nodes) return false;
  const int64_t row = (static_cast<int64_t>(s) * b.g + (i - c.lead)) * b.W;
  return (b.node_mask[row + (a >> 6)] >> (a & 63)) & 1;
}

// Entries that the tokens up to i_last of a chunk can see: 0 .. kv_end-1.
__device__ __forceinline__ int kv_end(const Chunk& c, int i_last) {
  return i_last < c.lead ? c.base + i_last + 1 : c.len;
}

}  // namespace gto
