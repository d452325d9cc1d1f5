// gto_pages_fork, gto_pages_resize, gto_pages_compact: who holds which pages of the cache.
//
// The state is a table of pages for every sequence and a count for every page of how often the tables name
// it; a page that nobody names is free, there is no list of free pages to keep in order.  Fresh pages are the
// lowest free ones, given out in the order of the sequences, so that equal calls give equal tables; counts
// change by integer atomics, whose order does not matter.  A call is a plan (what every sequence needs, read
// from the tables as they stood) and then its execution by another kernel, so that nothing is read after another
// sequence has changed it.
#include "decode_common.cuh"

namespace gto {
namespace {

constexpr int kPlanThreads = 1024;
constexpr int kThreads = 256;

// ---- workspace
struct Plan {           // of a sequence
  int need;             // slots that it will hold; -1: it stays as it is
  int keep;             // entries that it will have
  int base;             // its first place in the list of fresh pages
  int swaps;            // of those, how many replace a shared page
};
struct Copy {           // entries of a shared page that its replacement gets
  int src, dst, entries;
};
struct Workspace {
  int32_t* rows;        // [S, max_pages] rows to be / replacements of shared pages
  Plan* plan;           // [S]
  Copy* copies;         // [S]
  int32_t* list;        // [n_pages] fresh pages; pages that move
  int32_t* to;          // [n_pages] where they move; new number of every page
  int32_t* counts;      // [4]
};
size_t up(size_t n) { return (n + 255) & ~static_cast<size_t>(255); }
size_t layout(int64_t S, int64_t max_pages, int64_t n_pages, char* p, Workspace* w) {
  size_t at = 0;
  const auto take = [&](size_t n) {
    char* q = p + at;
    at += up(n);
    return q;
  };
  Workspace x;
  x.counts = reinterpret_cast<int32_t*>(take(16));
  x.plan = reinterpret_cast<Plan*>(take(S * sizeof(Plan)));
  x.copies = reinterpret_cast<Copy*>(take(S * sizeof(Copy)));
  x.rows = reinterpret_cast<int32_t*>(take(S * max_pages * sizeof(int32_t)));
  x.list = reinterpret_cast<int32_t*>(take(n_pages * sizeof(int32_t)));
  x.to = reinterpret_cast<int32_t*>(take(2 * n_pages * sizeof(int32_t)));
  if (w) *w = x;
  return at;
}

// Sum of v over the threads before this one; *all receives the sum over all.  s_warp: 33 ints.
__device__ __forceinline__ int scan_before(int v, int* s_warp, int* all) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int upto = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(kFull, upto, o);
    if (lane >= o) upto += y;
  }
  __syncthreads();  // (s_warp may still be read from the last call)
  if (lane == 31) s_warp[warp] = upto;
  __syncthreads();
  int before = 0, sum = 0;
  for (int w = 0; w < kPlanThreads / 32; ++w) {
    if (w == warp) before = sum;
    sum += s_warp[w];
  }
  *all = sum;
  return before + upto - v;
}

__device__ __forceinline__ bool is_page(const PoolArgs& p, int page) { return page >= 0 && page < p.n_pages; }
__device__ __forceinline__ int pages_of(const PoolArgs& p, int entries) {
  return static_cast<int>((static_cast<int64_t>(entries) + p.page_size - 1) / p.page_size);
}
// Whether a sequence's numbers fit each other.
__device__ __forceinline__ bool fits(const PoolArgs& p, int held, int len) {
  return held >= 0 && held <= p.max_pages && len >= 0 && len <= static_cast<int64_t>(held) * p.page_size;
}

// ---- fork
__global__ void __launch_bounds__(kThreads) fork_plan_kernel(PoolArgs p, const int32_t* parent, Workspace w) {
  const int s = blockIdx.x, tid = threadIdx.x;
  const int from = parent[s];
  const int held = p.held[s];
  int need = -1, len = 0;
  bool bad = false;
  if (from != s) {
    bad = from < -1 || from >= p.S || held < 0 || held > p.max_pages;
    if (!bad) {
      need = 0;
      if (from >= 0) {
        len = p.kv_len[from];
        bad = !fits(p, p.held[from], len);
        need = bad ? 0 : pages_of(p, len);
      }
    }
    const int32_t* row = p.page_table + static_cast<int64_t>(from < 0 ? 0 : from) * p.max_pages;
    if (!bad)
      for (int j = tid; j < need; j += kThreads) bad |= !is_page(p, row[j]);
    bad = __syncthreads_or(bad);
    if (!bad) {
      bool odd = false;
      for (int j = tid; j < need; j += kThreads) {
        const int page = row[j];
        w.rows[static_cast<int64_t>(s) * p.max_pages + j] = page;
        atomicAdd(p.ref_count + page, 1);
      }
      for (int j = tid; j < held; j += kThreads) {
        const int page = p.page_table[static_cast<int64_t>(s) * p.max_pages + j];
        if (is_page(p, page)) atomicSub(p.ref_count + page, 1);
        else odd = true;
      }
      if (odd) atomicOr(p.status, kStatusBadIndex);
    }
  }
  if (tid == 0) {
    w.plan[s] = Plan{bad ? -1 : need, len, 0, 0};
    if (bad) atomicOr(p.status, kStatusBadIndex);
  }
}

__global__ void __launch_bounds__(kThreads) fork_apply_kernel(PoolArgs p, Workspace w) {
  const int s = blockIdx.x;
  const Plan plan = w.plan[s];
  if (plan.need < 0) return;
  const int64_t row = static_cast<int64_t>(s) * p.max_pages;
  for (int j = threadIdx.x; j < p.max_pages; j += kThreads) p.page_table[row + j] = j < plan.need ? w.rows[row + j] : -1;
  if (threadIdx.x == 0) {
    p.held[s] = plan.need;
    p.kv_len[s] = plan.keep;
  }
}

// ---- resize
__global__ void __launch_bounds__(kPlanThreads) resize_plan_kernel(PoolArgs p, const int32_t* want, Workspace w) {
  __shared__ int s_warp[kPlanThreads / 32];
  const int tid = threadIdx.x;
  // Whether slot j of a sequence, which will be written, is named elsewhere too.
  const auto shared_slot = [&](int s, int j, bool* bad) {
    const int page = p.page_table[static_cast<int64_t>(s) * p.max_pages + j];
    if (!is_page(p, page)) {
      *bad = true;
      return false;
    }
    return p.ref_count[page] > 1;
  };
  int total = 0;
  for (int s0 = 0; s0 < p.S; s0 += kPlanThreads) {
    const int s = s0 + tid;
    Plan plan{-1, 0, 0, 0};
    int fresh = 0;
    if (s < p.S) {
      const int target = want[s];
      if (target >= 0) {
        const int held = p.held[s], len = p.kv_len[s];
        bool bad = !fits(p, held, len) || target > static_cast<int64_t>(p.max_pages) * p.page_size;
        if (!bad) {
          plan.need = pages_of(p, target);
          plan.keep = min(len, target);
          if (target > plan.keep)
            for (int j = plan.keep / p.page_size; j < min(held, plan.need); ++j) plan.swaps += shared_slot(s, j, &bad);
          fresh = plan.swaps + max(plan.need - held, 0);
        }
        if (bad) {
          plan = Plan{-1, 0, 0, 0};
          fresh = 0;
          atomicOr(p.status, kStatusBadIndex);
        }
      }
    }
    int sum;
    plan.base = total + scan_before(fresh, s_warp, &sum);
    total += sum;
    if (s < p.S) w.plan[s] = plan;
  }
  // the lowest free pages, as many as are needed
  int found = 0;
  for (int p0 = 0; p0 < p.n_pages && found < total; p0 += kPlanThreads) {
    const int page = p0 + tid;
    const bool is_free = page < p.n_pages && p.ref_count[page] == 0;
    int sum;
    const int at = found + scan_before(is_free, s_warp, &sum);
    if (is_free && at < total) w.list[at] = page;
    found += sum;
  }
  __syncthreads();
  int n_copies = 0;
  for (int s0 = 0; s0 < p.S; s0 += kPlanThreads) {
    const int s = s0 + tid;
    Copy copy{-1, -1, 0};
    if (s < p.S) {
      Plan plan = w.plan[s];
      if (plan.need >= 0) {
        const int held = p.held[s];
        const int fresh = plan.swaps + max(plan.need - held, 0);
        if (fresh > 0 && static_cast<int64_t>(plan.base) + fresh > found) {  // it does not fit any more
          w.plan[s].need = -1;
          atomicOr(p.status, kStatusNoPages);
        } else if (plan.swaps > 0) {
          int at = plan.base;
          const int first = plan.keep / p.page_size;
          bool bad = false;
          for (int j = first; j < min(held, plan.need); ++j) {
            const bool swap = shared_slot(s, j, &bad);
            if (swap && j == first && plan.keep % p.page_size > 0)
              copy = Copy{p.page_table[static_cast<int64_t>(s) * p.max_pages + j], w.list[at], plan.keep % p.page_size};
            w.rows[static_cast<int64_t>(s) * p.max_pages + j] = swap ? w.list[at++] : -1;
          }
        }
      }
    }
    int sum;
    const int at = n_copies + scan_before(copy.entries > 0, s_warp, &sum);
    if (copy.entries > 0) w.copies[at] = copy;
    n_copies += sum;
  }
  if (tid == 0) w.counts[0] = n_copies;
}

// 16-byte vectors of `entries` entries of a page, keys or values of one layer, from one page to another.
__device__ __forceinline__ void copy_entries(const CacheArgs& c, bool key, int layer, int src, int dst, int entries) {
  const int64_t page = key ? c.k_page : c.v_page, entry = key ? c.k_entry : c.v_entry, head = key ? c.k_head : c.v_head;
  char* base = (key ? c.k : c.v) + layer * (key ? c.k_layer : c.v_layer);
  const char* from = base + src * page;
  char* to = base + dst * page;
  const int per_head = c.head_dim * (c.dtype == GTO_F32 ? 4 : 2) / 16;
  const int cols = c.n_kv_heads * per_head;
  const int64_t n = static_cast<int64_t>(entries) * cols;
  constexpr int kBatch = 8;
  for (int64_t i0 = threadIdx.x; i0 < n; i0 += kBatch * kThreads) {
    uint4 x[kBatch];
    int64_t at[kBatch];
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
      const int64_t i = i0 + b * kThreads;
      if (i < n) {
        const int e = static_cast<int>(i / cols), col = static_cast<int>(i % cols);
        at[b] = e * entry + (col / per_head) * head + (col % per_head) * 16;
        x[b] = *reinterpret_cast<const uint4*>(from + at[b]);
      }
    }
#pragma unroll
    for (int b = 0; b < kBatch; ++b)
      if (i0 + b * kThreads < n) *reinterpret_cast<uint4*>(to + at[b]) = x[b];
  }
}

// Block s < S: the tables of sequence s; the others: the copies.
__global__ void __launch_bounds__(kThreads) resize_apply_kernel(PoolArgs p, CacheArgs c, Workspace w) {
  if (static_cast<int>(blockIdx.x) >= p.S) {
    const int n = w.counts[0], units = 2 * c.n_layers;
    for (int64_t i = blockIdx.x - p.S; i < static_cast<int64_t>(n) * units; i += gridDim.x - p.S) {
      const Copy copy = w.copies[i / units];
      const int u = static_cast<int>(i % units);
      copy_entries(c, u & 1, u >> 1, copy.src, copy.dst, copy.entries);
    }
    return;
  }
  const int s = blockIdx.x, tid = threadIdx.x;
  const Plan plan = w.plan[s];
  if (plan.need < 0) return;
  const int held = p.held[s], target_kept = min(held, plan.need);
  const int64_t row = static_cast<int64_t>(s) * p.max_pages;
  bool odd = false;
  for (int j = plan.keep / p.page_size + tid; j < max(held, plan.need); j += kThreads) {
    const bool had = j < held;
    int fresh = -1;
    if (j < target_kept) {
      if (plan.swaps == 0) continue;
      fresh = w.rows[row + j];
      if (fresh < 0) continue;
    } else if (j < plan.need) {
      fresh = w.list[plan.base + plan.swaps + (j - held)];
    }
    if (had) {
      const int old = p.page_table[row + j];
      if (is_page(p, old)) atomicSub(p.ref_count + old, 1);
      else odd = true;
    }
    p.page_table[row + j] = fresh;
    if (fresh >= 0) p.ref_count[fresh] = 1;
  }
  if (odd) atomicOr(p.status, kStatusBadIndex);
  __syncthreads();
  if (tid == 0) {
    p.held[s] = plan.need;
    p.kv_len[s] = plan.keep;
  }
}

// ---- compact
__global__ void __launch_bounds__(kPlanThreads) compact_plan_kernel(PoolArgs p, int32_t* ref_out, int32_t* n_used, Workspace w) {
  __shared__ int s_warp[kPlanThreads / 32];
  const int tid = threadIdx.x;
  int used = 0;
  for (int page = tid; page < p.n_pages; page += kPlanThreads) used += p.ref_count[page] > 0;
  int total;
  scan_before(used, s_warp, &total);
  int holes = 0, movers = 0;
  int32_t* hole = w.to + p.n_pages;
  for (int p0 = 0; p0 < p.n_pages; p0 += kPlanThreads) {
    const int page = p0 + tid;
    const bool in = page < p.n_pages;
    const bool is_used = in && p.ref_count[page] > 0;
    const bool is_hole = in && !is_used && page < total, moves = is_used && page >= total;
    int sum;
    const int at_hole = holes + scan_before(is_hole, s_warp, &sum);
    holes += sum;
    const int at_move = movers + scan_before(moves, s_warp, &sum);
    movers += sum;
    if (is_hole) hole[at_hole] = page;
    if (moves) w.list[at_move] = page;
    if (in) {
      w.to[page] = page;
      ref_out[page] = is_used && !moves ? p.ref_count[page] : 0;
    }
  }
  __syncthreads();
  for (int i = tid; i < movers; i += kPlanThreads) {  // as many as holes
    const int page = w.list[i], to = hole[i];
    w.to[page] = to;
    ref_out[to] = p.ref_count[page];
  }
  if (tid == 0) {
    *n_used = total;
    w.counts[0] = movers;
  }
}

// Block s < S: the table of sequence s; the others: the pages that move.
__global__ void __launch_bounds__(kThreads) compact_apply_kernel(PoolArgs p, CacheArgs c, int32_t* table_out, Workspace w) {
  if (static_cast<int>(blockIdx.x) >= p.S) {
    const int n = w.counts[0], units = 2 * c.n_layers;
    for (int64_t i = blockIdx.x - p.S; i < static_cast<int64_t>(n) * units; i += gridDim.x - p.S) {
      const int page = w.list[i / units], u = static_cast<int>(i % units);
      copy_entries(c, u & 1, u >> 1, page, w.to[page], p.page_size);
    }
    return;
  }
  const int s = blockIdx.x, held = p.held[s];
  bool bad = held < 0 || held > p.max_pages;
  for (int j = threadIdx.x; j < p.max_pages; j += kThreads) {
    const int64_t at = static_cast<int64_t>(s) * p.max_pages + j;
    const int page = p.page_table[at];
    const bool is = is_page(p, page);
    table_out[at] = is ? w.to[page] : page;
    bad |= !is && j < held;
  }
  if (bad) atomicOr(p.status, kStatusBadIndex);
}

Workspace workspace_of(const PoolArgs& p, int S, void* ws) {
  Workspace w;
  layout(S, p.max_pages, p.n_pages, static_cast<char*>(ws), &w);
  return w;
}

}  // namespace

size_t pages_workspace(const gto_decode_config& c) { return layout(c.S, c.max_pages, c.n_pages, nullptr, nullptr); }

cudaError_t launch_pages_fork(const PoolArgs& p, const int32_t* parent, void* ws, cudaStream_t stream, int64_t* launches) {
  const Workspace w = workspace_of(p, p.S, ws);
  *launches += 2;
  fork_plan_kernel<<<p.S, kThreads, 0, stream>>>(p, parent, w);
  fork_apply_kernel<<<p.S, kThreads, 0, stream>>>(p, w);
  return cudaGetLastError();
}

cudaError_t launch_pages_resize(const PoolArgs& p, const int32_t* want, const CacheArgs& c, void* ws, int sms,
                                cudaStream_t stream, int64_t* launches) {
  const Workspace w = workspace_of(p, p.S, ws);
  *launches += 2;
  resize_plan_kernel<<<1, kPlanThreads, 0, stream>>>(p, want, w);
  resize_apply_kernel<<<p.S + 8 * sms, kThreads, 0, stream>>>(p, c, w);
  return cudaGetLastError();
}

cudaError_t launch_pages_compact(const PoolArgs& p, const CacheArgs& c, int32_t* table_out, int32_t* ref_out, int32_t* n_used,
                                 void* ws, int sms, cudaStream_t stream, int64_t* launches) {
  const Workspace w = workspace_of(p, p.S, ws);
  *launches += 2;
  compact_plan_kernel<<<1, kPlanThreads, 0, stream>>>(p, ref_out, n_used, w);
  compact_apply_kernel<<<p.S + 8 * sms, kThreads, 0, stream>>>(p, c, table_out, w);
  return cudaGetLastError();
}

}  // namespace gto
