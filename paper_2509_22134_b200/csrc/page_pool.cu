// gto_pages_fork, gto_pages_resize, gto_pages_compact: who holds which pages of the cache.
//
// The state is a table of pages for every sequence and a count for every page of how often the tables name
// it; a page that nobody names is free, there is no list of free pages to keep in order.  Fresh pages are the
// lowest free ones, given out in the order of the sequences, so that equal calls give equal tables; counts
// change by integer atomics, whose order does not matter.  A call is a plan (what every sequence needs, read
// from the tables as they stood) and then its execution by another kernel, so that nothing is read after another
// sequence has changed it.
//
// What bounds it, as measured on a B200: moving pages, the copy (a pool of 48 sequences of which 1.47 GB move: 470 to 498 us, 91 to
// 97 % of a plain copy's rate); sharing and reserving, latency (6 us for two kernels that depend on one another at 4 sequences,
// 16 us where one CTA numbers 256 sequences and searches a table of free pages: three rounds of loads
// and block-wide sums, which a single CTA does without a barrier across the device).
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

// Sum of v over the threads before this one; *all receives the sum over all.  s_warp: 32 ints.
__device__ __forceinline__ int scan_before(int v, int* s_warp, int* all) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const auto scan = [&](int x) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(kFull, x, o);
      if (lane >= o) x += y;
    }
    return x;
  };
  const int upto = scan(v);
  __syncthreads();  // (s_warp may still be read from the last call)
  if (lane == 31) s_warp[warp] = upto;
  __syncthreads();
  const int warps = scan(s_warp[lane]);  // every warp for itself
  *all = __shfl_sync(kFull, warps, 31);
  return __shfl_sync(kFull, warps, warp) - s_warp[warp] + upto - v;
}

__device__ __forceinline__ bool is_page(const PoolArgs& p, int page) { return page >= 0 && page < p.n_pages; }
__device__ __forceinline__ int pages_of(const PoolArgs& p, int entries) {
  return static_cast<int>((static_cast<int64_t>(entries) + p.page_size - 1) / p.page_size);
}
// Whether a sequence's numbers fit each other.
__device__ __forceinline__ bool fits(const PoolArgs& p, int held, int len) {
  return held >= 0 && held <= p.max_pages && len >= 0 && len <= static_cast<int64_t>(held) * p.page_size;
}

// A plan lets its execution get ready, which waits for it.
__device__ __forceinline__ void plan_begins() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void wait_for_plan() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// ---- fork
__global__ void __launch_bounds__(kThreads) fork_plan_kernel(PoolArgs p, const int32_t* parent, Workspace w) {
  plan_begins();
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
    const int32_t* own = p.page_table + static_cast<int64_t>(s) * p.max_pages;
    constexpr int kKeep = 4;  // of each row's pages a thread reads these at once
    int page[kKeep], old[kKeep];
    if (bad) need = 0;
#pragma unroll
    for (int i = 0; i < kKeep; ++i) {
      const int j = tid + i * kThreads;
      page[i] = j < need ? row[j] : -1;
      old[i] = !bad && j < held ? own[j] : -1;
    }
#pragma unroll
    for (int i = 0; i < kKeep; ++i) bad |= tid + i * kThreads < need && !is_page(p, page[i]);
    for (int j = tid + kKeep * kThreads; j < need; j += kThreads) bad |= !is_page(p, row[j]);
    bad = __syncthreads_or(bad);
    if (!bad) {
      bool odd = false;
      const auto take = [&](int j, int q) {
        w.rows[static_cast<int64_t>(s) * p.max_pages + j] = q;
        atomicAdd(p.ref_count + q, 1);
      };
      const auto drop = [&](int q) {
        if (is_page(p, q)) atomicSub(p.ref_count + q, 1);
        else odd = true;
      };
#pragma unroll
      for (int i = 0; i < kKeep; ++i) {
        const int j = tid + i * kThreads;
        if (j < need) take(j, page[i]);
        if (j < held) drop(old[i]);
      }
      for (int j = tid + kKeep * kThreads; j < need; j += kThreads) take(j, row[j]);
      for (int j = tid + kKeep * kThreads; j < held; j += kThreads) drop(own[j]);
      if (odd) atomicOr(p.status, kStatusBadIndex);
    }
  }
  if (tid == 0) {
    w.plan[s] = Plan{bad ? -1 : need, len, 0, 0};
    if (bad) atomicOr(p.status, kStatusBadIndex);
  }
}

__global__ void __launch_bounds__(kThreads) fork_apply_kernel(PoolArgs p, Workspace w) {
  wait_for_plan();
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
  plan_begins();
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
  int total = 0, any_swaps = 0;
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
    any_swaps |= plan.swaps > 0;
  }
  any_swaps = __syncthreads_or(any_swaps);
  // the lowest free pages, as many as are needed (a thread looks at kLook neighbours at a time)
  constexpr int kLook = 4;
  int found = 0;
  for (int p0 = 0; p0 < p.n_pages && found < total; p0 += kLook * kPlanThreads) {
    const int first = p0 + kLook * tid;
    int count[kLook], n = 0;
#pragma unroll
    for (int i = 0; i < kLook; ++i) count[i] = first + i < p.n_pages ? p.ref_count[first + i] : 1;
#pragma unroll
    for (int i = 0; i < kLook; ++i) n += count[i] == 0;
    int sum;
    int at = found + scan_before(n, s_warp, &sum);
#pragma unroll
    for (int i = 0; i < kLook; ++i)
      if (count[i] == 0 && at < total) w.list[at++] = first + i;
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
    if (!any_swaps) continue;
    int sum;
    const int at = n_copies + scan_before(copy.entries > 0, s_warp, &sum);
    if (copy.entries > 0) w.copies[at] = copy;
    n_copies += sum;
  }
  if (tid == 0) w.counts[0] = n_copies;
}

// ---- copies of pages: units of kUnit bytes of the keys or the values of one layer, eight loads of 16 bytes a thread on their
// way at a time.
constexpr int kAtOnce = 8;
constexpr int kUnit = kAtOnce * kThreads;  // vectors
constexpr int kCopyBlocks = 6;             // CTAs an SM

struct Units {
  int cols;           // vectors of an entry: heads one after the other
  int per_head;       // vectors of a head
  int chunks;         // units of a page
  bool k_dense, v_dense;  // whether the entries of a page lie without gaps
};

// f(i, &from, &to, &entries): the i-th copy of n.
template <typename F>
__device__ __forceinline__ void copy_pages(const CacheArgs& c, const Units& u, int n, int block, int blocks, F f) {
  const int64_t parts = 2ll * c.n_layers * u.chunks, units = n * parts;
  for (int64_t unit = block; unit < units; unit += blocks) {
    const int copy = static_cast<int>(unit / parts);
    const uint32_t part = static_cast<uint32_t>(unit - copy * parts);
    const int layer = static_cast<int>(part / u.chunks >> 1), chunk = static_cast<int>(part % u.chunks);
    const bool key = part / u.chunks & 1;
    int src, dst, entries;
    f(copy, &src, &dst, &entries);
    const int64_t page = key ? c.k_page : c.v_page;
    char* base = (key ? c.k : c.v) + layer * (key ? c.k_layer : c.v_layer);
    const char* from = base + src * page;
    char* to = base + dst * page;
    const int64_t size = static_cast<int64_t>(entries) * u.cols;
    const int64_t first = static_cast<int64_t>(chunk) * kUnit + threadIdx.x;
    if (first - threadIdx.x >= size) continue;
    uint4 x[kAtOnce];
    if (key ? u.k_dense : u.v_dense) {
#pragma unroll
      for (int b = 0; b < kAtOnce; ++b)
        if (first + b * kThreads < size) x[b] = ld_stream16(from + (first + b * kThreads) * 16);
#pragma unroll
      for (int b = 0; b < kAtOnce; ++b)
        if (first + b * kThreads < size) st_stream16(to + (first + b * kThreads) * 16, x[b]);
    } else {
      const int64_t entry = key ? c.k_entry : c.v_entry, head = key ? c.k_head : c.v_head;
      const auto place = [&](int b) {
        const int64_t i = first + b * kThreads;
        const int64_t e = i / u.cols;
        const uint32_t col = static_cast<uint32_t>(i - e * u.cols);
        return e * entry + (col / u.per_head) * head + (col % u.per_head) * 16;
      };
#pragma unroll
      for (int b = 0; b < kAtOnce; ++b)
        if (first + b * kThreads < size) x[b] = ld_stream16(from + place(b));
#pragma unroll
      for (int b = 0; b < kAtOnce; ++b)
        if (first + b * kThreads < size) st_stream16(to + place(b), x[b]);
    }
  }
}

// Block s < S: the tables of sequence s; the others: the copies.
__global__ void __launch_bounds__(kThreads) resize_apply_kernel(PoolArgs p, CacheArgs c, Units u, Workspace w) {
  wait_for_plan();
  if (static_cast<int>(blockIdx.x) >= p.S) {
    copy_pages(c, u, w.counts[0], blockIdx.x - p.S, gridDim.x - p.S, [&](int i, int* src, int* dst, int* entries) {
      const Copy copy = w.copies[i];
      *src = copy.src;
      *dst = copy.dst;
      *entries = copy.entries;
    });
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
  plan_begins();
  const int tid = threadIdx.x;
  int used = 0;
#pragma unroll 8
  for (int page = tid; page < p.n_pages; page += kPlanThreads) used += p.ref_count[page] > 0;
  int total;
  scan_before(used, s_warp, &total);
  int holes = 0, movers = 0;
  int32_t* hole = w.to + p.n_pages;
  constexpr int kLook = 4;
  for (int p0 = 0; p0 < p.n_pages; p0 += kLook * kPlanThreads) {
    const int first = p0 + kLook * tid;
    int count[kLook], n = 0;  // holes below, movers from `total` on: never both at one page
#pragma unroll
    for (int i = 0; i < kLook; ++i) count[i] = first + i < p.n_pages ? p.ref_count[first + i] : 0;
#pragma unroll
    for (int i = 0; i < kLook; ++i) {
      const int page = first + i;
      if (page < p.n_pages) n += page < total ? count[i] <= 0 : (count[i] > 0) << 16;
    }
    int sum;
    const int before = scan_before(n, s_warp, &sum);  // (4096 pages a turn: neither half overflows)
    int at_hole = holes + (before & 0xffff), at_move = movers + (before >> 16);
    holes += sum & 0xffff;
    movers += sum >> 16;
#pragma unroll
    for (int i = 0; i < kLook; ++i) {
      const int page = first + i;
      if (page >= p.n_pages) continue;
      const bool is_used = count[i] > 0;
      if (!is_used && page < total) hole[at_hole++] = page;
      if (is_used && page >= total) w.list[at_move++] = page;
      w.to[page] = page;
      ref_out[page] = is_used && page < total ? count[i] : 0;
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
__global__ void __launch_bounds__(kThreads) compact_apply_kernel(PoolArgs p, CacheArgs c, Units u, int32_t* table_out, Workspace w) {
  wait_for_plan();
  if (static_cast<int>(blockIdx.x) >= p.S) {
    copy_pages(c, u, w.counts[0], blockIdx.x - p.S, gridDim.x - p.S, [&](int i, int* src, int* dst, int* entries) {
      *src = w.list[i];
      *dst = w.to[*src];
      *entries = p.page_size;
    });
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

Workspace workspace_of(const PoolArgs& p, void* ws) {
  Workspace w;
  layout(p.S, p.max_pages, p.n_pages, static_cast<char*>(ws), &w);
  return w;
}

Units units_of(const PoolArgs& p, const CacheArgs& c) {
  Units u;
  const int e = c.dtype == GTO_F32 ? 4 : 2, head = c.head_dim * e;
  u.per_head = head / 16;
  u.cols = c.n_kv_heads * u.per_head;
  u.chunks = static_cast<int>((static_cast<int64_t>(p.page_size) * u.cols + kUnit - 1) / kUnit);
  const auto dense = [&](int64_t entry, int64_t h) {
    return (c.n_kv_heads == 1 || h == head) && (p.page_size == 1 || entry == static_cast<int64_t>(c.n_kv_heads) * head);
  };
  u.k_dense = dense(c.k_entry, c.k_head);
  u.v_dense = dense(c.v_entry, c.v_head);
  return u;
}

// The execution of a plan.
template <typename... P, typename... A>
cudaError_t after_plan(void (*kernel)(P...), int blocks, cudaStream_t stream, A... args) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(static_cast<unsigned>(blocks));
  cfg.blockDim = dim3(kThreads);
  cfg.stream = stream;
  cudaLaunchAttribute attr{};
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}

}  // namespace

size_t pages_workspace(const gto_decode_config& c) { return layout(c.S, c.max_pages, c.n_pages, nullptr, nullptr); }

cudaError_t launch_pages_fork(const PoolArgs& p, const int32_t* parent, void* ws, cudaStream_t stream, int64_t* launches) {
  const Workspace w = workspace_of(p, ws);
  *launches += 2;
  fork_plan_kernel<<<p.S, kThreads, 0, stream>>>(p, parent, w);
  const cudaError_t e = cudaGetLastError();
  return e != cudaSuccess ? e : after_plan(fork_apply_kernel, p.S, stream, p, w);
}

cudaError_t launch_pages_resize(const PoolArgs& p, const int32_t* want, const CacheArgs& c, void* ws, int sms,
                                cudaStream_t stream, int64_t* launches) {
  const Workspace w = workspace_of(p, ws);
  *launches += 2;
  resize_plan_kernel<<<1, kPlanThreads, 0, stream>>>(p, want, w);
  const cudaError_t e = cudaGetLastError();
  return e != cudaSuccess ? e : after_plan(resize_apply_kernel, p.S + kCopyBlocks * sms, stream, p, c, units_of(p, c), w);
}

cudaError_t launch_pages_compact(const PoolArgs& p, const CacheArgs& c, int32_t* table_out, int32_t* ref_out, int32_t* n_used,
                                 void* ws, int sms, cudaStream_t stream, int64_t* launches) {
  const Workspace w = workspace_of(p, ws);
  *launches += 2;
  compact_plan_kernel<<<1, kPlanThreads, 0, stream>>>(p, ref_out, n_used, w);
  const cudaError_t e = cudaGetLastError();
  return e != cudaSuccess ? e : after_plan(compact_apply_kernel, p.S + kCopyBlocks * sms, stream, p, c, units_of(p, c), table_out, w);
}

}  // namespace gto
