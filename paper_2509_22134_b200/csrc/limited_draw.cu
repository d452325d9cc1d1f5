// gto_sample_tokens and gto_verify_tree_limited: tokens drawn from softmax(z / temperature) of which top-k,
// top-p and min-p leave a part.
//
// With w_i = exp((z_i - max z) / temperature) and the tokens in the order (z descending, id ascending), every
// limit keeps a prefix of that order, so that what stays is "above a border value, or at it with an id up
// to some id".  A border is found by asking how many tokens (top-k), or which mass (top-p), a value and all
// above it hold, bit by bit of the value; the token then is the first id at which the cumulative sum of
// what stays passes u times the whole.  A row is shared by a cluster of CTAs; all weights and sums are fp64.
#include "decode_common.cuh"
#include "exp2_fp64.cuh"

namespace gto {
namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kCluster = 8;

// The bits of orderable() in which values of a type differ.
template <typename T> constexpr int kKeyBits = 32;
template <> constexpr int kKeyBits<Bf16> = 16;
template <> constexpr int kKeyBits<F16> = 19;
template <typename T>
__device__ __forceinline__ uint32_t key_of(float z) {
  return orderable(z) >> (32 - kKeyBits<T>);
}

struct Sums {
  double mass;
  uint64_t top;  // maximum
  int count;
};
struct Found {
  double total, weight;
  int id;
};

struct Shared {
  Sums warp[kWarps], pub[2];
  double run_warp[kWarps], run_pub[2];
  Found found[2];
  int from;
  double from_at;
};

__device__ __forceinline__ uint32_t smem_of(const void* p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }
__device__ __forceinline__ uint32_t in_cta(uint32_t addr, int cta) {
  uint32_t r;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(cta));
  return r;
}
__device__ __forceinline__ double far_f64(const double* p, int cta) {
  double v;
  asm volatile("ld.shared::cluster.f64 %0, [%1];" : "=d"(v) : "r"(in_cta(smem_of(p), cta)) : "memory");
  return v;
}
__device__ __forceinline__ uint64_t far_u64(const uint64_t* p, int cta) {
  uint64_t v;
  asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(in_cta(smem_of(p), cta)) : "memory");
  return v;
}
__device__ __forceinline__ int far_i32(const int* p, int cta) {
  int v;
  asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(v) : "r"(in_cta(smem_of(p), cta)) : "memory");
  return v;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// A CTA's share of the row it is at.
template <typename T>
struct Share {
  const char* z;
  int vec0, vecs, run;  // vectors of 16 bytes; a thread owns `run` of them, one after the other
  int rank;
  int turn;  // of the double-buffered exchanges

  template <typename F>
  __device__ __forceinline__ void each(F f) const {  // f(value, id) over the thread's elements, ids ascending
    constexpr int E = T::kPerVec;
    const int lo = min(static_cast<int>(threadIdx.x) * run, vecs), hi = min(lo + run, vecs);
    for (int i = lo; i < hi; ++i) {
      const uint4 v = __ldg(reinterpret_cast<const uint4*>(z) + vec0 + i);
      float x[E];
      T::unpack(v, x);
#pragma unroll
      for (int e = 0; e < E; ++e) f(x[e], (vec0 + i) * E + e);
    }
  }

  // Sums over the row, the same in all threads of the cluster.
  __device__ __forceinline__ Sums reduce(Shared& sh, Sums v) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      v.mass += __shfl_xor_sync(kFull, v.mass, o);
      const uint64_t t = __shfl_xor_sync(kFull, v.top, o);
      v.top = t > v.top ? t : v.top;
      v.count += __shfl_xor_sync(kFull, v.count, o);
    }
    if (lane == 0) sh.warp[warp] = v;
    __syncthreads();
    if (threadIdx.x == 0) {
      Sums s = sh.warp[0];
      for (int w = 1; w < kWarps; ++w) {
        s.mass += sh.warp[w].mass;
        s.top = sh.warp[w].top > s.top ? sh.warp[w].top : s.top;
        s.count += sh.warp[w].count;
      }
      sh.pub[turn] = s;
    }
    cluster_sync();
    Sums s{0.0, 0, 0};
    for (int c = 0; c < kCluster; ++c) {
      s.mass += far_f64(&sh.pub[turn].mass, c);
      const uint64_t t = far_u64(&sh.pub[turn].top, c);
      s.top = t > s.top ? t : s.top;
      s.count += far_i32(&sh.pub[turn].count, c);
    }
    turn ^= 1;  // (the next exchange is of the other buffer; the one after it begins behind its barrier)
    return s;
  }

  // The first id at which the cumulative sum of weight(value, id) over the ids passes u * (the whole sum), or
  // `aim` where u < 0.  id -1 where nothing has a weight.
  template <typename F>
  __device__ __forceinline__ Found locate(Shared& sh, F weight, double u, double aim) {
    constexpr int E = T::kPerVec;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    double mine = 0.0;
    each([&](float x, int id) { mine += weight(x, id); });
    double upto = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const double y = __shfl_up_sync(kFull, upto, o);
      if (lane >= o) upto += y;
    }
    if (lane == 31) sh.run_warp[warp] = upto;
    if (threadIdx.x == 0) sh.from = -1;
    __syncthreads();
    double start = 0.0, all = 0.0;
    for (int w = 0; w < kWarps; ++w) {
      if (w == warp) start = all;
      all += sh.run_warp[w];
    }
    start += upto - mine;
    if (threadIdx.x == 0) sh.run_pub[turn] = all;
    cluster_sync();
    double total = 0.0, part[kCluster];
    for (int c = 0; c < kCluster; ++c) total += part[c] = far_f64(&sh.run_pub[turn], c);
    if (u >= 0.0) aim = u * total;
    // the last range that holds something and begins at or below aim
    int owner = -1;
    double before = 0.0, at = 0.0;
    for (int c = 0; c < kCluster; ++c) {
      if (part[c] > 0.0 && (owner < 0 || at <= aim)) {
        owner = c;
        before = at;
      }
      at += part[c];
    }
    if (owner == rank) {
      if (mine > 0.0 && before + start <= aim) atomicMax(&sh.from, static_cast<int>(threadIdx.x));
      __syncthreads();
      const bool none = sh.from < 0;  // (rounding: then the first that holds something)
      __syncthreads();
      if (none && mine > 0.0) atomicMax(&sh.from, kThreads + (kThreads - 1 - static_cast<int>(threadIdx.x)));
      __syncthreads();
      const int from = sh.from >= kThreads ? 2 * kThreads - 1 - sh.from : sh.from;
      if (static_cast<int>(threadIdx.x) == from) sh.from_at = before + start;
      __syncthreads();
      if (warp == 0) {
        const int lo = min(from * run, vecs) * E, hi = min(from * run + run, vecs) * E;
        double acc = sh.from_at;
        Found f{total, 0.0, -1};
        for (int e0 = lo; e0 < hi; e0 += 32) {
          const int id = vec0 * E + e0 + lane;
          const double w = e0 + lane < hi ? weight(T::load1(z, id), id) : 0.0;
          double sum = w;
#pragma unroll
          for (int o = 1; o < 32; o <<= 1) {
            const double y = __shfl_up_sync(kFull, sum, o);
            if (lane >= o) sum += y;
          }
          const unsigned hit = __ballot_sync(kFull, w > 0.0 && acc + sum > aim);
          const unsigned live = __ballot_sync(kFull, w > 0.0);
          const int at_lane = hit ? __ffs(hit) - 1 : live ? 31 - __clz(live) : -1;
          if (at_lane >= 0) {
            f.id = vec0 * E + e0 + at_lane;
            f.weight = __shfl_sync(kFull, w, at_lane);
          }
          if (hit) break;
          acc += __shfl_sync(kFull, sum, 31);
        }
        if (lane == 0) sh.found[turn] = f;
      }
    }
    cluster_sync();
    Found f{total, 0.0, -1};
    if (owner >= 0) {
      f.id = far_i32(&sh.found[turn].id, owner);
      f.weight = far_f64(&sh.found[turn].weight, owner);
    }
    turn ^= 1;
    return f;
  }
};

// What stays of a row.
struct Kept {
  uint32_t border;  // key
  int cut;          // of the tokens at the border those with an id up to cut stay
  double floor;     // weights below it do not
};

// kTree: walks a draft tree; else a row is a sequence.
template <typename T, bool kTree>
__global__ void __launch_bounds__(kThreads) limited_kernel(LimitedArgs a) {
  constexpr int E = T::kPerVec;
  __shared__ Shared sh;
  __shared__ int s_removed[kMaxNodes];
  __shared__ int s_child, s_removed_n;
  __shared__ double s_left;
  const int s = blockIdx.x / kCluster;
  const int tid = threadIdx.x, lane = tid & 31;
  Share<T> row;
  row.rank = static_cast<int>(blockIdx.x % kCluster);
  row.turn = 0;
  const bool first = row.rank == 0 && tid == 0;
  const int nvec = a.V / E, per = (nvec + kCluster - 1) / kCluster;
  row.vec0 = min(row.rank * per, nvec);
  row.vecs = min(row.vec0 + per, nvec) - row.vec0;
  row.run = (row.vecs + kThreads - 1) / kThreads;

  const float heat = a.temperature[s];
  const bool greedy = heat == 0.f;
  const int top_k = a.top_k ? a.top_k[s] : 0;
  const float top_p = a.top_p ? a.top_p[s] : 1.f, min_p = a.min_p ? a.min_p[s] : 0.f;
  const bool sound = heat >= 0.f && heat < INFINITY && top_p == top_p && min_p == min_p;
  const double scale = greedy ? 0.0 : 1.4426950408889634 / static_cast<double>(heat);
  const auto unit = [](float u) { return static_cast<double>(fminf(fmaxf(u, 0.f), 0.99999994f)); };
  const double u_last = unit(a.u[s]);

  int64_t at_row = s;
  bool lost = false;  // no such row
  if (!kTree && a.rows) {
    at_row = a.rows[s];
    lost = at_row < 0 || at_row >= a.n_rows;
    if (lost && first) atomicOr(a.status, kStatusBadIndex);
  }
  int nodes = 0;
  if (kTree) {
    nodes = a.n_nodes ? a.n_nodes[s] : a.g;
    if (nodes < 0 || nodes > a.g) {
      nodes = 0;
      if (first) atomicOr(a.status, kStatusBadIndex);
    }
  }
  // Target id of node n of the tree, -1 for one that is not to be followed.
  const auto node_id = [&](int n) {
    const int64_t at = static_cast<int64_t>(s) * a.g + n;
    const int tok = a.node_token[at], par = a.node_parent[at];
    int id = -1;
    if (tok >= 0 && tok < a.V_draft) id = a.d2t ? a.d2t[tok] : tok;
    return id >= 0 && id < a.V && par >= -1 && par < n ? id : -1;
  };
  if (kTree) {
    bool bad = false;
    for (int n = tid; n < nodes; n += kThreads) bad |= node_id(n) < 0;
    if (bad && row.rank == 0) atomicOr(a.status, kStatusBadIndex);
  }

  int len = 0, cur = -1, last = -1, kept_n = 0;
  float logp = 0.f;
  if (!sound && first) atomicOr(a.status, kStatusNonFinite);
  bool go = sound && !lost;
  if (kTree) at_row = static_cast<int64_t>(s) * a.rows_of_tree;
  int64_t here = at_row;
  while (go) {
    go = false;
    row.z = a.logits + here * a.row_stride;
    // ---- the largest logit
    Sums v{0.0, 0, 0};
    row.each([&](float x, int id) {
      const uint64_t k = make_key(x, id);
      v.top = k > v.top ? k : v.top;
      v.count += x != x;
      v.mass += x > -INFINITY ? 1.0 : 0.0;
    });
    v = row.reduce(sh, v);
    const float M = key_value(v.top);
    if (v.count > 0 || !(fabsf(M) < INFINITY)) {
      if (first) atomicOr(a.status, kStatusNonFinite);
      break;
    }
    const int finite = static_cast<int>(v.mass);
    const int best = key_id(v.top);
    const auto raw = [&](float x) { return exp2_neg((static_cast<double>(x) - static_cast<double>(M)) * scale); };
    // ---- what stays
    Kept kept{key_of<T>(-INFINITY), -1, static_cast<double>(fminf(fmaxf(min_p, 0.f), 1.f))};
    double total = 1.0;
    kept_n = 1;
    if (!greedy) {
      const auto stays = [&](float x, int id) {
        const uint32_t k = key_of<T>(x);
        return k > kept.border || (k == kept.border && id <= kept.cut);
      };
      if (top_k > 0 && top_k < finite) {
        uint32_t t = 0;
        for (int bit = kKeyBits<T> - 1; bit >= 0; --bit) {
          const uint32_t c = t | (1u << bit);
          Sums n{0.0, 0, 0};
          row.each([&](float x, int id) { n.count += key_of<T>(x) >= c; });
          if (row.reduce(sh, n).count >= top_k) t = c;
        }
        Sums n{0.0, 0, 0};
        row.each([&](float x, int id) { n.count += key_of<T>(x) > t; });
        const int ties = top_k - row.reduce(sh, n).count;
        kept.border = t;
        kept.cut = row.locate(sh, [&](float x, int id) { return key_of<T>(x) == t ? 1.0 : 0.0; }, -1.0, ties - 0.5).id;
      }
      if (top_p < 1.f) {
        Sums n{0.0, 0, 0};
        row.each([&](float x, int id) { n.mass += stays(x, id) ? raw(x) : 0.0; });
        const double goal = static_cast<double>(top_p) * row.reduce(sh, n).mass;
        uint32_t t = 0;
        for (int bit = kKeyBits<T> - 1; bit >= 0; --bit) {
          const uint32_t c = t | (1u << bit);
          n = Sums{0.0, 0, 0};
          row.each([&](float x, int id) {
            if (stays(x, id) && key_of<T>(x) >= c) {
              n.mass += raw(x);
              ++n.count;
            }
          });
          const Sums r = row.reduce(sh, n);
          if (r.count > 0 && r.mass >= goal) t = c;
        }
        if (t > kept.border || (t == kept.border && kept.cut >= 0)) {
          n = Sums{0.0, 0, 0};
          row.each([&](float x, int id) {
            const uint32_t k = key_of<T>(x);
            if (k > t) n.mass += raw(x);
            if (k == t && stays(x, id)) {
              ++n.count;
              n.top = make_key(x, 0);
            }
          });
          const Sums r = row.reduce(sh, n);
          const double w = raw(key_value(r.top));
          // the fewest of the equal ones that reach the goal
          double j = fmin(fmax(w > 0.0 ? ceil((goal - r.mass) / w) : 1.0, 1.0), static_cast<double>(r.count));
          while (j > 1.0 && r.mass + (j - 1.0) * w >= goal) j -= 1.0;
          while (j < r.count && r.mass + j * w < goal) j += 1.0;
          const Kept was = kept;
          kept.cut = row.locate(
              sh, [&](float x, int id) { return key_of<T>(x) == t && (t > was.border || id <= was.cut) ? 1.0 : 0.0; }, -1.0, j - 0.5).id;
          kept.border = t;
        }
      }
      Sums n{0.0, 0, 0};
      row.each([&](float x, int id) {
        if (!stays(x, id)) return;
        const double w = raw(x);
        if (kept.floor > 0.0 && w < kept.floor) return;
        n.mass += w;
        ++n.count;
      });
      n = row.reduce(sh, n);
      total = n.mass;
      kept_n = n.count;
    }
    const auto weight = [&](float x, int id) {
      const uint32_t k = key_of<T>(x);
      if (!(k > kept.border || (k == kept.border && id <= kept.cut))) return 0.0;
      const double w = raw(x);
      return kept.floor > 0.0 && w < kept.floor ? 0.0 : w;
    };
    int removed = 0;
    if (kTree) {
      // ---- the children of the context, in list order (the same in every CTA)
      __syncthreads();
      if (tid == 0) {
        int child = -1;
        double left = total;
        for (int n = cur + 1; n < nodes && child < 0; ++n) {
          if (a.node_parent[static_cast<int64_t>(s) * a.g + n] != cur) continue;
          const int id = node_id(n);
          if (id < 0) continue;
          if (greedy) {
            if (id == best) child = n;
            continue;
          }
          bool again = false;
          for (int r = 0; r < removed; ++r) again |= s_removed[r] == id;
          if (again) continue;
          const double p = weight(T::load1(row.z, id), id);
          if (unit(a.u_node[static_cast<int64_t>(s) * a.g + n]) * left < p) {
            child = n;
          } else {
            s_removed[removed++] = id;
            left -= p;
          }
        }
        s_child = child;
        s_removed_n = removed;
      }
      __syncthreads();
      removed = s_removed_n;
      const int child = s_child;
      if (child >= 0) {
        if (len == a.D) {  // a tree deeper than it may be
          if (first) atomicOr(a.status, kStatusBadIndex);
          break;
        }
        if (first) {
          a.path_node[static_cast<int64_t>(s) * a.D + len] = child;
          a.token[static_cast<int64_t>(s) * (a.D + 1) + len] = node_id(child);
        }
        ++len;
        cur = child;
        if (a.context_rows) {
          const int64_t at_node = static_cast<int64_t>(s) * a.g + child;
          const int depth = a.node_depth[at_node], slot = a.node_slot[at_node];
          if (slot < 0 || depth >= a.D) break;  // never expanded: no row, no token after it
          if (depth < 1 || slot >= a.k) {
            if (first) atomicOr(a.status, kStatusBadIndex);
            break;
          }
          here = at_row + 1 + (depth - 1) * a.k + slot;
        } else {
          here = at_row + 1 + child;
        }
        go = true;
        continue;
      }
    }
    if (greedy) {
      last = best;
      break;
    }
    const Found f = row.locate(
        sh,
        [&](float x, int id) {
          for (int r = 0; r < removed; ++r)
            if (s_removed[r] == id) return 0.0;
          return weight(x, id);
        },
        u_last, 0.0);
    last = f.id;
    if (f.id >= 0) logp = static_cast<float>(log(f.weight / total));
  }
  cluster_sync();  // nobody leaves while its shared memory is read
  if (row.rank != 0) return;
  if (kTree) {
    if (tid == 0) {
      a.accept_len[s] = len;
      a.token[static_cast<int64_t>(s) * (a.D + 1) + len] = last;
    }
    for (int j = len + tid; j < a.D; j += kThreads) a.path_node[static_cast<int64_t>(s) * a.D + j] = -1;
    for (int j = len + 1 + tid; j <= a.D; j += kThreads) a.token[static_cast<int64_t>(s) * (a.D + 1) + j] = -1;
  } else if (tid == 0) {
    a.token[s] = last;
    if (a.logp) a.logp[s] = last < 0 ? 0.f : logp;
    if (a.n_kept) a.n_kept[s] = last < 0 ? 0 : kept_n;
  }
}

template <typename T>
cudaError_t limited_as(const LimitedArgs& a, bool tree, cudaStream_t stream) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(static_cast<unsigned>(a.N) * kCluster);
  cfg.blockDim = dim3(kThreads);
  cfg.stream = stream;
  cudaLaunchAttribute attr{};
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = kCluster;
  attr.val.clusterDim.y = 1;
  attr.val.clusterDim.z = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return tree ? cudaLaunchKernelEx(&cfg, limited_kernel<T, true>, a) : cudaLaunchKernelEx(&cfg, limited_kernel<T, false>, a);
}

}  // namespace

cudaError_t launch_limited(const LimitedArgs& a, bool tree, cudaStream_t stream, int64_t* launches) {
  ++*launches;
  if (a.dtype == GTO_BF16) return limited_as<Bf16>(a, tree, stream);
  if (a.dtype == GTO_F16) return limited_as<F16>(a, tree, stream);
  return limited_as<F32>(a, tree, stream);
}

}  // namespace gto
