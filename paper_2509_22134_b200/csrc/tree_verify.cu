// gto_verify_tree: the walk of a drafted tree against the target's probabilities.
//
// One thread-block cluster of eight CTAs per sequence.  At every context it visits, the CTAs stream
// their eighths of the target row into shared memory once, exchange (maximum, sum) through
// distributed shared memory, and every CTA makes the same decisions about the children from the
// same numbers; where the walk ends, the CTA whose range the random number falls into finds the
// token from its shared copy.  A row that is not visited is not read.
//
// Every weight exp((z - max) / temperature), every sum and every comparison is fp64: the token drawn
// from a vocabulary of 10^5 ids is decided by a cumulative sum, and with fp32 terms (relative
// error 2^-23 each) about one draw in a hundred from a flat distribution would fall to rounding.
#include <cooperative_groups.h>

#include "decode_common.cuh"

namespace gto {
namespace {

namespace cg = cooperative_groups;

constexpr int kCluster = 8;
constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;

struct Part {
  double sum;     // of the CTA's weights, relative to the CTA's own maximum
  uint64_t best;  // (value, id) key of the CTA's largest logit
  int bad;        // saw NaN or +inf
};

__device__ __forceinline__ double sum64(double v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(kFull, v, o);
  return v;
}

template <typename T>
__global__ void __launch_bounds__(kThreads) verify_tree_kernel(VerifyArgs a) {
  constexpr int E = T::kPerVec;
  extern __shared__ __align__(16) unsigned char s_raw[];  // the CTA's share of the row
  __shared__ Part s_part[2];
  __shared__ double s_wsum[kWarps];
  __shared__ uint64_t s_wbest[kWarps];
  __shared__ int s_wbad[kWarps];
  __shared__ int s_id[kMaxNodes], s_parent[kMaxNodes];   // target ids and parents of the nodes
  __shared__ double s_p[kMaxNodes];                      // weights of the refused children
  __shared__ double s_rest[kCluster + 1];                // cumulative remaining weight of the CTAs
  __shared__ int s_child, s_removed[kMaxNodes], s_n_removed, s_owner;
  __shared__ double s_target;

  cg::cluster_group cluster = cg::this_cluster();
  const int rank = static_cast<int>(cluster.block_rank());
  const int s = blockIdx.x / kCluster;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int nvec = a.V_target / E;
  const int per = (nvec + kCluster - 1) / kCluster;
  const int vec0 = min(rank * per, nvec), vecs = min(vec0 + per, nvec) - vec0;
  const int per_warp = (vecs + kWarps - 1) / kWarps;  // a warp owns a contiguous range
  const int w0 = min(warp * per_warp, vecs), w1 = min(w0 + per_warp, vecs);
  const uint4* s_vec = reinterpret_cast<const uint4*>(s_raw);
  using Elem = typename T::Storage;

  const float temperature = a.temperature[s];
  const bool greedy = temperature == 0.f;
  const bool cold_ok = temperature >= 0.f && temperature < INFINITY;
  const double inv_t = greedy ? 1.0 : 1.0 / static_cast<double>(temperature);
  int nodes = a.n_nodes ? a.n_nodes[s] : a.g;
  bool tree_ok = nodes >= 0 && nodes <= a.g;
  if (!tree_ok) nodes = 0;
  bool report = !tree_ok;
  for (int n = tid; n < nodes; n += kThreads) {
    const int64_t at = static_cast<int64_t>(s) * a.g + n;
    const int tok = a.node_token[at], par = a.node_parent[at];
    int id = -1;
    if (tok >= 0 && tok < a.V_draft) id = a.d2t ? a.d2t[tok] : tok;
    const bool good = id >= 0 && id < a.V_target && par >= -1 && par < n;
    s_id[n] = good ? id : -1;
    s_parent[n] = good ? par : -2;  // no context's child
    report |= !good;
  }
  if (report) atomicOr(a.status, kStatusBadIndex);
  float u_last = a.u_bonus[s];
  u_last = fminf(fmaxf(u_last, 0.f), 0.99999994f);

  int cur = -1, row = 0, len = 0, bonus = -1;
  for (int step = 0; cold_ok; ++step) {
    const char* z = a.target + (static_cast<int64_t>(s) * a.rows + row) * a.V_target * T::kBytes;
    // ---- the row's share: shared memory, maximum, soundness
    float m = -INFINITY;
    int at = 0;
    bool bad = false;
    for (int i = w0 + lane; i < w1; i += 32) {
      const uint4 x = ld_stream16(z + static_cast<int64_t>(vec0 + i) * 16);
      reinterpret_cast<uint4*>(s_raw)[i] = x;
      float f[E];
      T::unpack(x, f);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        bad |= !(f[e] < INFINITY);
        if (f[e] > m) {
          m = f[e];
          at = (vec0 + i) * E + e;
        }
      }
    }
    const uint64_t best = warp_max_u64(make_key(m, at));
    bad = __any_sync(kFull, bad);
    if (lane == 0) {
      s_wbest[warp] = best;
      s_wbad[warp] = bad;
    }
    __syncthreads();
    uint64_t top = s_wbest[0];
    int any_bad = s_wbad[0];
#pragma unroll
    for (int w = 1; w < kWarps; ++w) {
      top = s_wbest[w] > top ? s_wbest[w] : top;
      any_bad |= s_wbad[w];
    }
    const float m_cta = key_value(top);
    // ---- the share's sum, relative to its own maximum
    if (!greedy) {
      double sum = 0.0;
      if (m_cta != -INFINITY) {
        for (int i = w0 + lane; i < w1; i += 32) {
          float f[E];
          T::unpack(s_vec[i], f);
#pragma unroll
          for (int e = 0; e < E; ++e)
            sum += exp((static_cast<double>(f[e]) - static_cast<double>(m_cta)) * inv_t);
        }
      }
      sum = sum64(sum);
      if (lane == 0) s_wsum[warp] = sum;
      __syncthreads();
    }
    Part& mine = s_part[step & 1];
    if (tid == 0) {
      mine.best = top;
      mine.bad = any_bad;
      double sum = 0.0;
      if (!greedy)
        for (int w = 0; w < kWarps; ++w) sum += s_wsum[w];
      mine.sum = sum;
    }
    cluster.sync();
    // ---- every CTA: the row's maximum and sum, and the children
    if (warp == 0) {
      uint64_t b = 0;
      int wrong = 0;
      double part = 0.0;
      if (lane < kCluster) {
        const Part* p = cluster.map_shared_rank(&s_part[step & 1], lane);
        b = p->best;
        wrong = p->bad;
        part = p->sum;
      }
      const uint64_t row_best = warp_max_u64(b);
      wrong = __any_sync(kFull, wrong);
      const float M = key_value(row_best);
      const bool sound = !wrong && M != -INFINITY;
      if (lane < kCluster && !greedy && sound)
        part = key_value(b) == -INFINITY
                   ? 0.0
                   : part * exp((static_cast<double>(key_value(b)) - static_cast<double>(M)) * inv_t);
      // the CTAs' weights in id order, and the row's sum, added in the same order everywhere
      double total = 0.0;
#pragma unroll
      for (int q = 0; q < kCluster; ++q) total += __shfl_sync(kFull, part, q);
      double left = total;
      int child = -1, removed = 0;
      if (sound) {
        for (int n0 = 0; n0 < nodes && child < 0; n0 += 32) {
          const int n = n0 + lane;
          const bool is = n < nodes && s_parent[n] == cur;
          unsigned kids = __ballot_sync(kFull, is);
          if (kids == 0) continue;
          const int id = is ? s_id[n] : -1;
          double p = 0.0;
          double u = 0.0;
          if (is && !greedy) {
            p = exp((static_cast<double>(T::load1(z, id)) - static_cast<double>(M)) * inv_t);
            u = static_cast<double>(fminf(fmaxf(a.u_node[static_cast<int64_t>(s) * a.g + n], 0.f), 0.99999994f));
          }
          while (kids != 0 && child < 0) {
            const int l = __ffs(kids) - 1;
            kids &= kids - 1;
            const int kid_id = __shfl_sync(kFull, id, l);
            if (greedy) {
              if (kid_id == key_id(row_best)) child = n0 + l;
              continue;
            }
            double kp = __shfl_sync(kFull, p, l);
            const double ku = __shfl_sync(kFull, u, l);
            // the token of an earlier sibling has nothing left
            bool gone = false;
            for (int r = lane; r < removed; r += 32) gone |= s_removed[r] == kid_id;
            if (__any_sync(kFull, gone)) continue;
            if (ku * left < kp) {
              child = n0 + l;
            } else {
              left -= kp;
              if (lane == 0) {
                s_removed[removed] = kid_id;
                s_p[removed] = kp;
              }
              ++removed;
              __syncwarp();
            }
          }
        }
      }
      int owner = -1;
      if (sound && child < 0 && !greedy) {
        // what is left of every CTA's range
        if (lane < kCluster) {
          const int lo = lane * per * E, hi = lo + per * E;
          for (int r = 0; r < removed; ++r)
            if (s_removed[r] >= lo && s_removed[r] < hi) part -= s_p[r];
          part = fmax(part, 0.0);
        } else {
          part = 0.0;
        }
        double acc = 0.0;
        double rest = 0.0;
#pragma unroll
        for (int q = 0; q < kCluster; ++q) rest += __shfl_sync(kFull, part, q);
        const double aim = static_cast<double>(u_last) * rest;
#pragma unroll
        for (int q = 0; q < kCluster; ++q) {
          const double pq = __shfl_sync(kFull, part, q);
          if (lane == 0) s_rest[q] = acc;
          if (pq > 0.0 && (owner < 0 || acc <= aim)) owner = q;
          acc += pq;
        }
        if (lane == 0) s_target = aim;
      }
      if (lane == 0) {
        s_child = sound ? child : -2;
        s_n_removed = removed;
        s_owner = greedy && sound ? key_id(row_best) : owner;
      }
    }
    __syncthreads();
    const int child = s_child;
    if (child == -2) {
      if (tid == 0) atomicOr(a.status, kStatusNonFinite);
      break;
    }
    if (child >= 0) {
      if (len == a.D) {  // a tree deeper than it may be
        if (tid == 0) atomicOr(a.status, kStatusBadIndex);
        break;
      }
      if (rank == 0 && tid == 0) {
        a.path_node[static_cast<int64_t>(s) * a.D + len] = child;
        a.token[static_cast<int64_t>(s) * (a.D + 1) + len] = s_id[child];
      }
      ++len;
      cur = child;
      if (a.context_rows) {
        const int64_t at_node = static_cast<int64_t>(s) * a.g + child;
        const int depth = a.node_depth[at_node], slot = a.node_slot[at_node];
        if (slot < 0 || depth >= a.D) break;  // never expanded: no row, no token after it
        if (depth < 1 || slot >= a.k) {
          if (tid == 0) atomicOr(a.status, kStatusBadIndex);
          break;
        }
        row = 1 + (depth - 1) * a.k + slot;
      } else {
        row = 1 + child;
      }
      continue;  // the shared decision is rewritten only after the next cluster.sync()
    }
    // ---- nothing accepted: the last token
    if (greedy) {
      bonus = s_owner;
      break;
    }
    if (rank == s_owner) {
      // the refused tokens leave the share, then the range's sums find the token
      for (int r = tid; r < s_n_removed; r += kThreads) {
        const int off = s_removed[r] - vec0 * E;
        if (off >= 0 && off < vecs * E) reinterpret_cast<Elem*>(s_raw)[off] = T::kNegInfElem;
      }
      __syncthreads();
      const float M = [&] {
        uint64_t b = 0;
        for (int q = 0; q < kCluster; ++q) {
          const uint64_t o = cluster.map_shared_rank(&s_part[step & 1], q)->best;
          b = o > b ? o : b;
        }
        return key_value(b);
      }();
      auto weight = [&](float f) {
        return exp((static_cast<double>(f) - static_cast<double>(M)) * inv_t);
      };
      double sum = 0.0;
      for (int i = w0 + lane; i < w1; i += 32) {
        float f[E];
        T::unpack(s_vec[i], f);
#pragma unroll
        for (int e = 0; e < E; ++e) sum += weight(f[e]);
      }
      sum = sum64(sum);
      if (lane == 0) s_wsum[warp] = sum;
      __syncthreads();
      if (warp == 0) {
        double before = s_rest[s_owner];
        const double aim = s_target;
        int from = 0;  // the warp range that holds the token: the last one that begins at or below aim
        double acc = before;
        bool any = false;
        for (int w = 0; w < kWarps; ++w) {
          if (s_wsum[w] > 0.0 && (!any || acc <= aim)) {
            from = w;
            before = acc;
            any = true;
          }
          acc += s_wsum[w];
        }
        int found = -1, last = -1;  // last: the last id with a weight, where rounding leaves aim behind it
        const int i0 = min(from * per_warp, vecs), i1 = min(i0 + per_warp, vecs);
        for (int i = i0; i < i1 && found < 0; i += 32) {
          float f[E];
          double wv[E];
          double mine_sum = 0.0;
          int mine_last = -1;
          const bool live = i + lane < i1;
          if (live) {
            T::unpack(s_vec[i + lane], f);
#pragma unroll
            for (int e = 0; e < E; ++e) {
              wv[e] = weight(f[e]);
              mine_sum += wv[e];
              if (wv[e] > 0.0) mine_last = (vec0 + i + lane) * E + e;
            }
          }
          double run = mine_sum;  // inclusive scan over the lanes
#pragma unroll
          for (int o = 1; o < 32; o <<= 1) {
            const double y = __shfl_up_sync(kFull, run, o);
            if (lane >= o) run += y;
          }
          const unsigned over = __ballot_sync(kFull, live && before + run > aim);
          if (over != 0) {
            const int l = __ffs(over) - 1;
            int hit = -1;
            if (lane == l) {
              double acc2 = before + (run - mine_sum);
              int tail = -1;
#pragma unroll
              for (int e = 0; e < E; ++e) {
                acc2 += wv[e];
                if (wv[e] > 0.0) {
                  tail = (vec0 + i + lane) * E + e;
                  if (hit < 0 && acc2 > aim) hit = tail;
                }
              }
              if (hit < 0) hit = tail;
            }
            found = __shfl_sync(kFull, hit, l);
          }
          const int batch_last = __reduce_max_sync(kFull, mine_last);
          last = batch_last > last ? batch_last : last;
          before += __shfl_sync(kFull, run, 31);
        }
        if (lane == 0)
          a.token[static_cast<int64_t>(s) * (a.D + 1) + len] = found >= 0 ? found : last;
      }
    }
    if (s_owner >= 0) bonus = -3;  // written by the owner
    break;
  }
  // what the walk did not fill
  if (rank == 0) {
    if (tid == 0) {
      if (!cold_ok) atomicOr(a.status, kStatusNonFinite);
      a.accept_len[s] = len;
      if (bonus != -3) a.token[static_cast<int64_t>(s) * (a.D + 1) + len] = bonus;
    }
    for (int j = len + tid; j < a.D; j += kThreads) a.path_node[static_cast<int64_t>(s) * a.D + j] = -1;
    for (int j = len + 1 + tid; j <= a.D; j += kThreads) a.token[static_cast<int64_t>(s) * (a.D + 1) + j] = -1;
  }
  cluster.sync();  // no CTA leaves while its partial sums may be read
}

template <typename T>
cudaError_t verify_as(const VerifyArgs& a, cudaStream_t stream) {
  const int nvec = a.V_target / T::kPerVec;
  const size_t smem = static_cast<size_t>((nvec + kCluster - 1) / kCluster) * 16;
  cudaError_t e = cudaFuncSetAttribute(verify_tree_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                       static_cast<int>(kMaxTargetRow / kCluster + 16));
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(static_cast<unsigned>(a.S) * kCluster);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr{};
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = kCluster;
  attr.val.clusterDim.y = 1;
  attr.val.clusterDim.z = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, verify_tree_kernel<T>, a);
}

}  // namespace

cudaError_t launch_verify_tree(const VerifyArgs& a, int sms, cudaStream_t stream, int64_t* launches) {
  (void)sms;
  ++*launches;
  if (a.dtype == GTO_BF16) return verify_as<Bf16>(a, stream);
  if (a.dtype == GTO_F16) return verify_as<F16>(a, stream);
  return verify_as<F32>(a, stream);
}

}  // namespace gto
