// gto_verify_tree: the walk of a drafted tree against the target's probabilities.
//
// One thread-block cluster of eight (or four) CTAs per sequence.  At every context it visits, the CTAs
// stream their shares of the target row into shared memory once, exchange (maximum, sum) through
// distributed shared memory, and every CTA makes the same decisions about the children from the
// same numbers; where the walk ends, the CTA whose range the random number falls into finds the
// token from its shared copy.  A row that is not visited is not read.
//
// Results are those of fp64 arithmetic: the token drawn from a vocabulary of 10^5 ids is decided by a
// cumulative sum, and with fp32 terms about one draw in a hundred from a flat distribution would fall
// to rounding.  But fp64 exponentials of all weights took 190 us where the row's bytes take 20
// (128 trees, 128 256 ids), so that every row is first summed with fp32 exponentials, and decisions
// are taken only where they are further from their border than the sum can be wrong (kSlack); a
// row where one is not is summed again in fp64, from shared memory.
#include <cooperative_groups.h>

#include "decode_common.cuh"

namespace gto {
namespace {

namespace cg = cooperative_groups;

constexpr int kMaxCluster = 8;
constexpr int kWarps = 8;                    // that share the row
constexpr int kThreads = (kWarps + 1) * 32;  // and one that knows the tree and decides

// How far a sum of fp32 weights can be from the true one, relative to the row's whole mass.  A weight
// 2^-a is off by 2^-22 (the exponential) and 3 * 2^-24 * a * ln 2 (roundings of its argument)
// relative to itself; the mean of a over the distribution is at most log2 V <= 19.6; eight weights are
// added in fp32, the rest in fp64.  In all below 3.2e-6.
constexpr double kSlack = 4e-6;

struct Part {
  double sum;     // of the CTA's weights, relative to the CTA's own maximum
  uint64_t best;  // key of the CTA's largest logit (with its id for the greedy walk)
  int bad;        // saw NaN
};

__device__ __forceinline__ double sum64(double v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(kFull, v, o);
  return v;
}

// Sum of the first kWidth lanes, for all lanes.
template <int kWidth>
__device__ __forceinline__ double sum_first(double v) {
#pragma unroll
  for (int o = kWidth / 2; o > 0; o >>= 1) v += __shfl_xor_sync(kFull, v, o);
  return __shfl_sync(kFull, v, 0);
}
// Inclusive sums over the lanes, up to `width` of them.
template <int kWidth>
__device__ __forceinline__ double scan64(double v, int lane) {
#pragma unroll
  for (int o = 1; o < kWidth; o <<= 1) {
    const double y = __shfl_up_sync(kFull, v, o);
    if (lane >= o) v += y;
  }
  return v;
}

// 2^x in fp64 for x <= 0, without branches, so that several run side by side (the library's exp took
// 300 cycles each, one after the other): Cody and Waite's reduction x = n + f, |f| <= 1/2, and the
// polynomial of degree 10 with the least largest relative error there (by Remez's exchange:
// 2.1e-16; 4.2e-16 in fp64).  Below 2^-1000 the result is 0; NaN gives NaN.
__device__ __forceinline__ double exp2_neg(double x) {
  const double t = x + 6755399441055744.0;  // 1.5 * 2^52: n in the low bits
  const double f = x - (t - 6755399441055744.0);
  double y = 7.0372933257405244e-09;
  y = fma(y, f, 1.0208538304121812e-07);
  y = fma(y, f, 1.321566273860974e-06);
  y = fma(y, f, 1.5252658114109489e-05);
  y = fma(y, f, 0.00015403529961352815);
  y = fma(y, f, 0.0013333558228566251);
  y = fma(y, f, 0.0096181291080343918);
  y = fma(y, f, 0.055504108664458804);
  y = fma(y, f, 0.24022650695908768);
  y = fma(y, f, 0.69314718055994973);
  y = fma(y, f, 1.0);
  const double r = __hiloint2double(__double2hiint(y) + (__double2loint(t) << 20), __double2loint(y));
  return x < -1000.0 ? 0.0 : r;
}

// Whether 16 bytes of logits hold a NaN.
template <typename T>
__device__ __forceinline__ bool has_nan(const uint4& v) {
  if (T::kBytes == 4) {
    const auto nan = [](uint32_t w) { return (w & 0x7fffffffu) > 0x7f800000u; };
    return nan(v.x) || nan(v.y) || nan(v.z) || nan(v.w);
  }
  // an absolute value above that of infinity carries into the sign
  constexpr uint32_t kInf = static_cast<uint32_t>(T::kNegInfElem) & 0x7fffu, kAdd = (0x7fffu - kInf) * 0x10001u;
  const auto nan = [](uint32_t w) { return (w & 0x7fff7fffu) + kAdd; };
  return ((nan(v.x) | nan(v.y) | nan(v.z) | nan(v.w)) & 0x80008000u) != 0;
}

// A 4- or 8-byte value into the same place of another CTA's shared memory.
template <typename V>
__device__ __forceinline__ void push(cg::cluster_group& cluster, V* place, int to, V value) {
  *cluster.map_shared_rank(place, to) = value;
}

template <typename T, int kCluster>
__global__ void __launch_bounds__(kThreads, kCluster == kMaxCluster ? 2 : 3) verify_tree_kernel(VerifyArgs a) {
  constexpr int E = T::kPerVec;
  constexpr int U = kCluster == kMaxCluster ? 8 : 4;  // vectors in flight per thread
  constexpr int kChunks = kMaxNodes / 32;
  extern __shared__ __align__(16) unsigned char s_raw[];  // the CTA's share of the row
  __shared__ Part s_part[2][kCluster];  // what the CTAs say of a row, sent by each to all
  __shared__ int s_redo;                // sent by the owner of the last token
  __shared__ double s_wsum[kWarps];
  __shared__ float s_wmax[kWarps];
  __shared__ int s_wbad[kWarps], s_wid[kWarps];
  __shared__ int s_id[kMaxNodes];                        // target ids of the nodes
  __shared__ int s_removed[kMaxNodes];                   // ids of the refused children
  __shared__ double s_p[kMaxNodes];                      // and their weights
  __shared__ int s_child, s_owner, s_close;
  __shared__ double s_run[kWarps * 32];                  // sums of runs of vectors
  __shared__ int s_from;
  __shared__ float s_top;

  cg::cluster_group cluster = cg::this_cluster();
  // the others' shared memory may be written once all have begun: waited for before the first push
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  bool joined = false;
  const int rank = static_cast<int>(cluster.block_rank());
  const int s = blockIdx.x / kCluster;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const bool control = warp == kWarps;
  const int nvec = a.V_target / E;
  const int per = (nvec + kCluster - 1) / kCluster;
  const int vec0 = min(rank * per, nvec), vecs = min(vec0 + per, nvec) - vec0;
  const int per_warp = (vecs + kWarps - 1) / kWarps;  // a warp owns a contiguous range
  const int w0 = control ? 0 : min(warp * per_warp, vecs), w1 = control ? 0 : min(w0 + per_warp, vecs);
  uint4* s_vec = reinterpret_cast<uint4*>(s_raw);
  using Elem = typename T::Storage;

  const float temperature = a.temperature[s];
  const bool greedy = temperature == 0.f;
  const bool cold_ok = temperature >= 0.f && temperature < INFINITY;
  const double c64 = greedy ? 0.0 : 1.4426950408889634 / static_cast<double>(temperature);  // to log2 units
  const float c2 = static_cast<float>(c64);
  const auto unit = [](float u) { return static_cast<double>(fminf(fmaxf(u, 0.f), 0.99999994f)); };

  const double u_last = unit(a.u_bonus[s]);
  // the control warp's: ids and parents of the tree
  int id[kChunks], parent[kChunks];
  if (control) {
    int nodes = a.n_nodes ? a.n_nodes[s] : a.g;
    bool report = nodes < 0 || nodes > a.g;
    if (report) nodes = 0;
#pragma unroll
    for (int c = 0; c < kChunks; ++c) {
      const int n = c * 32 + lane;
      id[c] = -1;
      parent[c] = -2;  // no context's child
      if (n < nodes) {
        const int64_t at = static_cast<int64_t>(s) * a.g + n;
        const int tok = a.node_token[at], par = a.node_parent[at];
        if (tok >= 0 && tok < a.V_draft) id[c] = a.d2t ? a.d2t[tok] : tok;
        if (id[c] >= 0 && id[c] < a.V_target && par >= -1 && par < n) parent[c] = par;
        else report = true;
        s_id[n] = id[c];
      }
    }
    if (report) atomicOr(a.status, kStatusBadIndex);
  }

  int cur = -1, row = 0, len = 0, bonus = -1;
  bool exact = false;  // the row is in shared memory and is summed again, in fp64
  float m_warp = -INFINITY;
  for (int step = 0; cold_ok; ++step) {
    const bool ex = exact || !(c2 < 1e30f);  // (a temperature next to 0 is beyond fp32)
    const char* z = a.target + (static_cast<int64_t>(s) * a.rows + row) * a.V_target * T::kBytes;
    float kid_z[kChunks], kid_u[kChunks];
    if (control) {
      // the children's logits and random numbers, on their way while the row is
#pragma unroll
      for (int c = 0; c < kChunks; ++c) {
        kid_z[c] = kid_u[c] = 0.f;
        if (parent[c] == cur) {
          kid_z[c] = T::load1(z, id[c]);
          if (!greedy) kid_u[c] = a.u_node[static_cast<int64_t>(s) * a.g + c * 32 + lane];
        }
      }
    } else if (!exact) {
      // ---- the row's share: shared memory, maximum, soundness
      typename T::MaxAcc acc = T::max_init();
      bool bad = false;
      for (int i = w0 + lane; i < w1; i += 32 * U) {
        uint4 x[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (i + 32 * u < w1) x[u] = ld_stream16(z + static_cast<int64_t>(vec0 + i + 32 * u) * 16);
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (i + 32 * u < w1) {
            s_vec[i + 32 * u] = x[u];
            T::max_update(acc, x[u]);
            bad |= has_nan<T>(x[u]);
          }
      }
      m_warp = warp_max_f32(T::max_value(acc));
      bad = __any_sync(kFull, bad);
      if (lane == 0) {
        s_wmax[warp] = m_warp;
        s_wbad[warp] = bad;
      }
    }
    __syncthreads();
    float m_cta = s_wmax[0];
    int any_bad = s_wbad[0];
#pragma unroll
    for (int w = 1; w < kWarps; ++w) {
      m_cta = fmaxf(m_cta, s_wmax[w]);
      any_bad |= s_wbad[w];
    }
    if (!control) {
      if (greedy) {
        // the lowest id of the share that has its maximum
        int at = 0x7fffffff;
        for (int i = w0 + lane; i < w1 && m_warp == m_cta; i += 32) {
          float f[E];
          T::unpack(s_vec[i], f);
#pragma unroll
          for (int e = E - 1; e >= 0; --e)
            if (f[e] == m_cta) at = min(at, (vec0 + i) * E + e);
        }
        at = __reduce_min_sync(kFull, at);
        if (lane == 0) s_wid[warp] = at;
      } else {
        // ---- the share's sum, relative to its own maximum
        double sum = 0.0;
        if (m_cta != -INFINITY) {
          if (ex) {
            for (int i = w0 + lane; i < w1; i += 32) {
              float f[E];
              T::unpack(s_vec[i], f);
#pragma unroll
              for (int e = 0; e < E; ++e)
                sum += exp2_neg((static_cast<double>(f[e]) - static_cast<double>(m_cta)) * c64);
            }
          } else {
            for (int i = w0 + lane; i < w1; i += 32) {
              float f[E];
              T::unpack(s_vec[i], f);
              float part = 0.f;
#pragma unroll
              for (int e = 0; e < E; ++e) part += ex2_approx((f[e] - m_cta) * c2);
              sum += static_cast<double>(part);
            }
          }
        }
        sum = sum64(sum);
        if (lane == 0) s_wsum[warp] = sum;
      }
    }
    __syncthreads();
    if (!joined) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    joined = true;
    if (tid < kCluster) {  // one thread for each CTA that hears it
      double sum = 0.0;
      int at = 0;
      if (greedy) {
        at = s_wid[0];
        for (int w = 1; w < kWarps; ++w) at = min(at, s_wid[w]);
        if (at == 0x7fffffff) at = 0;
      } else {
        for (int w = 0; w < kWarps; ++w) sum += s_wsum[w];
      }
      Part* mine = &s_part[step & 1][rank];
      push(cluster, &mine->sum, tid, sum);
      push(cluster, &mine->best, tid, make_key(m_cta, at));
      push(cluster, &mine->bad, tid, any_bad);
    }
    cluster.sync();
    // ---- the control warp of every CTA: the row's maximum and sum, and the children
    double scale = 0.0, total = 0.0, aim = 0.0, before_cta = 0.0;
    float M = 0.f;
    int removed = 0;
    if (control) {
      uint64_t b = 0;
      int wrong = 0;
      double part = 0.0;
      if (lane < kCluster) {
        const Part& p = s_part[step & 1][lane];
        b = p.best;
        wrong = p.bad;
        part = p.sum;
      }
      const uint64_t row_best = warp_max_u64(b);
      wrong = __any_sync(kFull, wrong);
      M = key_value(row_best);
      const bool sound = !wrong && M != -INFINITY && M != INFINITY;
      // a CTA's weights, to the row's maximum
      if (lane < kCluster && !greedy && sound && key_value(b) != -INFINITY)
        scale = exp2_neg((static_cast<double>(key_value(b)) - static_cast<double>(M)) * c64);
      part *= scale;
      // the row's sum, added in the same order everywhere
      total = sum_first<kCluster>(part);
      const double slack = ex ? 0.0 : kSlack * total;
      double gone = 0.0;  // weight of the refused children so far
      int child = -1;
      bool close = false;  // a decision is too near its border for these sums
      if (sound) {
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
          const bool is = parent[c] == cur;
          const unsigned kids = __ballot_sync(kFull, is);
          if (kids == 0 || child >= 0 || close) continue;
          if (greedy) {
            const unsigned hit = __ballot_sync(kFull, is && id[c] == key_id(row_best));
            if (hit != 0) child = c * 32 + __ffs(hit) - 1;
            continue;
          }
          // All children of the chunk at once: each as if those before it had been refused; the first
          // that is accepted is the child.  The token of an earlier sibling has nothing left.
          const unsigned same = __match_any_sync(kFull, is ? id[c] : -1 - lane);
          bool again = (same & ((1u << lane) - 1)) != 0;
          for (int r = 0; r < removed; ++r) again |= s_removed[r] == id[c];
          const bool tried = is && !again;
          double p = 0.0;
          if (tried) p = exp2_neg((static_cast<double>(kid_z[c]) - static_cast<double>(M)) * c64);
          const double upto = scan64<32>(p, lane);
          const double aim_p = unit(kid_u[c]) * (total - gone - (upto - p));
          const unsigned yes = __ballot_sync(kFull, tried && aim_p < p);
          const unsigned near = __ballot_sync(kFull, tried && p > 0.0 && fabs(aim_p - p) < slack);
          const int first = yes != 0 ? __ffs(yes) - 1 : 31;
          close = (near & (0xffffffffu >> (31 - first))) != 0;
          if (yes != 0) {
            child = c * 32 + first;
          } else {
            const unsigned out = __ballot_sync(kFull, tried);
            if (tried) {
              const int r = removed + __popc(out & ((1u << lane) - 1));
              s_removed[r] = id[c];
              s_p[r] = p;
            }
            removed += __popc(out);
            gone += __shfl_sync(kFull, upto, 31);
            __syncwarp();
          }
        }
        if (close) child = -1;
      }
      int owner = -1;
      if (sound && child < 0 && !greedy && !close) {
        // what is left of every CTA's range
        double rest_of = part;
        if (lane < kCluster) {
          const int lo = lane * per * E, hi = lo + per * E;
          for (int r = 0; r < removed; ++r)
            if (s_removed[r] >= lo && s_removed[r] < hi) rest_of -= s_p[r];
          rest_of = fmax(rest_of, 0.0);
        } else {
          rest_of = 0.0;
        }
        const double upto = scan64<kCluster>(rest_of, lane);
        aim = u_last * __shfl_sync(kFull, upto, kCluster - 1);
        // the last range that holds something and begins at or below aim, or the first that holds something
        const unsigned some = __ballot_sync(kFull, rest_of > 0.0) & ((1u << kCluster) - 1);
        const unsigned below = __ballot_sync(kFull, rest_of > 0.0 && upto - rest_of <= aim) & ((1u << kCluster) - 1);
        if (some != 0) owner = below != 0 ? 31 - __clz(below) : __ffs(some) - 1;
        before_cta = __shfl_sync(kFull, upto - rest_of, owner < 0 ? 0 : owner);
      }
      scale = __shfl_sync(kFull, scale, rank);
      if (lane == 0) {
        s_child = sound ? child : -2;
        s_owner = greedy && sound ? key_id(row_best) : owner;
        s_close = close;
      }
    }
    __syncthreads();
    const int child = s_child;
    if (child == -2) {
      if (tid == 0) atomicOr(a.status, kStatusNonFinite);
      break;
    }
    if (s_close) {  // the same everywhere
      exact = true;
      continue;
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
      exact = false;
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
    const int owner = s_owner;
    if (owner < 0) break;
    if (rank == owner) {
      double before = 0.0;
      if (control) {
        // what is left of the warps' ranges; the one that holds the token is the last that begins at or below aim
        double rest = lane < kWarps ? s_wsum[lane] * scale : 0.0;
        if (lane < kWarps) {
          const int lo = (vec0 + min(lane * per_warp, vecs)) * E, hi = (vec0 + min((lane + 1) * per_warp, vecs)) * E;
          for (int r = 0; r < removed; ++r)
            if (s_removed[r] >= lo && s_removed[r] < hi) rest -= s_p[r];
          rest = fmax(rest, 0.0);
        }
        const double upto = scan64<kWarps>(rest, lane);
        const unsigned some = __ballot_sync(kFull, rest > 0.0) & 0xffu;
        const unsigned below = __ballot_sync(kFull, rest > 0.0 && before_cta + (upto - rest) <= aim) & 0xffu;
        const int from = below != 0 ? 31 - __clz(below) : some != 0 ? __ffs(some) - 1 : 0;
        before = before_cta + __shfl_sync(kFull, upto - rest, from);
        // refused tokens leave the share
        for (int r = lane; r < removed; r += 32) {
          const int off = s_removed[r] - vec0 * E;
          if (off >= 0 && off < vecs * E) reinterpret_cast<Elem*>(s_raw)[off] = T::kNegInfElem;
        }
        if (lane == 0) {
          s_from = from;
          s_top = M;
        }
      }
      __syncthreads();
      // all row warps: a thread sums a run of that range's vectors
      const int i0 = min(s_from * per_warp, vecs), i1 = min(i0 + per_warp, vecs);
      const int run = (i1 - i0 + kWarps * 32 - 1) / (kWarps * 32);
      const float top = s_top;
      if (!control) {
        const int r0 = min(i0 + tid * run, i1), r1 = min(r0 + run, i1);
        double sum = 0.0;
        for (int i = r0; i < r1; ++i) {
          float f[E];
          T::unpack(s_vec[i], f);
          if (ex) {
#pragma unroll
            for (int e = 0; e < E; ++e) sum += exp2_neg((static_cast<double>(f[e]) - static_cast<double>(top)) * c64);
          } else {
            float part = 0.f;
#pragma unroll
            for (int e = 0; e < E; ++e) part += ex2_approx((f[e] - top) * c2);
            sum += static_cast<double>(part);
          }
        }
        s_run[tid] = sum;
      }
      __syncthreads();
      if (control) {
        const double slack = ex ? 0.0 : 2.0 * kSlack * total;
        // the lane whose runs hold the token, then the run: the first with a sum above aim, else the
        // last one with a weight
        double mine[kWarps], mine_sum = 0.0;
#pragma unroll
        for (int q = 0; q < kWarps; ++q) {
          mine[q] = s_run[lane * kWarps + q];
          mine_sum += mine[q];
        }
        const double upto = scan64<32>(mine_sum, lane);
        const unsigned over = __ballot_sync(kFull, mine_sum > 0.0 && before + upto > aim);
        const unsigned some = __ballot_sync(kFull, mine_sum > 0.0);
        const int l = over != 0 ? __ffs(over) - 1 : 31 - __clz(some | 1u);
        double at = before + (upto - mine_sum), acc = at;
        int which = 0;
        bool in = false;
#pragma unroll
        for (int q = 0; q < kWarps; ++q) {
          if (!in && mine[q] > 0.0) {
            which = q;
            at = acc;
            in = acc + mine[q] > aim;
          }
          acc += mine[q];
        }
        at = __shfl_sync(kFull, at, l);
        which = l * kWarps + __shfl_sync(kFull, which, l);
        const int v0 = min(i0 + which * run, i1), v1 = min(v0 + run, i1);
        int found = -1, last = -1;  // last: the last id with a weight, where rounding leaves aim behind it
        bool close = false;
        const int first_id = (vec0 + v0) * E, ids = (v1 - v0) * E;
        for (int e0 = 0; e0 < ids && found < 0; e0 += 32) {
          double wv = 0.0;
          if (e0 + lane < ids) {
            const float f = T::load1(s_raw, v0 * E + e0 + lane);
            wv = ex ? exp2_neg((static_cast<double>(f) - static_cast<double>(top)) * c64)
                    : static_cast<double>(ex2_approx((f - top) * c2));
          }
          const double sum = scan64<32>(wv, lane);
          const unsigned hit = __ballot_sync(kFull, wv > 0.0 && at + sum > aim);
          const unsigned live = __ballot_sync(kFull, wv > 0.0);
          if (hit != 0) {
            const int h = __ffs(hit) - 1;
            found = first_id + e0 + h;
            const bool near = aim - (at + sum - wv) < slack || at + sum - aim < slack;
            close = !ex && __shfl_sync(kFull, static_cast<int>(near), h) != 0;
          }
          if (live != 0) last = first_id + e0 + 31 - __clz(live);
          at += __shfl_sync(kFull, sum, 31);
        }
        if (found < 0) close = !ex;
        if (lane < kCluster) push(cluster, &s_redo, lane, static_cast<int>(close));
        if (lane == 0 && !close) a.token[static_cast<int64_t>(s) * (a.D + 1) + len] = found >= 0 ? found : last;
      }
    }
    cluster.sync();  // the owner's answer
    if (!ex && s_redo) {
      // the owner took the refused tokens out of its share: put them back
      if (rank == owner && control) {
        for (int r = lane; r < removed; r += 32) {
          const int off = s_removed[r] - vec0 * E;
          if (off >= 0 && off < vecs * E)
            reinterpret_cast<Elem*>(s_raw)[off] = reinterpret_cast<const Elem*>(z)[s_removed[r]];
        }
      }
      __syncthreads();
      exact = true;
      continue;
    }
    bonus = -3;  // written by the owner
    break;
  }
  if (!joined) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  // what the walk did not fill (nothing is sent to a CTA after the last cluster.sync() that it was in)
  if (rank == 0) {
    if (tid == 0) {
      if (!cold_ok) atomicOr(a.status, kStatusNonFinite);
      a.accept_len[s] = len;
      if (bonus != -3) a.token[static_cast<int64_t>(s) * (a.D + 1) + len] = bonus;
    }
    for (int j = len + tid; j < a.D; j += kThreads) a.path_node[static_cast<int64_t>(s) * a.D + j] = -1;
    for (int j = len + 1 + tid; j <= a.D; j += kThreads) a.token[static_cast<int64_t>(s) * (a.D + 1) + j] = -1;
  }
}

template <typename T, int kCluster>
cudaError_t verify_as(const VerifyArgs& a, cudaStream_t stream) {
  const int nvec = a.V_target / T::kPerVec;
  const size_t smem = static_cast<size_t>((nvec + kCluster - 1) / kCluster) * 16;
  if (smem > 48 * 1024) {
    const cudaError_t e = cudaFuncSetAttribute(verify_tree_kernel<T, kCluster>,
                                               cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem));
    if (e != cudaSuccess) return e;
  }
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
  return cudaLaunchKernelEx(&cfg, verify_tree_kernel<T, kCluster>, a);
}

template <typename T>
cudaError_t verify_as(const VerifyArgs& a, int sms, cudaStream_t stream) {
  // Eight CTAs a sequence give the shortest walk; where the sequences do not fit the device at three
  // CTAs an SM, four, as long as three shares of a row fit an SM.
  const size_t row = static_cast<size_t>(a.V_target) * T::kBytes;
  const bool many = static_cast<int64_t>(a.S) * kMaxCluster > 3ll * sms && row / 4 <= 70 * 1024;
  return many ? verify_as<T, kMaxCluster / 2>(a, stream) : verify_as<T, kMaxCluster>(a, stream);
}

}  // namespace

cudaError_t launch_verify_tree(const VerifyArgs& a, int sms, cudaStream_t stream, int64_t* launches) {
  ++*launches;
  if (a.dtype == GTO_BF16) return verify_as<Bf16>(a, sms, stream);
  if (a.dtype == GTO_F16) return verify_as<F16>(a, sms, stream);
  return verify_as<F32>(a, sms, stream);
}

}  // namespace gto
