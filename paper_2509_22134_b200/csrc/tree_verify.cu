// gto_verify_tree: the walk of a drafted tree against the target's probabilities.
//
// One thread-block cluster of eight CTAs per sequence.  At every context it visits, the CTAs go
// through their shares of the target row once (seven warps, each with a range of its own, so that a
// last token is looked for in one warp's range only), tell one another (reference, sum) by stores into
// each other's shared memory that a barrier there counts, and an eighth warp of every CTA makes the same decisions about the children from
// the same numbers.  Where the walk ends, the CTA whose range the random number falls into reads that
// range again and finds the token.  A row that is not visited is not read.
//
// Results are those of fp64 arithmetic: the token drawn from a vocabulary of 10^5 ids is decided by a
// cumulative sum, and with fp32 terms about one draw in a hundred from a flat distribution would fall
// to rounding.  But fp64 exponentials of all weights took 190 us where the row's bytes take 20
// (128 trees, 128 256 ids), so that every row is first summed with fp32 exponentials, and decisions
// are taken only where they are further from their border than the sum can be wrong (kSlack); a
// row where one is not is summed again in fp64.
//
// What bounds it is the chain: a sequence's rows come one after another, 8 of them for the longest
// walk of the 128, and a row is a load's latency (0.8 us), a thread's 72 to 144 weights (1.5 to 4 us,
// depending on how many CTAs share the SM), the exchange and the decision (2.5 us); a draw from
// the flat tail then costs the row in fp64 (4 us alone, 15 us when all sequences do).  Measured: one
// tree of 32 000 ids 12.6 us, 128 trees of 128 256 ids 80 us (13.2 and 84 us with the cluster's own
// barrier for the exchange; 103 us with the row kept in shared memory, which left room for three
// quarters of the clusters and took a second pass for the weights).
#include "decode_common.cuh"

namespace gto {
namespace {

constexpr int kCluster = 8;                  // CTAs of a sequence
constexpr int kWarps = 7;                    // that share the row
constexpr int kWidth = 8;                    // lanes that their sums take
constexpr int kLost = -4;                    // another CTA was not heard of
constexpr int kThreads = (kWarps + 1) * 32;  // and one that knows the tree and decides

// A thread's vectors of a row come through shared memory, kBatch at a time, kGroups batches on their way.
constexpr int kRowThreads = kWarps * 32;
constexpr int kBatch = 3, kGroups = 4;
constexpr int kStageBytes = kBatch * kGroups * kRowThreads * 16;
static_assert(((kMaxTargetRow / 16 / kCluster + 1) / kWarps + 1) * 16 <= kStageBytes, "a warp's range fits");

// How far a thread's reference may lie below its largest logit, in log2 units: rescaling for every new
// maximum took longer than the weights.
constexpr float kReach = 4.f;

// How far a sum of fp32 weights can be from the true one, relative to the row's whole mass.  A weight
// 2^-a is off by 2^-22 (the exponential) and 3 * 2^-24 * (a + kReach) * ln 2 (roundings of its argument)
// relative to itself; the mean of a over the distribution is at most log2 V <= 19.6; 24 weights are
// added in fp32, in five levels (5 * 2^-24), the rest in fp64.  In all below 3.5e-6.
constexpr double kSlack = 4e-6;

struct alignas(16) Part {
  double sum;     // of the CTA's weights, relative to the CTA's own reference; NaN: it saw one
  uint64_t best;  // key of the CTA's largest logit (with its id for the greedy walk)
};

__device__ __forceinline__ double sum64(double v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(kFull, v, o);
  return v;
}

// Sum of the first kLanes lanes, for all lanes.
template <int kLanes>
__device__ __forceinline__ double sum_first(double v) {
#pragma unroll
  for (int o = kLanes / 2; o > 0; o >>= 1) v += __shfl_xor_sync(kFull, v, o);
  return __shfl_sync(kFull, v, 0);
}
// Inclusive sums over the lanes, up to kLanes of them.
template <int kLanes>
__device__ __forceinline__ double scan64(double v, int lane) {
#pragma unroll
  for (int o = 1; o < kLanes; o <<= 1) {
    const double y = __shfl_up_sync(kFull, v, o);
    if (lane >= o) v += y;
  }
  return v;
}

// 2^x in fp64 for x <= 4, without branches, so that several run side by side (the library's exp took
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

// The largest of 16 bytes of logits, of two packed 16-bit ones at a time; NaN if one of them is.
template <typename T>
__device__ __forceinline__ uint32_t max_word(uint32_t a, uint32_t b) {
  uint32_t d;
  if (T::kBytes == 4) asm("max.NaN.f32 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  else if (T::kNegInfElem == 0xff80u) asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  else asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
template <typename T>
__device__ __forceinline__ uint32_t max_of(const uint4& v) {
  return max_word<T>(max_word<T>(v.x, v.y), max_word<T>(v.z, v.w));
}
template <typename T>
__device__ __forceinline__ float max_half(uint32_t w) {  // of the word's two halves
  if (T::kBytes == 4) return __uint_as_float(w);
  w = max_word<T>(w, __byte_perm(w, w, 0x1032));
  return T::load1(&w, 0);
}

// Sum of the weights of 16 bytes of logits, 2^((f - m) c2), in fp32: pairs side by side.
template <typename T>
__device__ __forceinline__ float weights(const uint4& v, float m, float c2) {
  constexpr int E = T::kPerVec;
  float f[E];
  T::unpack(v, f);
  uint64_t neg, scale, sum[E / 2];
  asm("mov.b64 %0, {%1, %1};" : "=l"(neg) : "f"(-m));
  asm("mov.b64 %0, {%1, %1};" : "=l"(scale) : "f"(c2));
#pragma unroll
  for (int e = 0; e < E / 2; ++e) {
    float a, b;
    asm("{\n .reg .b64 x;\n mov.b64 x, {%2, %3};\n add.rn.f32x2 x, x, %4;\n mul.rn.f32x2 x, x, %5;\n mov.b64 {%0, %1}, x;\n}"
        : "=f"(a), "=f"(b)
        : "f"(f[2 * e]), "f"(f[2 * e + 1]), "l"(neg), "l"(scale));
    a = ex2_approx(a);
    b = ex2_approx(b);
    asm("mov.b64 %0, {%1, %2};" : "=l"(sum[e]) : "f"(a), "f"(b));
  }
#pragma unroll
  for (int w = E / 4; w > 0; w /= 2)
#pragma unroll
    for (int e = 0; e < w; ++e) asm("add.rn.f32x2 %0, %1, %2;" : "=l"(sum[e]) : "l"(sum[e]), "l"(sum[e + w]));
  float a, b;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(sum[0]));
  return a + b;
}

// ---- what a CTA tells the others: a store into their shared memory that their barrier counts
__device__ __forceinline__ uint32_t smem_of(const void* p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }
__device__ __forceinline__ uint32_t in_cta(uint32_t addr, int cta) {
  uint32_t r;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(cta));
  return r;
}
__device__ __forceinline__ void tell(uint32_t to, uint64_t a, uint64_t b, uint32_t bar) {
  asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v2.b64 [%0], {%1, %2}, [%3];" ::"r"(to), "l"(a),
               "l"(b), "r"(bar)
               : "memory");
}
__device__ __forceinline__ void tell(uint32_t to, uint32_t a, uint32_t bar) {
  asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.b32 [%0], %1, [%2];" ::"r"(to), "r"(a), "r"(bar)
               : "memory");
}
__device__ __forceinline__ void expect(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
// Waits for the phase of that parity, at most about two seconds; false if it has not ended.
__device__ __forceinline__ bool heard(uint32_t bar, uint32_t parity) {
  uint32_t ok = 0;
  for (int i = 0; i < 20000 && !ok; ++i)
    asm volatile(
        "{\n .reg .pred p;\n mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2, 100000;\n"
        " selp.u32 %0, 1, 0, p;\n}"
        : "=r"(ok)
        : "r"(bar), "r"(parity)
        : "memory");
  return __all_sync(kFull, ok);
}

template <typename T, int kResident>
__global__ void __launch_bounds__(kThreads, kResident) verify_tree_kernel(VerifyArgs a) {
  constexpr int E = T::kPerVec;
  constexpr int kChunks = kMaxNodes / 32;
  extern __shared__ __align__(16) unsigned char s_raw[];  // vectors on their way; a warp's range, where the last token is
  __shared__ Part s_part[2][kCluster];  // what the CTAs say of a row, sent by each to all
  __shared__ int s_redo;                // sent by the owner of the last token
  __shared__ uint64_t s_bar[3];         // that s_part[0], s_part[1], s_redo have come
  __shared__ double s_wsum[kWarps];
  __shared__ float s_wmax[kWarps];
  __shared__ int s_wbad[kWarps], s_wid[kWarps];
  __shared__ int s_id[kMaxNodes];                        // target ids of the nodes
  __shared__ int s_removed[kMaxNodes];                   // ids of the refused children
  __shared__ double s_p[kMaxNodes];                      // and their weights
  __shared__ int s_child, s_owner, s_close;
  __shared__ double s_run[kWarps * 32];                  // sums of runs of vectors
  __shared__ int s_from, s_out;
  __shared__ float s_top;

  const uint32_t bar = smem_of(s_bar);
  if (threadIdx.x == 0) {
    for (int i = 0; i < 3; ++i) asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(bar + i * 8) : "memory");
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncwarp();
  // the others' shared memory may be written once all have begun: waited for before the first push
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  bool joined = false;
  const int rank = static_cast<int>(blockIdx.x % kCluster);
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

  // The warp's range of a row, for the row warps: take(x, i) with x the vectors i, i + 32, ... below w1.  A
  // thread waits only for what it copied itself.
  const auto fetch = [&](const char* z, int b) {
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const int i = w0 + lane + 32 * (b * kBatch + u);
      if (i < w1)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(static_cast<uint32_t>(
                         __cvta_generic_to_shared(s_vec + ((b % kGroups) * kBatch + u) * kRowThreads + tid))),
                     "l"(z + static_cast<int64_t>(vec0 + i) * 16)
                     : "memory");
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  const auto stream = [&](const char* z, auto&& take) {
#pragma unroll
    for (int b = 0; b < kGroups; ++b) fetch(z, b);
#pragma unroll 1
    for (int b = 0; w0 + 32 * kBatch * b < w1; ++b) {
      asm volatile("cp.async.wait_group %0;" ::"n"(kGroups - 1) : "memory");
      uint4 x[kBatch];
#pragma unroll
      for (int u = 0; u < kBatch; ++u) x[u] = s_vec[((b % kGroups) * kBatch + u) * kRowThreads + tid];
      take(x, w0 + lane + 32 * kBatch * b);
      fetch(z, b + kGroups);
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
  };

  int cur = -1, row = 0, len = 0, bonus = -1;
  bool exact = false;  // the row is summed again, in fp64
  uint32_t asked = 0;  // answers of an owner so far
  bool lost = false;   // another CTA was not heard of in time
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
      // ---- the row's share in one pass: a thread's weights are relative to about the largest logit that
      // it has met (what it had is rescaled in fp64, which costs the sum nothing)
      float m = -INFINITY;
      double sum = 0.0;
      bool bad = false;
      uint4 best[kBatch] = {};  // greedy: the first batch that had the maximum
      int best_i = w1;
      const float reach = kReach / c2;
      stream(z, [&](const uint4 (&x)[kBatch], int i) {
        uint32_t word = T::kNegInfWord;
#pragma unroll
        for (int u = 0; u < kBatch; ++u)
          if (i + 32 * u < w1) word = max_word<T>(word, max_of<T>(x[u]));
        const float top = max_half<T>(word);
        bad |= top != top;
        if (greedy || ex) {
          if (top > m) {
            m = top;
            best_i = i;
#pragma unroll
            for (int u = 0; u < kBatch; ++u) best[u] = x[u];
          }
          return;
        }
        if (m == -INFINITY ? top > m : top > m + reach) {
          if (sum != 0.0) sum *= exp2_neg((static_cast<double>(m) - static_cast<double>(top)) * c64);
          m = top;
        }
        if (m == -INFINITY) return;
        float part[kBatch];
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
          part[u] = 0.f;
          if (i + 32 * u < w1) part[u] = weights<T>(x[u], m, c2);
        }
        sum += static_cast<double>((part[0] + part[1]) + part[2]);
      });
      const float m_warp = warp_max_f32(m);
      if (sum != 0.0) sum *= exp2_neg((static_cast<double>(m) - static_cast<double>(m_warp)) * c64);
      sum = sum64(sum);
      bad = __any_sync(kFull, bad);
      if (lane == 0) {
        s_wmax[warp] = m_warp;
        s_wbad[warp] = bad;
        s_wsum[warp] = sum;
      }
      if (greedy) {
        // the lowest id of the warp's range that has its maximum
        int at = 0x7fffffff;
#pragma unroll
        for (int u = kBatch - 1; u >= 0; --u) {
          float f[E];
          T::unpack(best[u], f);
#pragma unroll
          for (int e = E - 1; e >= 0; --e)
            if (f[e] == m_warp && best_i + 32 * u < w1) at = (vec0 + best_i + 32 * u) * E + e;
        }
        at = __reduce_min_sync(kFull, at);
        if (lane == 0) s_wid[warp] = at;
      }
    }
    __syncthreads();
    float m_cta = s_wmax[0];
#pragma unroll
    for (int w = 1; w < kWarps; ++w) m_cta = fmaxf(m_cta, s_wmax[w]);
    if (ex && !greedy) {  // the sums once more (or for the first time), in fp64
      if (!control) {
        double sum = 0.0;
        if (m_cta != -INFINITY) {
          stream(z, [&](const uint4 (&x)[kBatch], int i) {
#pragma unroll 1
            for (int u = 0; u < kBatch; ++u) {
              if (i + 32 * u >= w1) break;
              float f[E];
              T::unpack(u == 0 ? x[0] : u == 1 ? x[1] : x[2], f);
#pragma unroll
              for (int e = 0; e < E; ++e) sum += exp2_neg((static_cast<double>(f[e]) - static_cast<double>(m_cta)) * c64);
            }
          });
        }
        sum = sum64(sum);
        if (lane == 0) s_wsum[warp] = sum;
      }
      __syncthreads();
    }
    if (!joined) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    joined = true;
    double warp_sum = 0.0;  // the control warp's lane w: the sum of warp w's range, relative to the CTA's maximum
    if (control) {
      int at = 0x7fffffff, wrong = 0;
      if (lane < kWarps) {
        wrong = s_wbad[lane];
        if (greedy) {
          if (s_wmax[lane] == m_cta) at = s_wid[lane];
        } else {
          warp_sum = s_wsum[lane];
          if (!ex && warp_sum != 0.0)
            warp_sum *= exp2_neg((static_cast<double>(s_wmax[lane]) - static_cast<double>(m_cta)) * c64);
        }
      }
      at = __reduce_min_sync(kFull, at);
      wrong = __any_sync(kFull, wrong);
      const double sum = sum_first<kWidth>(warp_sum);
      const uint32_t here = bar + (step & 1) * 8;
      if (lane == 0) expect(here, kCluster * sizeof(Part));
      if (lane < kCluster)  // one thread for each CTA that hears it
        tell(in_cta(smem_of(&s_part[step & 1][rank]), lane), __double_as_longlong(wrong ? NAN : sum),
             make_key(m_cta, at == 0x7fffffff ? 0 : at), in_cta(here, lane));
    }
    // ---- the control warp of every CTA: the row's maximum and sum, and the children
    double scale = 0.0, total = 0.0, aim = 0.0, before_cta = 0.0;
    float M = 0.f;
    int removed = 0;
    if (control) {
      // (a CTA is at most one step ahead of another: it needs the other's part of every step)
      const bool all = heard(bar + (step & 1) * 8, step >> 1 & 1);
      uint64_t b = 0;
      double part = 0.0;
      if (lane < kCluster) {
        const Part& p = s_part[step & 1][lane];
        b = p.best;
        part = p.sum;
      }
      const uint64_t row_best = warp_max_u64(b);
      const bool wrong = __any_sync(kFull, part != part);
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
        s_child = !all ? kLost : sound ? child : -2;
        s_owner = greedy && sound ? key_id(row_best) : owner;
        s_close = close;
      }
    }
    __syncthreads();
    const int child = s_child;
    if (child <= -2) {
      lost = child == kLost;
      if (tid == 0 && !lost) atomicOr(a.status, kStatusNonFinite);
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
      continue;  // the shared decision is rewritten only after the next row
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
        double rest = warp_sum * scale;
        if (lane < kWarps) {
          const int lo = (vec0 + min(lane * per_warp, vecs)) * E, hi = (vec0 + min((lane + 1) * per_warp, vecs)) * E;
          for (int r = 0; r < removed; ++r)
            if (s_removed[r] >= lo && s_removed[r] < hi) rest -= s_p[r];
          rest = fmax(rest, 0.0);
        }
        const double upto = scan64<kWidth>(rest, lane);
        const unsigned some = __ballot_sync(kFull, rest > 0.0) & ((1u << kWarps) - 1);
        const unsigned below = __ballot_sync(kFull, rest > 0.0 && before_cta + (upto - rest) <= aim) & ((1u << kWarps) - 1);
        const int from = below != 0 ? 31 - __clz(below) : some != 0 ? __ffs(some) - 1 : 0;
        before = before_cta + __shfl_sync(kFull, upto - rest, from);
        if (lane == 0) {
          s_from = from;
          s_out = removed;
          s_top = M;
        }
      }
      __syncthreads();
      // all row warps: a thread sums a run of that range's vectors, read again
      const int i0 = min(s_from * per_warp, vecs), i1 = min(i0 + per_warp, vecs);
      const int run = (i1 - i0 + kWarps * 32 - 1) / (kWarps * 32);
      const float top = s_top;
      if (!control) {
        const int r0 = min(i0 + tid * run, i1), r1 = min(r0 + run, i1);
        for (int i = r0; i < r1; ++i) s_vec[i - i0] = ld_stream16(z + static_cast<int64_t>(vec0 + i) * 16);
        for (int r = 0; r < s_out; ++r) {  // refused tokens have nothing left
          const int off = s_removed[r] - vec0 * E;
          if (off >= r0 * E && off < r1 * E) reinterpret_cast<Elem*>(s_raw)[off - i0 * E] = T::kNegInfElem;
        }
        double sum = 0.0;
        for (int i = r0; i < r1; ++i) {
          float f[E];
          T::unpack(s_vec[i - i0], f);
          if (ex) {
#pragma unroll
            for (int e = 0; e < E; ++e) sum += exp2_neg((static_cast<double>(f[e]) - static_cast<double>(top)) * c64);
          } else {
            sum += static_cast<double>(weights<T>(s_vec[i - i0], top, c2));
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
            const float f = T::load1(s_raw, (v0 - i0) * E + e0 + lane);
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
        if (!ex && lane < kCluster) tell(in_cta(smem_of(&s_redo), lane), close ? 1u : 0u, in_cta(bar + 16, lane));
        if (lane == 0 && !close) a.token[static_cast<int64_t>(s) * (a.D + 1) + len] = found >= 0 ? found : last;
      }
    }
    if (!ex) {  // the owner's answer
      if (control) {
        if (lane == 0) expect(bar + 16, sizeof(s_redo));
        if (!heard(bar + 16, asked & 1) && lane == 0) s_redo = kLost;
      }
      ++asked;
      __syncthreads();
      if (s_redo == kLost) {
        lost = true;
        break;
      }
      if (s_redo) {
        exact = true;
        continue;
      }
    }
    bonus = -3;  // written by the owner
    break;
  }
  if (!joined) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  if (lost) {  // what is late may still come: nobody leaves before the others
    if (tid == 0) atomicOr(a.status, kStatusTimeout);
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    // no verdict, also where the first CTA has heard of all (it has then written its own and left)
    if (tid == 0) a.accept_len[s] = -1;
    return;
  }
  // What the walk did not fill.  (Else a CTA may leave: whatever the others sent it, it has waited for.)
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

template <typename T, int kResident>
cudaError_t verify_as(const VerifyArgs& a, cudaStream_t stream) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(static_cast<unsigned>(a.S) * kCluster);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = kStageBytes;
  cfg.stream = stream;
  cudaLaunchAttribute attr{};
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = kCluster;
  attr.val.clusterDim.y = 1;
  attr.val.clusterDim.z = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, verify_tree_kernel<T, kResident>, a);
}

template <typename T>
cudaError_t verify_as(const VerifyArgs& a, int sms, cudaStream_t stream) {
  // Two CTAs an SM may have 128 registers a thread: one tree of 32 000 ids took 13.2 us against 14.1 with
  // 64.  Where the sequences do not fit the device so, four, with 64 registers (80 bytes a thread spill): 128
  // trees of 128 256 ids took 84 us against 97 at three an SM, and 91 in clusters of four CTAs (all with the
  // cluster's barrier for the exchange).
  const bool few = static_cast<int64_t>(a.S) * kCluster <= 2ll * sms;
  return few ? verify_as<T, 2>(a, stream) : verify_as<T, 4>(a, stream);
}

}  // namespace

cudaError_t launch_verify_tree(const VerifyArgs& a, int sms, cudaStream_t stream, int64_t* launches) {
  ++*launches;
  if (a.dtype == GTO_BF16) return verify_as<Bf16>(a, sms, stream);
  if (a.dtype == GTO_F16) return verify_as<F16>(a, sms, stream);
  return verify_as<F32>(a, sms, stream);
}

}  // namespace gto
