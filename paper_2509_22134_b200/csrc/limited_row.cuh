// A row of logits of which top-k, top-p and min-p leave a part: what stays, and a token of it.
#pragma once

#include "decode_common.cuh"
#include "logit_weights.cuh"

namespace gto {

constexpr int kUnroll = 4;              // vectors of 16 bytes a thread takes in a step
constexpr int kBins = 128;              // of the slots' maxima, by their distance from the row's
constexpr int kWideBins = 2048;         // of the tokens, where more stays than a list holds

// How far a sum of fp32 weights can be from the true one, relative to the row's whole mass.  A weight 2^-a is off by
// 2^-22 (the exponential) and 3 * 2^-24 * (a + kReach) * ln 2 (roundings of its argument) relative to itself; the mean of a
// over the distribution is at most log2 V <= 19.6; a thread's 32 weights and those of 32 threads are added in fp32, in twelve
// levels (12 * 2^-24), the rest in fp64.  In all below 3.9e-6.  (The argument in two words halved that and took half as long again.)
constexpr float kReach = 4.f;
constexpr double kSlack = 4e-6;

// ---- shared memory of the CTAs of a cluster
__device__ __forceinline__ uint64_t far_u64(const void* p, int cta) {
  uint64_t v;
  asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(in_cta(smem_of(p), cta)) : "memory");
  return v;
}
__device__ __forceinline__ double far_f64(const double* p, int cta) { return __longlong_as_double(far_u64(p, cta)); }
__device__ __forceinline__ int far_i32(const int* p, int cta) {
  int v;
  asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(v) : "r"(in_cta(smem_of(p), cta)) : "memory");
  return v;
}
__device__ __forceinline__ void put_u64x2(uint32_t to, uint64_t a, uint64_t b) {
  asm volatile("st.shared::cluster.v2.b64 [%0], {%1, %2};" ::"r"(to), "l"(a), "l"(b) : "memory");
}

// Inclusive sums over the lanes.
template <typename N>
__device__ __forceinline__ N scan_warp(N v, int lane) {
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const N y = __shfl_up_sync(kFull, v, o);
    if (lane >= o) v += y;
  }
  return v;
}
template <typename N>
__device__ __forceinline__ N sum_warp(N v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(kFull, v, o);
  return v;
}

// The next bf16 at or above x, as its bits.
__device__ __forceinline__ uint16_t up16(float x) {
  const uint32_t u = __float_as_uint(x);
  return static_cast<uint16_t>((u >> 31 ? u : u + 0xffffu) >> 16);
}
__device__ __forceinline__ float from16(uint16_t b) { return __uint_as_float(static_cast<uint32_t>(b) << 16); }

struct Part {
  float sum, ref;  // weights of a warp's step, relative to ref
};
struct alignas(16) Mail {  // what a warp tells all others
  double a, b, c, d;
  float f, g;
  int n, m;
};
struct Found {
  double total, weight;
  int id;
  bool mine;   // this lane has it (the others do not know)
  bool close;  // the sums are not exact enough to tell
};
struct Cut {
  int n;            // tokens that stay
  double total;     // their mass
  uint64_t border;
  bool enough;      // the list holds all that stay
  bool close;       // the row's mass is not exact enough to tell
};

// kCluster CTAs of kThreads a row.  kServesAll: rows of which much stays are served too, by lists twice as long.
template <int kCluster, int kThreads, bool kServesAll>
struct Shared {
  static constexpr int kWarps = kThreads / 32;
  static constexpr int kSlots = kServesAll ? 16 : 8;      // maxima that a thread leaves, of one step or several
  static constexpr int kList = kServesAll ? 1024 : 512;   // tokens that a list holds
  static constexpr int kItems = 768 / kWarps;             // slots that a warp reads again
  static constexpr int kMaxSteps = static_cast<int>(kMaxTargetRow / 16 / (kThreads * kUnroll)) / kCluster;
  union {
    uint16_t top[kSlots][kThreads];
    uint32_t wide[kServesAll ? kWideBins : 1];
  };
  union {
    struct {
      uint64_t merged[kCluster > 1 ? kList : 1];
      double scan[kList];
    };
    struct {
      alignas(16) int wide_n[kServesAll ? kWideBins : 4];
      alignas(16) float wide_m[kServesAll ? kWideBins : 4];
    };
  };
  uint64_t list[kList];
  Part part[kMaxSteps][kWarps];
  double group[kMaxSteps];
  uint16_t items[kWarps][kItems];
  alignas(16) int bins[kBins];
  Mail mail[2][kCluster * kWarps];
  double red[2][kWarps];
  int red_n[2][kWarps];
  int n_list, bin, bin2, from, enough;
  float tau;
  double value, value2;
  Cut cut;
  double pow2[kServesAll ? 32 : 1];  // 2^(j/32)
};

// A CTA's share of a row: of the row's blocks of kThreads vectors every kCluster-th, so that tokens fall to threads
// by chance wherever the likely ones stand.
template <typename T, int kCluster, int kThreads, bool kServesAll>
struct Row {
  using Mem = Shared<kCluster, kThreads, kServesAll>;
  static constexpr int kWarps = Mem::kWarps;
  static constexpr int E = T::kPerVec;
  static constexpr int kSlots = Mem::kSlots, kList = Mem::kList, kMaxSteps = Mem::kMaxSteps, kItems = Mem::kItems;
  // tokens that a list is made for (where many rows share an SM, only so many that a thread sorts one each)
  static constexpr int kAim = kServesAll ? kList * 5 / 6 : 240;
  static constexpr int kEach = kList / kThreads;
  static constexpr int kMails = kCluster * kWarps;
  static constexpr int kMailRounds = (kMails + 31) / 32;
  Mem& sh;
  const char* z;
  int nvec, blocks, steps, per_slot, slots;
  int rank, tid, lane, warp;
  int turn, flip;  // of the double-buffered exchanges between CTAs / warps
  bool alone;      // the other CTAs of the cluster may not have begun yet
  float M;         // the row's largest logit
  double scale;    // to log2 units
  float c2;        // the same in fp32

  __device__ __forceinline__ Row(Mem& shared, int V, int r) : sh(shared) {
    rank = r;
    tid = threadIdx.x;
    lane = tid & 31;
    warp = tid >> 5;
    nvec = V / E;
    const int all = (nvec + kThreads - 1) / kThreads;
    blocks = (all - rank + kCluster - 1) / kCluster;
    // (the same number in every CTA)
    steps = ((all + kCluster - 1) / kCluster + kUnroll - 1) / kUnroll;
    per_slot = (steps + kSlots - 1) / kSlots;
    slots = (steps + per_slot - 1) / per_slot;
    turn = flip = 0;
    alone = false;
  }
  __device__ __forceinline__ void scale_to(double s) {
    scale = s;
    c2 = static_cast<float>(s);
  }
  __device__ __forceinline__ void cluster_sync() const {
    if (kCluster == 1) __syncthreads();
    else asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
  }
  // Another CTA's shared memory may be written once that CTA has begun.  Every thread says at its kernel's start that it has,
  // and waits for the others before its first exchange.
  static __device__ __forceinline__ void begun() {
    if (kCluster > 1) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  }
  static __device__ __forceinline__ void wait_for_others() {
    if (kCluster > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  }
  __device__ __forceinline__ void meet() {
    if (kCluster > 1 && alone) {
      wait_for_others();
      alone = false;
    }
  }
  // Vector that thread t of this CTA has in block q of its blocks; nvec or more: none.
  __device__ __forceinline__ int vec_of(int q, int t) const {
    return q < blocks ? (q * kCluster + rank) * kThreads + t : nvec;
  }
  __device__ __forceinline__ uint4 load(int v) const { return ld_stream16(z + static_cast<int64_t>(v) * 16); }
  __device__ __forceinline__ double raw(float x) const {
    return exp2_neg((static_cast<double>(x) - static_cast<double>(M)) * scale);
  }

  __device__ __forceinline__ void fill_table() {
    if (tid < 32) sh.pow2[tid] = 2.0 * exp2_neg(tid * (1.0 / 32) - 1.0);
  }
  // As raw(), for many tokens, and only where the weight is at least 2^-1000 (a number without meaning elsewhere): 2^x = 2^e 2^(j/32) 2^f
  // with |f| <= 1/64, whose polynomial of degree 5 (through the Chebyshev points of (2^f - 1) / f) is off by 1.4e-16.
  __device__ __forceinline__ double raw_near(float x) const {
    constexpr double kMagic = 211106232532992.0;  // 1.5 * 2^47: 32 x in the low bits
    const double d = static_cast<double>(x) - static_cast<double>(M);
    const double t = fma(d, scale, kMagic);
    const double f = fma(d, scale, -(t - kMagic));
    double y = 0.0013333604694153824;
    y = fma(y, f, 0.009618176115571158);
    y = fma(y, f, 0.05550410866453748);
    y = fma(y, f, 0.24022650695623157);
    y = fma(y, f, 0.6931471805599453);
    y = fma(y, f, 1.0);
    const int k = __double2loint(t);
    y *= sh.pow2[k & 31];
    return __hiloint2double(__double2hiint(y) + ((k >> 5) << 20), __double2loint(y));
  }
  // The value from which on it serves.  (Rounded up: of cold rows of fp32 a step of the logits is hundreds of halvings, and a value
  // half a step lower would take exponents below the least one.)
  __device__ __forceinline__ float near_from() const {
    return fmaxf(__double2float_ru(static_cast<double>(M) - 999.0 / scale), -3.4028235e38f);
  }

  __device__ __forceinline__ double raw_any(float x, float from) const { return x >= from ? raw_near(x) : 0.0; }

  // f(vector, its number) over the thread's vectors; the next three are on their way meanwhile.
  template <typename F>
  __device__ __forceinline__ void vectors(F f) const {
    ahead([&](int i) { return vec_of(i, tid); }, blocks, f);
  }
  template <typename N, typename F>
  __device__ __forceinline__ void ahead(N number, int n, F f) const {
    const auto get = [&](int i) {
      const int at = i < n ? number(i) : nvec;
      return at < nvec ? __ldg(reinterpret_cast<const uint4*>(z) + at) : uint4{};
    };
    uint4 v0 = get(0), v1 = get(1), v2 = get(2);
#pragma unroll 1
    for (int i = 0; i < n; ++i) {
      const uint4 v = v0;
      v0 = v1;
      v1 = v2;
      v2 = get(i + 3);
      const int at = number(i);
      if (at < nvec) f(v, at);
    }
  }
  // f(value, id) over the thread's tokens.
  template <typename F>
  __device__ __forceinline__ void each(F f) const {
    vectors([&](const uint4& v, int at) {
      float x[E];
      T::unpack(v, x);
#pragma unroll
      for (int e = 0; e < E; ++e) f(x[e], at * E + e);
    });
  }

  // ---- between the warps of a CTA
  __device__ __forceinline__ int sum_cta(int v) {
    v = __reduce_add_sync(kFull, v);
    if (lane == 0) sh.red_n[flip][warp] = v;
    __syncthreads();
    int s = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) s += sh.red_n[flip][w];
    flip ^= 1;
    return s;
  }
  // Sum over the threads before this one; *all: over all.
  __device__ __forceinline__ double before_cta(double v, double* all) {
    const double upto = scan_warp(v, lane);
    if (lane == 31) sh.red[flip][warp] = upto;
    __syncthreads();
    double s = 0.0, b = 0.0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      if (w == warp) b = s;
      s += sh.red[flip][w];
    }
    flip ^= 1;
    *all = s;
    return b + (upto - v);
  }

  // ---- between all warps of the cluster: each posts, and after the barrier reads what all have posted, in the order of
  // CTAs and warps (so that all compute the same)
  __device__ __forceinline__ const Mail* post(const Mail& mine) {
    Mail* box = &sh.mail[turn][rank * kWarps + warp];
    if (kCluster == 1) {
      if (lane == 0) *box = mine;
    } else if (lane < kCluster) {
      const uint32_t to = in_cta(smem_of(box), lane);
      put_u64x2(to, __double_as_longlong(mine.a), __double_as_longlong(mine.b));
      put_u64x2(to + 16, __double_as_longlong(mine.c), __double_as_longlong(mine.d));
      put_u64x2(to + 32, static_cast<uint64_t>(__float_as_uint(mine.g)) << 32 | __float_as_uint(mine.f),
                static_cast<uint64_t>(static_cast<uint32_t>(mine.m)) << 32 | static_cast<uint32_t>(mine.n));
    }
    cluster_sync();
    const Mail* all = sh.mail[turn];
    turn ^= 1;  // (a box is filled again behind the barrier of the next post)
    return all;
  }
  // Sums over the row.
  __device__ __forceinline__ Mail reduce(double a, double b, int n, int m) {
    Mail s{sum_warp(a), sum_warp(b), 0.0, 0.0, 0.f, 0.f, __reduce_add_sync(kFull, n), __reduce_add_sync(kFull, m)};
    const Mail* all = post(s);
    s = Mail{};
#pragma unroll
    for (int r = 0; r < kMailRounds; ++r) {
      const int i = r * 32 + lane;
      if (i < kMails) {
        s.a += all[i].a;
        s.b += all[i].b;
        s.n += all[i].n;
        s.m += all[i].m;
      }
    }
    s.a = sum_warp(s.a);
    s.b = sum_warp(s.b);
    s.n = __reduce_add_sync(kFull, s.n);
    s.m = __reduce_add_sync(kFull, s.m);
    return s;
  }
  // The least of n and the largest of m over the row.
  __device__ __forceinline__ void least_most(uint32_t* n, uint32_t* m) {
    Mail s{};
    s.n = static_cast<int>(__reduce_min_sync(kFull, *n));
    s.m = static_cast<int>(__reduce_max_sync(kFull, *m));
    const Mail* all = post(s);
    uint32_t lo = 0xffffffffu, hi = 0;
#pragma unroll
    for (int r = 0; r < kMailRounds; ++r) {
      const int i = r * 32 + lane;
      if (i < kMails) {
        lo = min(lo, static_cast<uint32_t>(all[i].n));
        hi = max(hi, static_cast<uint32_t>(all[i].m));
      }
    }
    *n = __reduce_min_sync(kFull, lo);
    *m = __reduce_max_sync(kFull, hi);
  }

  // ---- the row in one pass.  Returns whether it holds a NaN; sets M, and *mass where the weights are summed.
  // masked: whether to look for -inf; then whether there is one.
  template <bool kSum>
  __device__ __forceinline__ bool stream(double* mass, bool* masked) {
    const float reach = kReach / c2;
    float ref = -INFINITY, most = -INFINITY, slot_top = -INFINITY;
    bool bad = false, low = false;
    int slot = 0, in_slot = 0;
    // (what the next steps count in, behind the barrier below)
    if (tid < kBins) sh.bins[tid] = 0;
    if (tid == 0) sh.n_list = 0;
#pragma unroll 1
    for (int step = 0; step < steps; ++step) {
      uint4 v[kUnroll];
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        const int at = vec_of(step * kUnroll + u, tid);
        v[u] = make_uint4(T::kNegInfWord, T::kNegInfWord, T::kNegInfWord, T::kNegInfWord);
        if (at < nvec) v[u] = load(at);
      }
      uint32_t word = max_of<T>(v[0]);
#pragma unroll
      for (int u = 1; u < kUnroll; ++u) word = max_word<T>(word, max_of<T>(v[u]));
      const float top = max_half<T>(word);
      bad |= top != top;
      if (*masked) {
        uint32_t least = min_of<T>(v[0]);
#pragma unroll
        for (int u = 1; u < kUnroll; ++u)
          if (vec_of(step * kUnroll + u, tid) < nvec) least = min_word<T>(least, min_of<T>(v[u]));
        low |= vec_of(step * kUnroll, tid) < nvec && min_half<T>(least) == -INFINITY;
      }
      slot_top = fmaxf(slot_top, top);
      if (++in_slot == per_slot || step == steps - 1) {
        sh.top[slot++][tid] = up16(slot_top);
        most = fmaxf(most, slot_top);
        slot_top = -INFINITY;
        in_slot = 0;
      }
      if (kSum) {
        if (__any_sync(kFull, ref == -INFINITY ? top > ref : top > ref + reach)) ref = fmaxf(ref, warp_max_f32(top));
        float s = 0.f;
        if (ref != -INFINITY) {
#pragma unroll
          for (int u = 0; u < kUnroll; ++u) s += weights<T>(v[u], ref, c2);
        }
        s = warp_sum_f32(s);
        if (lane == 0) sh.part[step][warp] = Part{s, ref};
      }
    }
    // (a reference never falls: the warp's last one is its largest)
    double sum = 0.0;
    if (kSum && ref > -INFINITY && ref < INFINITY) {
      __syncwarp();
      for (int i = lane; i < steps; i += 32) {
        const Part p = sh.part[i][warp];
        if (p.ref != -INFINITY) sum += static_cast<double>(p.sum) * exp2_neg((static_cast<double>(p.ref) - static_cast<double>(ref)) * scale);
      }
    }
    if (kSum) sum = sum_warp(sum);
    Mail s{};
    s.a = sum;
    s.f = ref;
    s.g = warp_max_f32(most);
    s.n = __any_sync(kFull, bad);
    s.m = __any_sync(kFull, low);
    meet();  // (the first exchange of every kernel; behind the loads)
    const Mail* all = post(s);
    float top = -INFINITY;
    bad = low = false;
#pragma unroll
    for (int r = 0; r < kMailRounds; ++r) {
      const int i = r * 32 + lane;
      if (i < kMails) {
        top = fmaxf(top, all[i].g);
        bad |= all[i].n != 0;
        low |= all[i].m != 0;
      }
    }
    M = warp_max_f32(top);
    *masked = __any_sync(kFull, low);
    if (kSum) {
      double total = 0.0;
#pragma unroll
      for (int r = 0; r < kMailRounds; ++r) {
        const int i = r * 32 + lane;
        if (i < kMails && all[i].f > -INFINITY)
          total += all[i].a * exp2_neg((static_cast<double>(all[i].f) - static_cast<double>(M)) * scale);
      }
      *mass = sum_warp(total);
    }
    return __any_sync(kFull, bad);
  }

  // Tokens of the warp's slots that reach tau: f(value, id) for those at or above it.  False if there are too many slots.
  template <typename F>
  __device__ __forceinline__ bool visit(float tau, F f) {
    const int each_item = per_slot * kUnroll;
    int n = 0;
    for (int s = 0; s < slots; ++s) {
      const bool hit = from16(sh.top[s][tid]) >= tau;
      const unsigned all = __ballot_sync(kFull, hit);
      const int at = n + __popc(all & ((1u << lane) - 1));
      if (hit && at < kItems) sh.items[warp][at] = static_cast<uint16_t>(s << 8 | tid);
      n += __popc(all);
    }
    if (n > kItems) return false;
    __syncwarp();
    constexpr int kAtOnce = 4;
    for (int i0 = lane; i0 < n * each_item; i0 += 32 * kAtOnce) {
      uint4 v[kAtOnce];
      int at[kAtOnce];
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u) {
        const int i = i0 + 32 * u;
        at[u] = nvec;
        if (i < n * each_item) {
          const int item = sh.items[warp][i / each_item];
          at[u] = vec_of((item >> 8) * each_item + i % each_item, item & 255);
        }
        if (at[u] < nvec) v[u] = load(at[u]);
      }
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u) {
        if (at[u] >= nvec || !(max_half<T>(max_of<T>(v[u])) >= tau)) continue;
        float x[E];
        T::unpack(v[u], x);
#pragma unroll
        for (int e = 0; e < E; ++e)
          if (x[e] >= tau) f(x[e], at[u] * E + e);
      }
    }
    __syncwarp();
    return true;
  }

  // The lowest id with the row's largest logit.
  __device__ __forceinline__ int best() {
    uint32_t id = 0xffffffffu, unused = 0;
    if (!visit(M, [&](float x, int i) { id = min(id, static_cast<uint32_t>(i)); })) {
      each([&](float x, int i) {
        if (x == M) id = min(id, static_cast<uint32_t>(i));
      });
    }
    least_most(&id, &unused);
    return static_cast<int>(id);
  }

  // A value that all that stays should lie above, by the slots' maxima (and with top-p a tenth of what it leaves out, since
  // the slots tell masses to a few per cent).  False where too much stays, or the slots cannot tell.
  __device__ __forceinline__ bool aim_at(int top_k, float top_p, double mass, float floor, float* tau) {
    const float unit = fminf(static_cast<float>(scale), 1e30f);
    for (int s = 0; s < slots; ++s) {
      const float top = from16(sh.top[s][tid]);
      if (top == -INFINITY) continue;
      const float x = fmaxf((M - top) * unit, 0.f);  // up to 8: bins of 1/8; from there up to 40 of 1/2
      const int b = x < 8.f ? static_cast<int>(x * 8.f) : x < 40.f ? 64 + static_cast<int>((x - 8.f) * 2.f) : kBins;
      if (b < kBins) atomicAdd(&sh.bins[b], 1);
    }
    cluster_sync();
    if (warp == 0) {
      constexpr int kOf = kBins / 32;
      const auto reaches = [](int b) { return b < 64 ? static_cast<float>(b) * (1.f / 8) : 8.f + static_cast<float>(b - 64) * (1.f / 2); };
      const float buckets = static_cast<float>(nvec) / static_cast<float>(kUnroll * per_slot), bucket = 1.f / buckets;
      const auto tokens = [&](int j) { return -buckets * __logf(1.f - fminf(static_cast<float>(j) * bucket, 0.995f)); };
      // slots, then tokens, then mass, up to each bin
      int n[kOf] = {0, 0, 0, 0};
#pragma unroll
      for (int d = 0; d < kCluster; ++d) {
        if (kCluster == 1) {
          const int4 q = *reinterpret_cast<const int4*>(sh.bins + lane * kOf);
          n[0] = q.x, n[1] = q.y, n[2] = q.z, n[3] = q.w;
        } else {
          const uint64_t q0 = far_u64(&sh.bins[lane * kOf], d), q1 = far_u64(&sh.bins[lane * kOf + 2], d);
          n[0] += static_cast<int>(q0), n[1] += static_cast<int>(q0 >> 32), n[2] += static_cast<int>(q1), n[3] += static_cast<int>(q1 >> 32);
        }
      }
      int j = n[0] + n[1] + n[2] + n[3];
      j = scan_warp(j, lane) - j;
      float t[kOf], m[kOf], before = tokens(j), sum = 0.f;
      bool k_enough[kOf];
#pragma unroll
      for (int i = 0; i < kOf; ++i) {
        const int b = lane * kOf + i;
        j += n[i];
        k_enough[i] = j >= top_k;
        t[i] = tokens(j);
        sum += (t[i] - before) * ex2_approx(-0.5f * (reaches(b) + reaches(b + 1)));
        m[i] = sum;
        before = t[i];
      }
      const float m0 = scan_warp(sum, lane) - sum;
      // the first bin that is enough for one of the limits
      const bool k = top_k > 0, p = top_p < 1.f && !k;
      const float goal = p ? static_cast<float>(mass * (top_p + 0.1 * (1.0 - top_p))) : 0.f;
      // (with top-p over top-k's tokens all of those are needed)
      const float x_floor = floor > 0.f && !(k && top_p < 1.f) ? -__log2f(floor) * 1.001f + 1e-3f : INFINITY;
      int found = kBins;
      float expect = 0.f;
#pragma unroll
      for (int i = kOf - 1; i >= 0; --i) {
        const int b = lane * kOf + i;
        if ((k && k_enough[i]) || (p && m0 + m[i] >= goal) || reaches(b + 1) >= x_floor) {
          found = b;
          expect = t[i];
        }
      }
      const unsigned any = __ballot_sync(kFull, found < kBins);
      const int l = any ? __ffs(any) - 1 : 0;
      found = __shfl_sync(kFull, found, l);
      expect = __shfl_sync(kFull, expect, l);
      if (lane == 0) {
        // (slots' maxima of finer types were rounded up, by 2^-7 of themselves at most)
        const float round = T::kNegInfElem == 0xff80u ? 1e-6f : 0x1p-7f;
        const float at = M - reaches(found + 1) / unit;
        sh.tau = at - round * fmaxf(fabsf(M), fabsf(at));
        sh.enough = found < kBins && expect <= static_cast<float>(kAim);
      }
    }
    __syncthreads();
    *tau = sh.tau;
    return sh.enough;
  }

  // All tokens at or above tau, in all CTAs.  Their number; above kList: too many.
  __device__ __forceinline__ int gather(float tau) {
    const bool ok = visit(tau, [&](float x, int id) {
      if (x == -INFINITY) return;
      const int at = atomicAdd(&sh.n_list, 1);
      if (at < kList) sh.list[at] = make_key(x, id);
    });
    if (!ok && lane == 0) atomicAdd(&sh.n_list, kList + 1);
    cluster_sync();
    return join();
  }
  // Joins the CTAs' lists, which a barrier has made known.
  __device__ __forceinline__ int join() {
    if (kCluster == 1) return sh.n_list;
    int total = 0, from[kCluster + 1];
#pragma unroll
    for (int d = 0; d < kCluster; ++d) {
      from[d] = total;
      total += min(far_i32(&sh.n_list, d), kList + 1);
    }
    from[kCluster] = total;
    if (total <= kList) {
      for (int i = tid; i < total; i += kThreads) {
        int of = 0;
#pragma unroll
        for (int d = 1; d < kCluster; ++d) of += i >= from[d];
        int first = 0;
#pragma unroll
        for (int d = 1; d < kCluster; ++d)
          if (d == of) first = from[d];
        sh.merged[i] = far_u64(&sh.list[i - first], of);
      }
    }
    __syncthreads();
    return total;
  }
  __device__ __forceinline__ uint64_t* tokens() { return kCluster == 1 ? sh.list : sh.merged; }

  // Distinct keys, descending.
  __device__ __forceinline__ void sort(uint64_t* a, int n) {
    if (n <= kThreads) {  // every key counts those before it
      const uint64_t mine = tid < n ? a[tid] : 0;
      int at = 0;
      if (warp * 32 < n) {
#pragma unroll 4
        for (int j = 0; j < n; ++j) at += a[j] > mine;
      }
      __syncthreads();
      if (tid < n) a[at] = mine;
      __syncthreads();
      return;
    }
    int size = kThreads;
    while (size < n) size *= 2;
    for (int i = n + tid; i < size; i += kThreads) a[i] = 0;
    for (int k = 2; k <= size; k *= 2)
      for (int j = k / 2; j > 0; j /= 2) {
        __syncthreads();
        for (int p = tid; p < size / 2; p += kThreads) {
          const int i = 2 * p - (p & (j - 1));
          const uint64_t x = a[i], y = a[i + j];
          if ((x < y) == ((i & k) == 0)) {
            a[i] = y;
            a[i + j] = x;
          }
        }
      }
    __syncthreads();
  }

  // What stays of a list of n tokens that all lie at or above tau (sorts it; the weights go into sh.scan).  mass: the whole
  // row's, to `slack`.
  __device__ __forceinline__ Cut cut(int n, int top_k, float top_p, double mass, double slack, float floor, float tau) {
    const bool k = top_k > 0, p = top_p < 1.f, m = floor > 0.f;
    const int stay_k = k ? min(top_k, n) : n;
    const double least = static_cast<double>(floor), share = static_cast<double>(top_p);
    uint64_t* list = tokens();
    // From the numbers of tokens whose sums are below the goal (and below it less / more the slack), or which are heavy enough.
    const auto decide = [&](int below, int lo, int hi, int heavy, Cut* out) {
      bool bounded = k && top_k <= n;  // (then no token below the list stays)
      int stay = stay_k;
      out->close = p && lo != hi;
      if (p && below < n) {
        stay = min(stay, below + 1);
        bounded = bounded || !k;
      }
      if (m) {
        stay = min(stay, max(heavy, 1));
        if (heavy < n || raw(tau) < least) bounded = true;
      }
      // (top-p of what top-k leaves needs all of that)
      out->enough = bounded && !(k && p && top_k > n);
      out->n = stay;
    };
    if (n <= 64) {  // one warp's work
      if (warp == 0) {
        uint64_t key[2] = {lane < n ? list[lane] : 0, 32 + lane < n ? list[32 + lane] : 0};
        int at[2] = {0, 0};
        for (int j = 0; j < n; ++j) {
          const uint64_t y = list[j];
          at[0] += y > key[0];
          at[1] += y > key[1];
        }
        __syncwarp();
        if (lane < n) list[at[0]] = key[0];
        if (32 + lane < n) list[at[1]] = key[1];
        __syncwarp();
        key[0] = lane < n ? list[lane] : 0;
        key[1] = 32 + lane < n ? list[32 + lane] : 0;
        const double w0 = lane < n ? raw(key_value(key[0])) : 0.0, w1 = 32 + lane < n ? raw(key_value(key[1])) : 0.0;
        sh.scan[lane] = w0;
        sh.scan[32 + lane] = w1;
        const double s0 = scan_warp(w0, lane), s1 = __shfl_sync(kFull, s0, 31) + scan_warp(w1, lane);
        const auto sum_to = [&](int i) { return __shfl_sync(kFull, i < 32 ? s0 : s1, i & 31); };
        const double goal = share * (k ? sum_to(stay_k - 1) : mass), off = k ? 0.0 : share * slack;
        const auto count = [&](bool a, bool b) {
          return __popc(__ballot_sync(kFull, lane < n && a)) + __popc(__ballot_sync(kFull, 32 + lane < n && b));
        };
        Cut c;
        decide(count(s0 < goal, s1 < goal), count(s0 < goal - off, s1 < goal - off), count(s0 < goal + off, s1 < goal + off),
               count(w0 >= least, w1 >= least), &c);
        c.total = sum_to(c.n - 1);
        const uint64_t key_n = c.n - 1 < 32 ? key[0] : key[1];
        c.border = __shfl_sync(kFull, key_n, (c.n - 1) & 31);
        if (lane == 0) sh.cut = c;
      }
      __syncthreads();
      return sh.cut;
    }
    sort(list, n);
    const int each_thread = (n + kThreads - 1) / kThreads;
    double w[kEach], mine = 0.0;
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      const int i = tid * each_thread + e;
      w[e] = e < each_thread && i < n ? raw(key_value(list[i])) : 0.0;
      mine += w[e];
    }
    double all;
    const double before = before_cta(mine, &all);
    double acc = before;
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      const int i = tid * each_thread + e;
      acc += w[e];
      if (e < each_thread && i < n) {
        sh.scan[i] = w[e];
        if (i == stay_k - 1) sh.value = acc;
      }
    }
    __syncthreads();
    const double goal = share * (k ? sh.value : mass), off = k ? 0.0 : share * slack;
    int below = 0, below_lo = 0, below_hi = 0, heavy = 0;
    acc = before;
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      acc += w[e];
      if (e >= each_thread || tid * each_thread + e >= n) continue;
      below += acc < goal;
      below_lo += acc < goal - off;
      below_hi += acc < goal + off;
      heavy += w[e] >= least;
    }
    below = sum_cta(below | below_lo << 16);
    heavy = sum_cta(heavy | below_hi << 16);
    Cut c;
    decide(below & 0xffff, below >> 16, heavy >> 16, heavy & 0xffff, &c);
    acc = before;
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      acc += w[e];
      if (e < each_thread && tid * each_thread + e == c.n - 1) {
        sh.value2 = acc;
        sh.cut.border = list[c.n - 1];
      }
    }
    __syncthreads();
    c.total = sh.value2;
    c.border = sh.cut.border;
    return c;
  }

  // Puts the first n of the sorted list into the order of their ids, each with its place in the list (low word).
  __device__ __forceinline__ void by_id(int n) {
    uint64_t* list = tokens();
    uint64_t mine[kEach];
    __syncthreads();
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      const int i = tid + e * kThreads;
      mine[e] = i < n ? list[i] << 32 | static_cast<uint32_t>(i) : 0;
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < kEach; ++e)
      if (tid + e * kThreads < n) list[tid + e * kThreads] = mine[e];
    __syncthreads();
    sort(list, n);
  }
  // The token of the first n of the sorted list, some ids taken out; u in [0, 1).  Found in thread 0 of the first CTA.
  template <typename F>
  __device__ __forceinline__ Found draw_listed(int n, double u, F out) {
    Found f{0.0, 0.0, -1, rank == 0 && tid == 0, false};
    uint64_t* list = tokens();
    if (n <= 64) {  // one warp's work: for every token the mass of those up to its id
      if (warp != 0) return f;
      int id[2], last = -1;
      double w[2], upto[2] = {0.0, 0.0}, all = 0.0;
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const int i = r * 32 + lane;
        id[r] = i < n ? key_id(list[i]) : 0x7fffffff;
        w[r] = i < n && !out(id[r]) ? sh.scan[i] : 0.0;
      }
      for (int j = 0; j < n; ++j) {
        const int at = __shfl_sync(kFull, j < 32 ? id[0] : id[1], j & 31);
        const double y = __shfl_sync(kFull, j < 32 ? w[0] : w[1], j & 31);
        all += y;
#pragma unroll
        for (int r = 0; r < 2; ++r) upto[r] += at <= id[r] ? y : 0.0;
      }
      const double aim = u * all;
      int first = 0x7fffffff;
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        if (w[r] > 0.0 && upto[r] > aim) first = min(first, id[r]);
        if (w[r] > 0.0) last = max(last, id[r]);
      }
      first = __reduce_min_sync(kFull, first);
      last = __reduce_max_sync(kFull, last);
      f.id = first != 0x7fffffff ? first : last;  // (rounding: the last one that holds something)
      f.total = all;
      const unsigned has[2] = {__ballot_sync(kFull, w[0] > 0.0 && id[0] == f.id), __ballot_sync(kFull, w[1] > 0.0 && id[1] == f.id)};
      if (f.id >= 0) f.weight = __shfl_sync(kFull, has[0] ? w[0] : w[1], __ffs(has[0] ? has[0] : has[1]) - 1);
      return f;
    }
    if (tid == 0) sh.from = 0x7fffffff;
    by_id(n);
    const int each_thread = (n + kThreads - 1) / kThreads;
    double w[kEach], sum = 0.0;
    int last = -1;
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      const int i = tid * each_thread + e;
      w[e] = 0.0;
      if (e < each_thread && i < n) {
        const int id = static_cast<int>(0xffffffffu - static_cast<uint32_t>(list[i] >> 32));
        if (!out(id)) w[e] = sh.scan[static_cast<uint32_t>(list[i])];
        if (w[e] > 0.0) last = i;
      }
      sum += w[e];
    }
    double all;
    const double before = before_cta(sum, &all);
    const double aim = u * all;
    double acc = before;
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      acc += w[e];
      if (e < each_thread && w[e] > 0.0 && acc > aim) {
        atomicMin(&sh.from, tid * each_thread + e);
        break;
      }
    }
    last = __reduce_max_sync(kFull, last);
    if (lane == 0) sh.red_n[flip][warp] = last;
    __syncthreads();
    int at = sh.from;
    if (at == 0x7fffffff) {  // (rounding) the last one that holds something
      at = -1;
      for (int v = 0; v < kWarps; ++v) at = max(at, sh.red_n[flip][v]);
    }
    flip ^= 1;
    f.total = all;
    if (at >= 0) {
      f.id = static_cast<int>(0xffffffffu - static_cast<uint32_t>(list[at] >> 32));
      f.weight = sh.scan[static_cast<uint32_t>(list[at])];
    }
    return f;
  }

  // The entry of kMails (in the order of CTAs and warps) that holds aim: the last one with a mass that begins at or below
  // it, among several rows of entries one after the other.  mass(row, i); returns row * kMails + i, or -1; *begin: where it begins.
  template <int kRows, typename F>
  __device__ __forceinline__ int holder(double at, double aim, F mass, double* begin) {
    int found = -1;
#pragma unroll
    for (int q = 0; q < kRows; ++q)
#pragma unroll
      for (int r = 0; r < kMailRounds; ++r) {
        const int i = r * 32 + lane;
        const double x = i < kMails ? mass(q, i) : 0.0;
        const double upto = scan_warp(x, lane);
        unsigned is = __ballot_sync(kFull, x > 0.0 && at + (upto - x) <= aim);
        if (!is && found < 0) is = __ballot_sync(kFull, x > 0.0) & -__ballot_sync(kFull, x > 0.0);  // (the first that holds something)
        if (is) {
          const int l = 31 - __clz(is);
          found = q * kMails + r * 32 + l;
          *begin = at + __shfl_sync(kFull, upto - x, l);
        }
        at += __shfl_sync(kFull, upto, 31);
      }
    return found;
  }

  // The token of a row of which all stays, by the warps' sums: the step that holds it is read again.  taken(lo, hi): mass that is
  // taken out of ids lo .. hi-1, out(id): whether one is.  Found in one lane of the cluster, in thread 0 of the first CTA where
  // the sums cannot tell where it is.
  template <typename G, typename F>
  __device__ __forceinline__ Found draw_all(double u, double whole, G taken, F out) {
    const double slack = 2.0 * kSlack * whole;
    // mass of every step
    const auto mass_of = [&](int s) {
      double m = 0.0;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        const Part p = sh.part[s][w];
        if (p.ref != -INFINITY) m += static_cast<double>(p.sum) * exp2_neg((static_cast<double>(p.ref) - static_cast<double>(M)) * scale);
      }
      return m;
    };
    if (kCluster > 1) {
      for (int s = tid; s < steps; s += kThreads) sh.group[s] = mass_of(s);
      cluster_sync();
    }
    constexpr int kSpan = kThreads * kUnroll * kCluster * E;  // ids of a step
    double total = 0.0;
    constexpr int kRounds = (kMaxSteps + 31) / 32;  // (the same in all warps)
    double m[kRounds];
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
      const int s = r * 32 + lane;
      m[r] = 0.0;
      if (s < steps) {
        if (kCluster == 1) {
          m[r] = mass_of(s);
        } else {
#pragma unroll
          for (int d = 0; d < kCluster; ++d) m[r] += far_f64(&sh.group[s], d);
        }
        m[r] = fmax(m[r] - taken(s * kSpan, s * kSpan + kSpan), 0.0);
      }
      total += sum_warp(m[r]);
    }
    const double aim = u * total;
    // the last step that holds something and begins at or below aim
    int step = -1;
    double at = 0.0, base = 0.0;
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
      const double upto = scan_warp(m[r], lane);
      const unsigned is = __ballot_sync(kFull, m[r] > 0.0 && base + (upto - m[r]) <= aim);
      if (is) {
        const int l = 31 - __clz(is);
        step = r * 32 + l;
        at = base + __shfl_sync(kFull, upto - m[r], l);
      }
      base += __shfl_sync(kFull, upto, 31);
    }
    Found f{total, 0.0, -1, false, true};
    // its vectors: id order is (u, CTA, thread)
    uint4 v[kUnroll];
    double w[kUnroll], upto[kUnroll];
#pragma unroll
    for (int q = 0; q < kUnroll; ++q) {
      const int i = step < 0 ? nvec : vec_of(step * kUnroll + q, tid);
      w[q] = 0.0;
      if (i < nvec) v[q] = load(i);
    }
#pragma unroll
    for (int q = 0; q < kUnroll; ++q) {
      const int i = step < 0 ? nvec : vec_of(step * kUnroll + q, tid);
      if (i < nvec) {
        const double gone = taken(i * E, i * E + E);
        if (gone > 0.0) {  // summed without what is taken out
          float x[E];
          T::unpack(v[q], x);
#pragma unroll
          for (int e = 0; e < E; ++e)
            if (!out(i * E + e)) w[q] += static_cast<double>(ex2_approx((x[e] - M) * c2));
        } else {
          w[q] = static_cast<double>(weights<T>(v[q], M, c2));
        }
      }
      upto[q] = scan_warp(w[q], lane);
    }
    Mail s{};
    s.a = __shfl_sync(kFull, upto[0], 31);
    s.b = __shfl_sync(kFull, upto[1], 31);
    s.c = __shfl_sync(kFull, upto[2], 31);
    s.d = __shfl_sync(kFull, upto[3], 31);
    const Mail* all = post(s);
    double begin = 0.0;
    const int held = holder<kUnroll>(at, aim, [&](int q, int i) { return q == 0 ? all[i].a : q == 1 ? all[i].b : q == 2 ? all[i].c : all[i].d; },
                                     &begin);
    if (held < 0) {
      f.mine = rank == 0 && tid == 0;
      return f;
    }
    if (held % kMails != rank * kWarps + warp) return f;
    const int block = held / kMails;
    double mw = w[0], start = begin + (upto[0] - w[0]);
    uint4 mv = v[0];
#pragma unroll
    for (int q = 1; q < kUnroll; ++q)
      if (q == block) {
        mw = w[q];
        start = begin + (upto[q] - w[q]);
        mv = v[q];
      }
    const unsigned is = __ballot_sync(kFull, mw > 0.0 && start <= aim);
    // (rounding: it is too close then anyway)
    if (lane != (is ? 31 - __clz(is) : 0)) return f;
    f.mine = true;
    const int i = vec_of(step * kUnroll + block, tid);
    if (i >= nvec) return f;
    float x[E];
    T::unpack(mv, x);
    double acc = start;
    float found = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int id = i * E + e;
      const double y = out(id) ? 0.0 : static_cast<double>(ex2_approx((x[e] - M) * c2));
      if (f.id < 0 && y > 0.0 && acc + y > aim) {
        f.id = id;
        found = x[e];
        f.close = aim - acc < slack || acc + y - aim < slack;
      }
      acc += y;
    }
    f.weight = raw(found);
    return f;
  }

  // ---- ranges: a warp's share of the row's ids, one after the other.  (Its lanes stand side by side: with a run of ids for every
  // thread the pass in fp64 over a row of 128 256 took 10.9 us in place of 7.4.)
  __device__ __forceinline__ void range_of(int w, int* lo, int* hi) const {  // in vectors
    const int per = (nvec + kCluster - 1) / kCluster;
    const int vec0 = min(rank * per, nvec), vecs = min(vec0 + per, nvec) - vec0;
    const int range = (vecs + kWarps - 1) / kWarps;
    *lo = vec0 + min(w * range, vecs);
    *hi = min(*lo + range, vec0 + vecs);
  }
  // f(vector, its number) over the thread's part of its warp's range.
  template <typename F>
  __device__ __forceinline__ void along(F f) const {
    int lo, hi;
    range_of(warp, &lo, &hi);
    ahead([&](int i) { return lo + lane + 32 * i; }, (hi - lo - lane + 31) / 32, f);
  }
  // fp64 weights of the tokens of a vector; from: near_from().
  __device__ __forceinline__ void raw_of(const uint4& v, float from, float (&x)[E], double (&w)[E]) const {
    T::unpack(v, x);
#pragma unroll
    for (int e = 0; e < E; ++e) w[e] = raw_near(x[e]);
#pragma unroll
    for (int e = 0; e < E; ++e) w[e] = x[e] >= from ? w[e] : 0.0;
  }
  static __device__ __forceinline__ double sum_of(const double (&w)[E]) {
    if (E == 4) return (w[0] + w[1]) + (w[2] + w[3]);
    return ((w[0] + w[1]) + (w[2] + w[3])) + ((w[E - 4] + w[E - 3]) + (w[E - 2] + w[E - 1]));
  }
  // The row's mass in fp64.
  __device__ __forceinline__ double whole() {
    double m = 0.0;
    const float from = near_from();
    vectors([&](const uint4& v, int) {
      float x[E];
      double w[E];
      raw_of(v, from, x, w);
      m += sum_of(w);
    });
    return reduce(m, 0.0, 0, 0).a;
  }
  // Of the mass of every warp's range (sum over the lanes of `mine`): the first id at which the cumulative sum of
  // weight(value, id) passes u * (the whole sum), or `aim` where u < 0; the range that holds it is read again.  Found in one
  // thread of the cluster; id -1 where nothing has a weight.
  template <typename F>
  __device__ __forceinline__ Found pick(double mine, F weight, double u, double aim) {
    Mail s{};
    s.a = sum_warp(mine);
    const Mail* all = post(s);
    double total = 0.0;
#pragma unroll
    for (int r = 0; r < kMailRounds; ++r) total += r * 32 + lane < kMails ? all[r * 32 + lane].a : 0.0;
    total = sum_warp(total);
    if (u >= 0.0) aim = u * total;
    Found f{total, 0.0, -1, false, false};
    double begin = 0.0;
    const int held = holder<1>(0.0, aim, [&](int, int i) { return all[i].a; }, &begin);
    if (held < 0) {
      f.mine = rank == 0 && tid == 0;
      return f;
    }
    if (held / kWarps != rank) return f;
    // the CTA's threads have runs of that range
    int lo, hi;
    range_of(held % kWarps, &lo, &hi);
    const int run = (hi - lo + kThreads - 1) / kThreads, v0 = min(lo + tid * run, hi), v1 = min(v0 + run, hi);
    double of_run = 0.0, unused;
    for (int id = v0 * E; id < v1 * E; ++id) of_run += weight(T::load1(z, id), id);
    if (tid == 0) sh.from = -1;
    const double start = begin + before_cta(of_run, &unused);
    if (of_run > 0.0 && start <= aim) atomicMax(&sh.from, tid);
    __syncthreads();
    const bool none = sh.from < 0;  // (rounding: then the first that holds something)
    __syncthreads();
    if (none && of_run > 0.0) atomicMax(&sh.from, kThreads + (kThreads - 1 - tid));
    __syncthreads();
    const int from = sh.from >= kThreads ? 2 * kThreads - 1 - sh.from : sh.from;
    if (warp != from / 32) return f;
    // the tokens of that run, by the warp of its thread
    const int e_lo = __shfl_sync(kFull, v0, from & 31) * E, e_hi = __shfl_sync(kFull, v1, from & 31) * E;
    double acc = __shfl_sync(kFull, start, from & 31);
    for (int e0 = e_lo; e0 < e_hi; e0 += 32) {
      const int id = e0 + lane;
      const double w = id < e_hi ? weight(T::load1(z, id), id) : 0.0;
      const double sum = scan_warp(w, lane);
      const unsigned hit = __ballot_sync(kFull, w > 0.0 && acc + sum > aim);
      const unsigned live = __ballot_sync(kFull, w > 0.0);
      const int at_lane = hit ? __ffs(hit) - 1 : live ? 31 - __clz(live) : -1;
      if (at_lane >= 0) {
        f.id = e0 + at_lane;
        f.weight = __shfl_sync(kFull, w, at_lane);
      }
      if (hit) break;
      acc += __shfl_sync(kFull, sum, 31);
    }
    f.mine = lane == 0;
    return f;
  }
  // The same where no sums are known yet.
  template <typename F>
  __device__ __forceinline__ Found locate(F weight, double u, double aim) {
    double mine = 0.0;
    along([&](const uint4& v, int at) {
      float x[E];
      T::unpack(v, x);
      double w[E];
#pragma unroll
      for (int e = 0; e < E; ++e) w[e] = weight(x[e], at * E + e);
#pragma unroll
      for (int e = 0; e < E; ++e) mine += w[e];
    });
    return pick(mine, weight, u, aim);
  }

  // The token of a row of which all stays, in fp64.
  __device__ __forceinline__ Found locate_all(double u) {
    double m = 0.0;
    const float from = near_from();
    along([&](const uint4& v, int) {
      float x[E];
      double w[E];
      raw_of(v, from, x, w);
      m += sum_of(w);
    });
    return pick(m, [&](float x, int) { return raw(x); }, u, 0.0);
  }

  // ---- rows of which more stays than a list holds: the tokens are counted by their distance from the largest logit, which
  // tells where the border lies to a bin; one pass in fp64 then sums what lies above that interval, range by range, and
  // lists what lies in it.  All that is decided is decided by these sums; where the border does not lie in the interval, or
  // that holds too many, ok is false.
  struct Wide {
    bool ok;
    int n, listed;      // tokens that stay, how many of them in the list
    uint64_t border;
    double total, run;  // mass of what stays; of the thread's part of its warp's range above the interval
    bool near;          // not ok for more tokens than a list holds between these values, and the mass looked for
    uint32_t lo, hi;
    double goal;
  };
  // Values from bin b0 to bin b1 (a little more: what rounds is looked at, not trusted).
  __device__ __forceinline__ void interval(int b0, int b1, uint32_t* lo, uint32_t* hi) const {
    const float unit = fminf(static_cast<float>(scale), 1e30f), nudge = 1e-6f * (fabsf(M) + 32.f / unit);
    *hi = b0 <= 0 ? 0xffffffffu : orderable(M - static_cast<float>(b0) * (1.f / 64) / unit + nudge);
    *lo = max(orderable(M - static_cast<float>(b1 + 1) * (1.f / 64) / unit - nudge), orderable(-INFINITY) + 1);
  }
  __device__ __forceinline__ void clear_bins() {
    __syncthreads();
    for (int i = tid; i < kWideBins; i += kThreads) sh.wide[i] = 0;
    __syncthreads();
  }
  // Sums the CTAs' bins, each CTA a part of them, and tells all: tokens in wide_n, with kPlaces about their mass in wide_m.
  template <bool kPlaces>
  __device__ __forceinline__ void join_bins() {
    cluster_sync();
    constexpr int kPart = kWideBins / kCluster;
#pragma unroll
    for (int t = 0; t < kPart / kThreads; ++t) {
      const int b = rank * kPart + t * kThreads + tid;
      uint32_t n = 0, places = 0;
#pragma unroll
      for (int d = 0; d < kCluster; ++d) {
        const uint32_t w = static_cast<uint32_t>(far_i32(reinterpret_cast<const int*>(&sh.wide[b]), d));
        n += kPlaces ? w >> 20 : w;
        places += kPlaces ? w & 0xfffffu : 0;
      }
      const float place = n > 0 ? (static_cast<float>(places) / static_cast<float>(n) + 0.5f) * (1.f / 256) : 0.f;
      const float m = kPlaces ? n * ex2_approx(-(static_cast<float>(b) + place) * (1.f / 64)) : 0.f;
#pragma unroll
      for (int d = 0; d < kCluster; ++d) {
        asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(in_cta(smem_of(&sh.wide_n[b]), d)), "r"(n) : "memory");
        if (kPlaces) asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(in_cta(smem_of(&sh.wide_m[b]), d)), "f"(m) : "memory");
      }
    }
    cluster_sync();
  }
  __device__ __forceinline__ void wide(int top_k, float top_p, float floor, Wide* out) {
    constexpr int kOf = kWideBins / kThreads;
    out->ok = out->near = false;
    const float unit = fminf(static_cast<float>(scale), 1e30f);
    // bins of 1/64 in log2 units, the last one for all from 32 on
    clear_bins();
    each([&](float x, int) {
      // (the number of tokens in the upper 12 bits, the sum of their places in the bin, in 256ths, in the lower 20: more
      // than 4095 tokens in a bin spoil both: they then tell of fewer, and what follows from them is looked at)
      const int d = static_cast<int>(fminf((M - x) * (unit * (64.f * 256.f)), kWideBins * 256.f - 1.f));
      if (x > -INFINITY) atomicAdd(&sh.wide[d >> 8], (1u << 20) + (d & 255));
    });
    if (tid == 0) sh.bin = sh.bin2 = kWideBins;
    join_bins<true>();
    int n[kOf];
    float each_m[kOf];  // about the mass of a bin's tokens
    double sum_n = 0.0, sum_m = 0.0;
#pragma unroll
    for (int i = 0; i < kOf; ++i) {
      n[i] = sh.wide_n[tid * kOf + i];
      each_m[i] = sh.wide_m[tid * kOf + i];
      sum_n += n[i];
      sum_m += each_m[i];
    }
    double all_n, all_m;
    const double before_n = before_cta(sum_n, &all_n), before_m = before_cta(sum_m, &all_m);
    const bool k = top_k > 0 && all_n >= top_k, p = top_p < 1.f;
    double at_n = before_n, at_m = before_m;
    if (tid == 0 && !k) sh.value = all_m;
    if (k && before_n < top_k && before_n + sum_n >= top_k) {
#pragma unroll
      for (int i = 0; i < kOf; ++i) {
        if (at_n < top_k && at_n + n[i] >= top_k) {
          sh.bin2 = tid * kOf + i;
          sh.value = at_m + (top_k - at_n) / n[i] * each_m[i];  // about the mass of the first top_k
        }
        at_n += n[i];
        at_m += each_m[i];
      }
    }
    __syncthreads();
    const int b_k = sh.bin2;
    const double goal_about = static_cast<double>(top_p) * sh.value, off_about = 5e-5 * all_m;
    int mine = kWideBins;
    if (p) {
      at_m = before_m;
#pragma unroll
      for (int i = 0; i < kOf; ++i) {
        at_m += each_m[i];
        if (mine == kWideBins && n[i] > 0 && at_m >= goal_about) {
          mine = tid * kOf + i;
          // whether the border may lie in the bin before it, or behind it
          sh.wide[mine] = (at_m - each_m[i] > goal_about - off_about ? 1 : 0) | (at_m < goal_about + off_about ? 2 : 0);
        }
      }
      mine = static_cast<int>(__reduce_min_sync(kFull, static_cast<unsigned>(mine)));
      if (lane == 0 && mine < kWideBins) atomicMin(&sh.bin, mine);
    }
    __syncthreads();
    const int b_p = p ? sh.bin : kWideBins;
    const float x_floor = floor > 0.f ? -__log2f(floor) * 64.f : static_cast<float>(kWideBins);
    const int b_m = static_cast<int>(fminf(x_floor, static_cast<float>(kWideBins)));
    const int b = min(min(b_k, b_p), b_m);
    const bool two = k && p;  // the mass of the first top_k is needed, whatever binds
    if (b >= kWideBins - 1 || (two && b_k >= kWideBins - 1)) return;
    int edge = b == b_p ? static_cast<int>(sh.wide[b]) : 0;  // (a count is exact)
    if (b == b_m) edge |= (x_floor - b < 0.02f ? 1 : 0) | (x_floor - b > 0.98f ? 2 : 0);
    const int held = sh.wide_n[b] + (two ? sh.wide_n[b_k] : 0);
    const int up = edge & 1 && b > 0 ? sh.wide_n[b - 1] : 0, down = edge & 2 ? sh.wide_n[b + 1] : 0;
    int b0 = b, b1 = b;
    if (held + up + down <= kAim) {
      if (edge & 1) b0 = max(b - 1, 0);
      if (edge & 2) b1 = min(b + 1, kWideBins - 2);
    }
    // (a border that the estimate puts next to where it is, is looked for in the bins there)
#pragma unroll 1
    for (int turn_ = 0; turn_ < 4; ++turn_) {
      uint32_t lo, hi, lo2 = 0xffffffffu, hi2 = orderable(-INFINITY);  // (the second one holds nothing)
      interval(b0, b1, &lo, &hi);
      if (two) {
        interval(b_k, b_k, &lo2, &hi2);
        if (hi2 >= lo || hi2 == 0xffffffffu) {  // they meet: one
          lo = min(lo, lo2);
          hi = max(hi, hi2);
          lo2 = lo;
          hi2 = hi;
        }
      }
      const float f_lo = from_orderable(lo), f_lo2 = two ? from_orderable(lo2) : INFINITY;
      const float f_hi = hi == 0xffffffffu ? INFINITY : from_orderable(hi), f_hi2 = hi2 == 0xffffffffu ? INFINITY : from_orderable(hi2);
      if (tid == 0) sh.n_list = 0;
      __syncthreads();
      // ---- the pass in fp64: mass and number above the interval, and above the second one (without top-k: of all)
      double above = 0.0, above2 = 0.0;
      int n_above = 0, n_above2 = 0;
      const float near = near_from();
      along([&](const uint4& v, int at) {
        float x[E];
        double w[E];
        raw_of(v, near, x, w);
        bool in = false;
        if (p) {  // (what lies above the second interval is more)
#pragma unroll
          for (int e = 0; e < E; ++e) {
            const bool a2 = x[e] > f_hi2;
            w[e] = a2 ? w[e] : 0.0;
            n_above2 += a2;
            in |= !a2 && x[e] >= f_lo2;
          }
          above2 += sum_of(w);
        }
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const bool a1 = x[e] > f_hi;
          w[e] = a1 ? w[e] : 0.0;
          n_above += a1;
          in |= !a1 && x[e] >= f_lo;
        }
        above += sum_of(w);
        if (in) {
#pragma unroll
          for (int e = 0; e < E; ++e)
            if ((x[e] >= f_lo && x[e] <= f_hi) || (x[e] >= f_lo2 && x[e] <= f_hi2)) {
              const int i = atomicAdd(&sh.n_list, 1);
              if (i < kList) sh.list[i] = make_key(x[e], at * E + e);
            }
        }
      });
      out->run = above;
      const Mail r = reduce(above, above2, n_above, n_above2);
      const int n_all = join();
      if (n_all > kList) {
        cluster_sync();  // (the others may still read this CTA's count, which is begun anew)
        out->near = top_k == 0 || !p;
        out->lo = lo;
        out->hi = hi;
        out->goal = static_cast<double>(top_p) * r.b;
        return;
      }
      uint64_t* list = tokens();
      sort(list, n_all);
      // ---- the list: first the interval's, then (with both limits) the second one's
      const int each_thread = (n_all + kThreads - 1) / kThreads;
      double w[kEach], of_mine = 0.0, all;
      int first_n = 0, later = 0;  // tokens of the interval; tokens above the second one
#pragma unroll
      for (int e = 0; e < kEach; ++e) {
        const int i = tid * each_thread + e;
        w[e] = 0.0;
        if (e < each_thread && i < n_all) {
          const uint32_t key = static_cast<uint32_t>(list[i] >> 32);
          w[e] = raw(from_orderable(key));
          sh.scan[i] = w[e];
          first_n += key >= lo;
          later += key > hi2;
        }
        of_mine += w[e];
      }
      const double before = before_cta(of_mine, &all);
      first_n = sum_cta(first_n | later << 16);
      later = first_n >> 16;
      first_n &= 0xffff;
      // mass of the first top_k: what lies above the second interval, and the first of its tokens
      double mass = r.b;
      const int of2 = top_k - r.m;
      if (two) {
        if (of2 < 1 || later + of2 > n_all) return;
        double acc = before;
        if (tid == 0) sh.value2 = 0.0;
        __syncthreads();
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
          const int i = tid * each_thread + e;
          acc += w[e];
          if (e < each_thread && i < n_all) {
            if (i == later - 1) sh.value2 = acc;
            if (i == later + of2 - 1) sh.value = acc;
          }
        }
        __syncthreads();
        mass = r.b + (sh.value - sh.value2);
      } else if (p && top_k > 0 && r.m >= top_k) {
        return;  // (the bins, spoiled, told of fewer tokens than there are)
      }
      const double goal = static_cast<double>(top_p) * mass;
      int below = 0, heavy = 0;
      double acc = r.a + before;
#pragma unroll
      for (int e = 0; e < kEach; ++e) {
        const int i = tid * each_thread + e;
        acc += w[e];
        if (e < each_thread && i < first_n) {
          below += acc < goal;
          heavy += w[e] >= static_cast<double>(floor);
        }
      }
      below = sum_cta(below | heavy << 16);
      heavy = below >> 16;
      below &= 0xffff;
      int stay = first_n + 1;  // (more than the interval holds)
      bool higher = false;     // the border lies above the interval
      if (k) {
        stay = min(stay, top_k - r.n);
        higher |= top_k - r.n < 1;
      }
      if (p) {
        stay = min(stay, below + 1);
        higher |= r.n > 0 && r.a >= goal;
      }
      if (floor > 0.f) {
        if (heavy < first_n || raw(from_orderable(lo)) < static_cast<double>(floor)) stay = min(stay, heavy);
        higher |= heavy == 0 && (r.n == 0 || raw(f_hi) < static_cast<double>(floor));
      }
      if (higher || stay > first_n) {
        if (higher ? b0 == 0 : b1 >= kWideBins - 2) return;
        cluster_sync();  // (as above, and the list)
        if (higher) {
          b1 = b0 - 1;
          b0 = max(b1 - 3, 0);
        } else {
          b0 = b1 + 1;
          b1 = min(b0 + 3, kWideBins - 2);
        }
        continue;
      }
      if (top_k > 0 && r.n + stay > top_k) return;  // (as above)
      __syncthreads();
      if (tid == 0) {  // (of the interval none: what lies above it)
        sh.value = r.a;
        sh.cut.border = static_cast<uint64_t>(hi) + 1 << 32;
      }
      __syncthreads();
      acc = r.a + before;
#pragma unroll
      for (int e = 0; e < kEach; ++e) {
        acc += w[e];
        if (e < each_thread && tid * each_thread + e == stay - 1) {
          sh.value = acc;
          sh.cut.border = list[stay - 1];
        }
      }
      __syncthreads();
      out->ok = true;
      out->n = r.n + stay;
      out->listed = stay;
      out->border = sh.cut.border;
      out->total = sh.value;
      return;
    }
  }
  // The token of such a row.  taken(lo, hi): mass that is taken out of ids lo .. hi-1.
  template <typename G, typename F>
  __device__ __forceinline__ Found draw_wide(const Wide& of, double u, G taken, F weight) {
    const uint64_t* list = tokens();
    int lo, hi;
    range_of(warp, &lo, &hi);
    double run = of.run;
    for (int i = lane; i < of.listed; i += 32) {
      const int id = key_id(list[i]);
      if (id >= lo * E && id < hi * E) run += sh.scan[i];
    }
    const double gone = hi > lo ? taken(lo * E, hi * E) : 0.0;
    if (gone > 0.0) {
      const double rest = sum_warp(run) - gone;
      run = lane == 0 ? rest : 0.0;
      if (rest < 1e-4 * gone) {  // (few digits of it are left, it may be nothing: added up without what is taken out)
        run = 0.0;
#pragma unroll 1
        for (int id = lo * E + lane; id < hi * E; id += 32) run += weight(T::load1(z, id), id);
      }
    }
    return pick(run, weight, u, 0.0);
  }

  // ---- rows of which much stays.  The border of a count of tokens (goal_n > 0) or of a mass, among those at or above `kept`:
  // an interval of values is narrowed to the border's, first by the tokens' distances from the row's largest logit,
  // then (of.near: from there on) by equal parts of what is left, until a list takes its tokens or they are all equal.
  __device__ __forceinline__ uint64_t wide_border(uint64_t kept, int goal_n, double goal, const Wide& of) {
    const bool by_n = goal_n > 0;
    const float from = near_from();
    const float unit = fminf(static_cast<float>(scale), 1e30f);
    // The bin at which the count, or about the mass, is reached: (bin, tokens in it).  weight(b): mass of a token in bin b.
    const auto find = [&](auto weight, bool by_n, double goal_n, double n0, double m0, double stretch) {
      join_bins<false>();
      constexpr int kOf = kWideBins / kThreads;
      int n[kOf];
      double sum_n = 0.0, sum_m = 0.0;
#pragma unroll
      for (int i = 0; i < kOf; ++i) {
        n[i] = sh.wide_n[tid * kOf + i];
        sum_n += n[i];
        if (!by_n && n[i] > 0) sum_m += n[i] * static_cast<double>(weight(tid * kOf + i));
      }
      double all_n, all_m = 0.0;
      double at_n = n0 + before_cta(sum_n, &all_n), at_m = 0.0;
      if (!by_n) {
        at_m = before_cta(sum_m, &all_m);
        // the bins' masses are estimates: stretched to the whole that is known
        const double s = stretch > 0.0 && all_m > 0.0 ? stretch / all_m : 1.0;
        at_m = m0 + at_m * s;
        sum_m = s;
      }
      if (tid == 0) sh.bin = kWideBins;
      __syncthreads();
      int last = -1;
#pragma unroll
      for (int i = 0; i < kOf; ++i) {
        at_n += n[i];
        if (!by_n && n[i] > 0) at_m += n[i] * static_cast<double>(weight(tid * kOf + i)) * sum_m;
        if (n[i] > 0) last = tid * kOf + i;
        if (n[i] > 0 && (by_n ? at_n >= goal_n : at_m >= goal)) {
          atomicMin(&sh.bin, tid * kOf + i);
          break;
        }
      }
      last = __reduce_max_sync(kFull, last);
      if (lane == 0) sh.red_n[flip][warp] = last;
      __syncthreads();
      int b = sh.bin;
      if (b == kWideBins) {
        b = -1;
        for (int v = 0; v < kWarps; ++v) b = max(b, sh.red_n[flip][v]);
      }
      flip ^= 1;
      return b;
    };
    uint32_t lo = of.lo, hi = of.hi;
    if (!of.near) {
      // ---- by distance: bins of 1/64 in log2 units, the last one for all from 32 on
      clear_bins();
      each([&](float x, int id) {
        if (x == -INFINITY || make_key(x, id) < kept) return;
        const float d = (M - x) * unit;
        atomicAdd(&sh.wide[d < 31.98f ? static_cast<int>(d * 64.f) : kWideBins - 1], 1);
      });
      const int b0 = find([](int b) { return ex2_approx(-(static_cast<float>(b) + 0.5f) * (1.f / 64)); }, by_n, goal_n, 0.0, 0.0, 0.0);
      // (a little more than the bin: what rounds is looked at, not trusted)
      const auto value_at = [&](float d) { return M - d / unit; };
      const float nudge = 1e-6f * (fabsf(M) + 32.f / unit);
      hi = b0 <= 0 ? 0xffffffffu : orderable(value_at(static_cast<float>(b0) * (1.f / 64)) + nudge);
      lo = b0 >= kWideBins - 1 ? 0u : orderable(value_at(static_cast<float>(b0 + 1) * (1.f / 64)) - nudge);
    }
    // (bounds that are known, and how often an estimate has missed: then the part with the middle token is taken, every other time)
    uint32_t lo_known = 0, hi_known = 0xffffffffu;
    int missed = 0;
    for (int turn_ = 0;; ++turn_) {
      // ---- what lies above the interval, and in it
      if (tid == 0) sh.n_list = 0;
      __syncthreads();
      double above = 0.0, in = 0.0;
      int n_above = 0, n_in = 0;
      uint32_t least = 0xffffffffu, most = 0;
      each([&](float x, int id) {
        const uint32_t k = orderable(x);
        if (x == -INFINITY || k < lo || make_key(x, id) < kept) return;
        const double w = by_n ? 0.0 : raw_any(x, from);
        if (k > hi) {
          ++n_above;
          above += w;
          return;
        }
        ++n_in;
        in += w;
        least = min(least, k);
        most = max(most, k);
        const int at = atomicAdd(&sh.n_list, 1);
        if (at < kList) sh.list[at] = make_key(x, id);
      });
      const Mail s = reduce(above, in, n_above, n_in);
      least_most(&least, &most);
      const bool is_above = s.n > 0 && (by_n ? s.n >= goal_n : s.a >= goal);
      const bool is_in = s.m > 0 && (by_n ? s.n + s.m >= goal_n : s.a + s.b >= goal);
      const bool last_turn = turn_ >= 100;  // (sums of 1e5 terms that round differently: then either is right)
      if (!last_turn && ((is_above && hi != 0xffffffffu) || (!is_above && !is_in && lo > 0))) {
        if (is_above) lo_known = hi + 1;
        else hi_known = lo - 1;
        if (lo_known > hi_known) {  // (sums that round differently)
          lo_known = 0;
          hi_known = 0xffffffffu;
        }
        lo = lo_known;
        hi = hi_known;
        ++missed;
        continue;
      }
      if (s.m == 0) return kept;  // (nothing below: all stays)
      if (s.m <= kList) {
        const int n = join();
        uint64_t* list = tokens();
        sort(list, n);
        int stay = by_n ? goal_n - s.n : 0;
        if (!by_n) {
          const int each_thread = (n + kThreads - 1) / kThreads;
          double w[kEach], mine = 0.0, all;
#pragma unroll
          for (int e = 0; e < kEach; ++e) {
            const int i = tid * each_thread + e;
            w[e] = e < each_thread && i < n ? raw(key_value(list[i])) : 0.0;
            mine += w[e];
          }
          double acc = s.a + before_cta(mine, &all);
          int below = 0;
#pragma unroll
          for (int e = 0; e < kEach; ++e) {
            acc += w[e];
            below += e < each_thread && tid * each_thread + e < n && acc < goal;
          }
          stay = sum_cta(below) + 1;
        }
        const uint64_t border = list[min(max(stay, 1), n) - 1];
        __syncthreads();
        return border;
      }
      if (least == most) {  // all equal: the first of them by id
        const float value = from_orderable(least);
        double j;
        if (by_n) {
          j = goal_n - s.n;
        } else {
          const double w = raw(value);
          j = fmin(fmax(w > 0.0 ? ceil((goal - s.a) / w) : 1.0, 1.0), static_cast<double>(s.m));
          while (j > 1.0 && s.a + (j - 1.0) * w >= goal) j -= 1.0;
          while (j < s.m && s.a + j * w < goal) j += 1.0;
        }
        j = fmin(fmax(j, 1.0), static_cast<double>(s.m));
        const Found f = locate(
            [&](float x, int id) { return orderable(x) == least && make_key(x, id) >= kept ? 1.0 : 0.0; }, -1.0, j - 0.5);
        uint32_t id = f.mine ? static_cast<uint32_t>(f.id) : 0xffffffffu, unused = 0;
        least_most(&id, &unused);
        return make_key(value, static_cast<int>(id));
      }
      lo = least;
      hi = most;
      const int shift = max(0, 32 - __clz(hi - lo) - 11);
      clear_bins();
      each([&](float x, int id) {
        const uint32_t k = orderable(x);
        if (k < lo || k > hi || make_key(x, id) < kept) return;
        atomicAdd(&sh.wide[(hi - k) >> shift], 1);
      });
      const int b = find(
          [&](int i) {
            const uint64_t far = (static_cast<uint64_t>(i) << shift) + ((1u << shift) >> 1);
            return raw(from_orderable(hi - static_cast<uint32_t>(min(static_cast<uint64_t>(hi - lo), far))));
          },
          by_n || missed % 2 == 1, by_n ? goal_n : s.n + 0.5 * s.m, s.n, s.a, s.b);
      const uint32_t from = static_cast<uint32_t>(max(b, 0)) << shift;
      const uint32_t top = hi - from;
      lo = top - lo >= (1u << shift) ? top - ((1u << shift) - 1) : lo;
      hi = top;
    }
  }
};

}  // namespace gto
