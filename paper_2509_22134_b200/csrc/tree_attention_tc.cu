// gto_tree_attention on the tensor cores: 16-bit tensors, heads of 64 or 128.
//
// Rows.  A query row is one token and one of the query heads that share a key head; the rows of a
// chunk and key head are cut into blocks of 256, two tiles of 128 (the M of the matrix
// instruction), so that a tile of keys and values read once serves up to 256 rows.  With 128 rows
// or fewer (single tokens, small trees) the two halves of the CTA take the even and the odd tiles
// of the same rows instead and join at the end, which halves the dependent chain product -> softmax
// -> product that a tile costs.
//
// Work.  A block of rows costs one unit for each 128 cache entries that it sees, plus kOverhead.
// All units of the call, in the order (sequence, key head, block, entries), are cut into as
// many equal spans as there are SMs; every CTA takes one.  A block that a cut goes through leaves
// its unnormalised parts in the workspace and a second, small kernel joins them in the order of
// the entries.  The lengths are read on the device; the cut depends on nothing else, so that equal
// calls give equal bits.
//
// A CTA is 12 warps: two groups of four own a tile's 128 rows, one thread a row, and do the
// softmax and the epilogue; one warp issues the copies of keys and values (TMA boxes out of the
// pages into a ring of stages), one the matrix instructions, two the copies of queries and the
// tidying of tiles at the end of a sequence.  Scores, weights and accumulators live in tensor
// memory: S0 S1 (128 columns each; the weights P overwrite the first 64), O0 O1.
//
// Rounding.  Scores, maxima, sums and outputs are fp32; the weights are rounded to the 16-bit type
// to be an operand of the second product (half a step each, independent errors), while their sum
// is taken before that rounding.  The reference maximum of a row follows its true maximum only when
// it has risen by more than 8 in log2 units: weights stay below 2^8, and most tiles need no
// rescaling of the output.
#include <cuda.h>

#include "decode_common.cuh"

namespace gto {
namespace {

constexpr int kThreads = 384;
constexpr int kTile = 128;       // cache entries of a tile, rows of a row tile
constexpr int kOverhead = 1;     // cost of a block beside its tiles, in tiles
constexpr int kTidyRing = 8;     // more than the value tiles that the ring of stages can hold
constexpr float kLazy = 8.0f;    // log2 units the maximum may rise before the output is rescaled
constexpr long long kWaitCycles = 1ll << 32;  // about two seconds

template <int DH>
struct Layout {
  static constexpr int kTileBytes = kTile * DH * 2;
  static constexpr int kHalves = DH / 64;              // 128-byte columns of a tile
  static constexpr int kHalfBytes = kTile * 128;
  static constexpr int kStages = DH == 128 ? 5 : 12;
  static constexpr int kQ = 0;
  static constexpr int kRing = 2 * kTileBytes;
  static constexpr int kTail = kRing + kStages * kTileBytes;
};

struct Tail {
  uint64_t full[12], empty[12];
  uint64_t q_full, q_empty, other;
  uint64_t s_ready[2], p_ready[2], pv_done[2], o_free[2];
  // a value tile at the end of what its rows see: loaded (go), then tidied; `full` of its stage says
  // only that it was issued, the weights that meet it wait for `tidy`
  uint64_t go[kTidyRing], tidy[kTidyRing];
  uint32_t bad[kTidyRing][4];   // entries of the tile whose values are not finite
  float ml[kTile][2];           // maximum and sum of the odd tiles' rows
  int64_t scan[kThreads / 32];
  int64_t span, rem;
  int64_t units;
  int seq, ctas;
  uint32_t tmem;
  int abort;
};

// ------------------------------------------------------------------ instructions
__device__ __forceinline__ uint32_t smem_u32(const void* p) {
  return static_cast<uint32_t>(__cvta_generic_to_shared(p));
}
__device__ __forceinline__ void bar_init(uint64_t* b, int count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_u32(b)), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint64_t* b) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(b)) : "memory");
}
__device__ __forceinline__ void bar_expect(uint64_t* b, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(smem_u32(b)), "r"(bytes)
               : "memory");
}
__device__ __forceinline__ bool bar_try(uint64_t* b, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}"
      : "=r"(ok)
      : "r"(smem_u32(b)), "r"(parity)
      : "memory");
  return ok != 0;
}
// Waits until the phase of that parity has completed; false after kWaitCycles or when another
// warp has given up.
__device__ __forceinline__ bool bar_wait(uint64_t* b, uint32_t parity, volatile int* abort) {
  if (bar_try(b, parity)) return true;
  const long long t0 = clock64();
  while (!bar_try(b, parity)) {
    if (*abort) return false;
    if (clock64() - t0 > kWaitCycles) {
      *abort = 1;
      return false;
    }
  }
  return true;
}
__device__ __forceinline__ void fence_async() {
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
}
__device__ __forceinline__ void tc_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_commit(uint64_t* b) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(b))
               : "memory");
}
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool acc) {
  asm volatile(
      "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n"
      " tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}" ::"r"(d), "l"(a), "l"(b), "r"(idesc),
      "r"(static_cast<uint32_t>(acc))
      : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, bool acc) {
  asm volatile(
      "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n"
      " tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}" ::"r"(d), "r"(a), "l"(b), "r"(idesc),
      "r"(static_cast<uint32_t>(acc))
      : "memory");
}
__device__ __forceinline__ void tma_4d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, int w,
                                       uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], "
      "[%6];" ::"r"(dst),
      "l"(map), "r"(x), "r"(y), "r"(z), "r"(w), "r"(smem_u32(bar))
      : "memory");
}
#define GTO_R8(p, i) "=r"(p[i]), "=r"(p[i + 1]), "=r"(p[i + 2]), "=r"(p[i + 3]), "=r"(p[i + 4]), "=r"(p[i + 5]), "=r"(p[i + 6]), "=r"(p[i + 7])
#define GTO_I8(p, i) "r"(p[i]), "r"(p[i + 1]), "r"(p[i + 2]), "r"(p[i + 3]), "r"(p[i + 4]), "r"(p[i + 5]), "r"(p[i + 6]), "r"(p[i + 7])
// 32 columns of the thread's own tensor-memory row
__device__ __forceinline__ void tm_ld32(uint32_t (&r)[32], uint32_t addr) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : GTO_R8(r, 0), GTO_R8(r, 8), GTO_R8(r, 16), GTO_R8(r, 24)
      : "r"(addr));
}
__device__ __forceinline__ void tm_st32(uint32_t addr, const uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
      "{%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};" ::"r"(addr),
      GTO_I8(r, 0), GTO_I8(r, 8), GTO_I8(r, 16), GTO_I8(r, 24)
      : "memory");
}
__device__ __forceinline__ void tm_st16(uint32_t addr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
      "{%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(addr),
      GTO_I8(r, 0), GTO_I8(r, 8)
      : "memory");
}
// The registers of a load hold its values only after the wait: naming them as operands of the wait
// (and of an empty statement after it) keeps arithmetic on them from moving ahead of it.
#define GTO_P8(p, i) "+r"(p[i]), "+r"(p[i + 1]), "+r"(p[i + 2]), "+r"(p[i + 3]), "+r"(p[i + 4]), "+r"(p[i + 5]), "+r"(p[i + 6]), "+r"(p[i + 7])
__device__ __forceinline__ void tm_wait_ld(uint32_t (&r)[32]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;" : GTO_P8(r, 0), GTO_P8(r, 8), GTO_P8(r, 16), GTO_P8(r, 24)::"memory");
}
__device__ __forceinline__ void tm_after_wait(uint32_t (&r)[32]) {
  asm volatile("" : GTO_P8(r, 0), GTO_P8(r, 8), GTO_P8(r, 16), GTO_P8(r, 24)::"memory");
}
__device__ __forceinline__ void tm_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Shared-memory operand, 128-byte swizzle: start, leading and stride byte offsets over 16, the
// version bit of this generation, swizzle mode 2.
__device__ __forceinline__ uint64_t smem_desc(uint32_t addr, uint32_t leading, uint32_t stride) {
  return static_cast<uint64_t>((addr >> 4) & 0x3fffu) | (static_cast<uint64_t>(leading >> 4) << 16) |
         (static_cast<uint64_t>(stride >> 4) << 32) | (1ull << 46) | (2ull << 61);
}
// fp32 accumulator, both operands of one 16-bit type, M = 128
__host__ __device__ constexpr uint32_t instr_desc(bool bf16, int n, bool b_rows_are_k) {
  return (1u << 4) | (bf16 ? (1u << 7) | (1u << 10) : 0u) | (b_rows_are_k ? 1u << 16 : 0u) |
         (static_cast<uint32_t>(n >> 3) << 17) | (static_cast<uint32_t>(128 >> 4) << 24);
}

template <typename T>
__device__ __forceinline__ uint32_t pack2(float a, float b);
template <>
__device__ __forceinline__ uint32_t pack2<Bf16>(float a, float b) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}
template <>
__device__ __forceinline__ uint32_t pack2<F16>(float a, float b) {
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}

// ------------------------------------------------------------------ work
struct Geometry {
  int group;  // query heads of a key head
  __device__ __forceinline__ int blocks(const Chunk& c) const {
    return c.ok ? static_cast<int>((static_cast<int64_t>(c.n) * group + 2 * kTile - 1) / (2 * kTile)) : 0;
  }
  // first and last token of block rb, its rows
  __device__ __forceinline__ int rows(const Chunk& c, int rb) const {
    const int64_t left = static_cast<int64_t>(c.n) * group - static_cast<int64_t>(rb) * 2 * kTile;
    return left < 2 * kTile ? static_cast<int>(left) : 2 * kTile;
  }
  __device__ __forceinline__ int end(const Chunk& c, int rb) const {
    const int64_t last = static_cast<int64_t>(rb) * 2 * kTile + rows(c, rb) - 1;
    return kv_end(c, static_cast<int>(last / group));
  }
  __device__ __forceinline__ int tiles(const Chunk& c, int rb) const { return (end(c, rb) + kTile - 1) / kTile; }
};

struct Item {
  int s, kvh, rb, rows;
  int t0, t1, n;       // tiles [t0, t1) of n
  int end;             // entries that any row of the block sees
  int common;          // entries that every row sees
  bool alike;          // all rows see the same entries
  int64_t after;       // units of the block that later CTAs do
  __device__ __forceinline__ bool whole() const { return t0 == 0 && t1 == n; }
  __device__ __forceinline__ bool dual() const { return rows > kTile; }
  __device__ __forceinline__ bool masked(int t) const { return (t + 1) * kTile > common; }
  // tiles of this item that stream st does before its tile number j (of the item)
};

struct Walk {
  const BatchArgs& b;
  Geometry g;
  int heads;
  int s, kvh, rb, nrb;
  int64_t off, left;
  Chunk c;

  __device__ Walk(const BatchArgs& batch, Geometry geo, int n_kv_heads, const Tail& t)
      : b(batch), g(geo), heads(n_kv_heads), s(t.seq), kvh(0), rb(0), nrb(0), off(t.rem), left(t.span) {
    if (left <= 0) return;
    c = load_chunk(b, s);
    nrb = g.blocks(c);
    int64_t per_head = 0;
    for (int i = 0; i < nrb; ++i) per_head += g.tiles(c, i) + kOverhead;
    kvh = static_cast<int>(off / per_head);
    off -= per_head * kvh;
    while (off >= g.tiles(c, rb) + kOverhead) {
      off -= g.tiles(c, rb) + kOverhead;
      ++rb;
    }
  }
  __device__ bool next(Item& it) {
    while (left > 0) {
      if (s >= b.S) return false;
      const int n = g.tiles(c, rb);
      const int64_t u = n + kOverhead;
      const int64_t take = left < u - off ? left : u - off;
      it.s = s;
      it.kvh = kvh;
      it.rb = rb;
      it.rows = g.rows(c, rb);
      it.n = n;
      it.t0 = off > kOverhead ? static_cast<int>(off - kOverhead) : 0;
      it.t1 = off + take > kOverhead ? static_cast<int>(off + take - kOverhead) : 0;
      it.end = g.end(c, rb);
      const int first = static_cast<int>(static_cast<int64_t>(rb) * 2 * kTile / g.group);
      const int last = static_cast<int>((static_cast<int64_t>(rb) * 2 * kTile + it.rows - 1) / g.group);
      it.common = first < c.lead ? c.base + first + 1 : c.base + c.lead;
      it.alike = first == last && first < c.lead;
      it.after = u - off - take;
      chunk = c;
      left -= take;
      off = 0;
      if (++rb == nrb) {
        rb = 0;
        if (++kvh == heads) {
          kvh = 0;
          do {
            if (++s >= b.S) break;
            c = load_chunk(b, s);
            nrb = g.blocks(c);
          } while (nrb == 0);
        }
      }
      if (it.t1 > it.t0) return true;
    }
    return false;
  }
  Chunk chunk;  // of the item that next() gave
};

struct Meta {  // of a block whose first part a CTA did
  int32_t s, kvh, rb, parts;
};

struct TcArgs {
  AttnArgs a;
  Meta* meta;
  float4* part;   // [slot][DH/4][256]
  float2* part_ml;  // [slot][256]
  int boxes;      // TMA boxes that make up a tile's rows
  int box_rows;
};

__device__ __forceinline__ int64_t cut(int64_t units, int ctas, int c) { return units * c / ctas; }

// Every thread of the CTA: units of the call, this CTA's span and where it begins.
__device__ void plan(const BatchArgs& b, Geometry g, int heads, Tail& t) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  // a thread owns a run of sequences
  const int per = (b.S + kThreads - 1) / kThreads;
  const int s0 = min(tid * per, b.S), s1 = min(s0 + per, b.S);
  int64_t mine = 0;
  for (int s = s0; s < s1; ++s) {
    const Chunk c = load_chunk(b, s);
    if (!c.ok) {
      if (blockIdx.x == 0) atomicOr(b.status, kStatusBadIndex);
      continue;
    }
    const int nrb = g.blocks(c);
    int64_t u = 0;
    for (int i = 0; i < nrb; ++i) u += g.tiles(c, i) + kOverhead;
    mine += u * heads;
  }
  int64_t run = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int64_t y = __shfl_up_sync(kFull, run, o);
    if (lane >= o) run += y;
  }
  if (lane == 31) t.scan[warp] = run;
  if (tid == 0) {
    t.span = 0;
    t.rem = 0;
    t.seq = 0;
  }
  __syncthreads();
  int64_t units = 0;
  for (int w = 0; w < kThreads / 32; ++w) {
    if (w < warp) run += t.scan[w];
    units += t.scan[w];
  }
  const int ctas = units < static_cast<int64_t>(gridDim.x) ? static_cast<int>(units) : static_cast<int>(gridDim.x);
  if (tid == 0) {
    t.units = units;
    t.ctas = ctas;
  }
  if (static_cast<int>(blockIdx.x) < ctas) {
    const int64_t from = cut(units, ctas, blockIdx.x), to = cut(units, ctas, blockIdx.x + 1);
    int64_t before = run - mine;
    if (from >= before && from < run) {
      for (int s = s0; s < s1; ++s) {
        const Chunk c = load_chunk(b, s);
        const int nrb = g.blocks(c);
        int64_t u = 0;
        for (int i = 0; i < nrb; ++i) u += g.tiles(c, i) + kOverhead;
        u *= heads;
        if (from < before + u) {
          t.seq = s;
          t.rem = from - before;
          t.span = to - from;
          break;
        }
        before += u;
      }
    }
  }
  __syncthreads();
}

// ------------------------------------------------------------------ the kernel
template <typename T, int DH>
__global__ void __launch_bounds__(kThreads, 1)
    attention_tc_kernel(const __grid_constant__ TcArgs p, const __grid_constant__ CUtensorMap k_map,
                        const __grid_constant__ CUtensorMap v_map) {
  using L = Layout<DH>;
  extern __shared__ unsigned char s_dyn[];
  unsigned char* smem = s_dyn + ((1024u - (smem_u32(s_dyn) & 1023u)) & 1023u);
  Tail& t = *reinterpret_cast<Tail*>(smem + L::kTail);
  const uint32_t q_base = smem_u32(smem + L::kQ), ring = smem_u32(smem + L::kRing);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const AttnArgs& a = p.a;
  const Geometry geo{a.n_q_heads / a.c.n_kv_heads};
  volatile int* abort = &t.abort;

  if (tid == 0) {
    for (int i = 0; i < L::kStages; ++i) {
      bar_init(&t.full[i], 1);
      bar_init(&t.empty[i], 1);
    }
    bar_init(&t.q_full, 64);
    bar_init(&t.q_empty, 1);
    bar_init(&t.other, 4);
    for (int i = 0; i < 2; ++i) {
      bar_init(&t.s_ready[i], 1);
      bar_init(&t.p_ready[i], 4);
      bar_init(&t.pv_done[i], 1);
      bar_init(&t.o_free[i], 4);
    }
    for (int i = 0; i < kTidyRing; ++i) {
      bar_init(&t.go[i], 1);
      bar_init(&t.tidy[i], 64);
    }
    t.abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 9) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&t.tmem))
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  plan(a.b, geo, a.c.n_kv_heads, t);
  tc_before();
  __syncthreads();
  tc_after();
  const uint32_t tmem = t.tmem;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

  if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
    Walk walk(a.b, geo, a.c.n_kv_heads, t);
    Item it;
    if (warp == 8) {
      // ---- keys and values: TMA boxes into the ring
      uint32_t slot = 0, gone = 0;
      bool ok = true;
      while (ok && walk.next(it)) {
        for (int tile = it.t0; tile < it.t1 && ok; ++tile) {
          const int box = lane % p.boxes, half = lane / p.boxes;
          const int e = tile * kTile + box * p.box_rows;
          int page = -1;
          if (half < L::kHalves && e < it.end) {
            page = page_of(a.b, it.s, e);
            if (page < 0) atomicOr(a.b.status, kStatusBadIndex);
          }
          const uint32_t bytes = __popc(__ballot_sync(kFull, page >= 0)) * p.box_rows * 128;
          const int place = e % a.b.page_size;
#pragma unroll
          for (int kv = 0; kv < 2; ++kv, ++slot) {
            const uint32_t st = slot % L::kStages, round = slot / L::kStages;
            if (round > 0) ok = ok && bar_wait(&t.empty[st], (round - 1) & 1, abort);
            ok = __all_sync(kFull, ok);
            if (!ok) break;
            const bool apart = kv == 1 && it.masked(tile);
            uint64_t* bar = apart ? &t.go[gone % kTidyRing] : &t.full[st];
            if (lane == 0) bar_expect(bar, bytes);
            __syncwarp();
            if (page >= 0)
              tma_4d(ring + st * L::kTileBytes + half * L::kHalfBytes + box * p.box_rows * 128,
                     kv ? &v_map : &k_map, half * 64, it.kvh, place, page, bar);
            if (apart) {
              ++gone;
              if (lane == 0) bar_arrive(&t.full[st]);
            }
          }
        }
      }
      // copies in flight end before the CTA does
      for (uint32_t i = slot > L::kStages ? slot - L::kStages : 0; i < slot; ++i) {
        const long long t0 = clock64();
        while (!bar_try(&t.full[i % L::kStages], (i / L::kStages) & 1) && clock64() - t0 < kWaitCycles) {
        }
      }
      for (uint32_t i = gone > kTidyRing ? gone - kTidyRing : 0; i < gone; ++i) {
        const long long t0 = clock64();
        while (!bar_try(&t.go[i % kTidyRing], (i / kTidyRing) & 1) && clock64() - t0 < kWaitCycles) {
        }
      }
    } else if (warp == 9) {
      // ---- matrix instructions, by one thread
      if (lane == 0) {
        constexpr bool kBf16 = T::kNegInfElem == 0xff80u;
        constexpr uint32_t kIdQk = instr_desc(kBf16, kTile, false), kIdPv = instr_desc(kBf16, DH, true);
        uint32_t slot = 0, items = 0, pv[2] = {0, 0}, fin[2] = {0, 0};
        bool ok = true;
        auto qk = [&](int st, int q_tile, uint32_t stage) {
          const uint32_t qa = q_base + q_tile * L::kTileBytes, ka = ring + stage * L::kTileBytes;
#pragma unroll
          for (int k = 0; k < DH / 16; ++k) {
            const uint32_t at = (k / 4) * L::kHalfBytes + (k % 4) * 32;
            mma_ss(tmem + st * kTile, smem_desc(qa + at, 16, 1024), smem_desc(ka + at, 16, 1024), kIdQk, k > 0);
          }
          tc_commit(&t.s_ready[st]);
        };
        while (ok && walk.next(it)) {
          const bool dual = it.dual();
          const int nt = it.t1 - it.t0;
          const uint32_t base = slot;
          slot += 2 * nt;
          ok = bar_wait(&t.q_full, items & 1, abort);
          ++items;
          auto k_stage = [&](int j) { return (base + 2 * j) % L::kStages; };
          auto v_stage = [&](int j) { return (base + 2 * j + 1) % L::kStages; };
          auto wait_k = [&](int j) {
            return bar_wait(&t.full[k_stage(j)], ((base + 2 * j) / L::kStages) & 1, abort);
          };
          // first scores: both row tiles of tile 0, or tiles 0 and 1
          ok = ok && wait_k(0);
          if (!ok) break;
          tc_after();
          qk(0, 0, k_stage(0));
          if (dual) qk(1, 1, k_stage(0));
          tc_commit(&t.empty[k_stage(0)]);
          if (!dual && nt > 1) {
            ok = wait_k(1);
            if (!ok) break;
            qk(1, 0, k_stage(1));
            tc_commit(&t.empty[k_stage(1)]);
          }
          if (nt <= (dual ? 1 : 2)) tc_commit(&t.q_empty);
          bool started[2] = {false, false};
          for (int j = 0; j < nt && ok; ++j) {
            const uint32_t vs = v_stage(j);
            ok = bar_wait(&t.full[vs], ((base + 2 * j + 1) / L::kStages) & 1, abort);
            const int left = it.end - (it.t0 + j) * kTile;
            const int ks = left < kTile ? (left + 15) / 16 : kTile / 16;
            for (int st = dual ? 0 : (j & 1); st < (dual ? 2 : (j & 1) + 1) && ok; ++st) {
              if (!started[st]) {  // the block before this one has left its accumulator
                if (fin[st] > 0) ok = ok && bar_wait(&t.o_free[st], (fin[st] - 1) & 1, abort);
                ++fin[st];
              }
              ok = ok && bar_wait(&t.p_ready[st], pv[st] & 1, abort);
              if (!ok) break;
              ++pv[st];
              tc_after();
              const uint32_t va = ring + vs * L::kTileBytes;
              for (int k = 0; k < ks; ++k)
                mma_ts(tmem + 2 * kTile + st * kTile, tmem + st * kTile + k * 8,
                       smem_desc(va + k * 2048, L::kHalfBytes, 1024), kIdPv, started[st] || k > 0);
              started[st] = true;
              tc_commit(&t.pv_done[st]);
              const int jn = dual ? j + 1 : j + 2;  // the stream's next tile
              if (jn < nt) {
                if (!dual || st == 0) ok = wait_k(jn);
                if (!ok) break;
                qk(st, dual ? st : 0, k_stage(jn));
                if (!dual || st == 1) {
                  tc_commit(&t.empty[k_stage(jn)]);
                  if (jn == nt - 1) tc_commit(&t.q_empty);
                }
              }
            }
            if (ok) tc_commit(&t.empty[vs]);
          }
        }
        if (!ok) {  // given up: matrix instructions in flight end before tensor memory is freed
          tc_commit(&t.other);
          const long long t0 = clock64();
          while (clock64() - t0 < (1ll << 22)) {
          }
        }
      }
      __syncwarp();
    } else {
      // ---- queries, and tiles at the end of a sequence
      const int w = tid - 320;  // 0..63
      uint32_t items = 0, slot = 0, tidied = 0;
      int kept = 0;  // whether this CTA began a block that others end
      bool ok = true;
      while (ok && walk.next(it)) {
        if (items > 0) ok = bar_wait(&t.q_empty, (items - 1) & 1, abort);
        ok = __all_sync(kFull, ok);
        if (!ok) break;
        ++items;
        const Chunk& ch = walk.chunk;
        for (int v = w; v < it.rows * (DH / 8); v += 64) {
          const int r = v / (DH / 8), c = v % (DH / 8);
          const int64_t row = static_cast<int64_t>(it.rb) * 2 * kTile + r;
          const int64_t tok = ch.q0 + row / geo.group;
          const int h = it.kvh * geo.group + static_cast<int>(row % geo.group);
          const char* src = a.q + tok * a.q_stride + static_cast<int64_t>(h) * (DH * 2) + c * 16;
          const int rr = r % kTile;
          const uint32_t dst = q_base + (r / kTile) * L::kTileBytes + (c / 8) * L::kHalfBytes + rr * 128 +
                               (((c & 7) ^ (rr & 7)) << 4);
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
        fence_async();
        bar_arrive(&t.q_full);
        if (w == 0 && it.t0 == 0 && it.t1 < it.n) {
          int parts = 1;
          int64_t after = it.after;
          for (int c = blockIdx.x + 1; after > 0; ++c, ++parts)
            after -= cut(t.units, t.ctas, c + 1) - cut(t.units, t.ctas, c);
          p.meta[blockIdx.x] = Meta{it.s, it.kvh, it.rb, parts};
          kept = 1;
        }
        for (int tile = it.t0; tile < it.t1 && ok; ++tile) {
          if (!it.masked(tile)) continue;
          const uint32_t vslot = slot + 2 * (tile - it.t0) + 1, st = vslot % L::kStages;
          ok = bar_wait(&t.go[tidied % kTidyRing], (tidied / kTidyRing) & 1, abort);
          ok = __all_sync(kFull, ok);
          if (!ok) break;
          unsigned char* v = smem + L::kRing + st * L::kTileBytes;
          const int n = min(kTile, it.end - tile * kTile);
          uint32_t* bad = t.bad[tidied % kTidyRing];
          // a warp takes 64 of the tile's entries
          const int lo = (w >> 5) * 64, hi = lo + 64;
          if (lane < 2) bad[(lo >> 5) + lane] = 0;
          __syncwarp();
          // rows of the last instruction's 16 that hold no entry: a weight 0 times NaN is NaN
          const int z0 = max(n, lo), z1 = min((n + 15) & ~15, hi);
          for (int i = lane; i < (z1 - z0) * L::kHalves * 8; i += 32) {
            const int r = z0 + i / (L::kHalves * 8), c = i % (L::kHalves * 8);
            *reinterpret_cast<uint4*>(v + (c / 8) * L::kHalfBytes + r * 128 + (c % 8) * 16) = make_uint4(0, 0, 0, 0);
          }
          // entries that some rows do not see must be finite for those; the rows that see an entry
          // that is not get NaN from the softmax
          if (!it.alike) {
            constexpr uint32_t kExp = T::kNegInfWord & 0x7fff7fffu;
            const int r0 = max(lo, it.common - tile * kTile), r1 = min(n, hi);
            for (int i = lane; i < (r1 - r0) * L::kHalves * 8; i += 32) {
              const int r = r0 + i / (L::kHalves * 8), c = i % (L::kHalves * 8);
              uint4* at = reinterpret_cast<uint4*>(v + (c / 8) * L::kHalfBytes + r * 128 + (c % 8) * 16);
              const uint4 x = *at;
              auto inf = [](uint32_t y) {
                y &= kExp;
                return (y & 0xffffu) == (kExp & 0xffffu) || (y >> 16) == (kExp >> 16);
              };
              if (inf(x.x) || inf(x.y) || inf(x.z) || inf(x.w)) {
                *at = make_uint4(0, 0, 0, 0);
                atomicOr(&bad[r >> 5], 1u << (r & 31));
              }
            }
          }
          __syncwarp();
          fence_async();
          bar_arrive(&t.tidy[tidied % kTidyRing]);
          ++tidied;
        }
        slot += 2 * (it.t1 - it.t0);
      }
      if (w == 0 && !kept) p.meta[blockIdx.x] = Meta{0, 0, 0, 0};
    }
  } else {
    // ---- softmax and epilogue: one thread a row
    asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
    const int st = warp >> 2;                 // stream: a row tile, or the even / odd tiles
    const int r_tile = tid & 127;
    const uint32_t lanes = static_cast<uint32_t>(warp & 3) << 21;  // first tensor-memory row of the warp
    const uint32_t s_addr = tmem + lanes + st * kTile;
    const uint32_t o_addr = tmem + lanes + 2 * kTile + st * kTile;
    const float sl = a.scale * kLog2e;
    uint32_t seen = 0, tidied = 0, others = 0;  // tiles of this stream, tidied tiles, joins so far
    bool ok = true;
    Walk walk(a.b, geo, a.c.n_kv_heads, t);
    Item it;
    while (ok && walk.next(it)) {
      const bool dual = it.dual();
      const Chunk& ch = walk.chunk;
      const int r = (dual ? st * kTile : 0) + r_tile;
      const bool valid = r < it.rows;
      const int64_t row = static_cast<int64_t>(it.rb) * 2 * kTile + (valid ? r : 0);
      const int i = static_cast<int>(row / geo.group);
      // what the row sees: entries before `free`, and the nodes of its mask
      const bool node = i >= ch.lead;
      const int free_end = node ? ch.base + ch.lead : ch.base + i + 1;
      uint64_t m0 = 0, m1 = 0;
      if (node) {
        const uint64_t* words = a.b.node_mask + (static_cast<int64_t>(it.s) * a.b.g + (i - ch.lead)) * a.b.W;
        m0 = words[0];
        if (a.b.W > 1) m1 = words[1];
        if (ch.nodes < 64) m0 &= (1ull << ch.nodes) - 1;
        if (ch.nodes <= 64) m1 = 0;
        else if (ch.nodes < 128) m1 &= (1ull << (ch.nodes - 64)) - 1;
      }
      const int nt = it.t1 - it.t0;
      const int step = dual ? 1 : 2, j0 = dual ? 0 : st;
      int first_masked = it.common / kTile;  // tile numbers from here on are masked
      if (first_masked < it.t0) first_masked = it.t0;
      float m = -INFINITY, l = 0.f;
      for (int j = j0; j < nt && ok; j += step) {
        const int tile = it.t0 + j;
        ok = bar_wait(&t.s_ready[st], seen & 1, abort);
        ok = __all_sync(kFull, ok);
        if (!ok) break;
        tc_after();
        uint32_t x[4][32];
#pragma unroll
        for (int c = 0; c < 4; ++c) tm_ld32(x[c], s_addr + c * 32);
        tm_wait_ld(x[0]);
#pragma unroll
        for (int c = 1; c < 4; ++c) tm_after_wait(x[c]);
        if (it.masked(tile)) {
          const uint32_t no = tidied + (tile - first_masked);
          ok = bar_wait(&t.tidy[no % kTidyRing], (no / kTidyRing) & 1, abort);
          ok = __all_sync(kFull, ok);
          if (!ok) break;
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const int e0 = tile * kTile + c * 32;
            const int before = free_end - e0;  // visible entries at the start of these 32
            uint32_t see;
            if (before >= 32) {
              see = 0xffffffffu;
            } else {
              see = before > 0 ? (1u << before) - 1 : 0u;
              if (node) {
                // bits of the mask from node e0 - free_end on
                const int sh = -before;
                uint64_t bits;
                if (sh <= 0) bits = m0 << -sh;
                else if (sh < 64) bits = (m0 >> sh) | (sh ? m1 << (64 - sh) : 0);
                else bits = sh < 128 ? m1 >> (sh - 64) : 0;
                see |= static_cast<uint32_t>(bits);
              }
            }
            const uint32_t nan = t.bad[no % kTidyRing][c];
#pragma unroll
            for (int q = 0; q < 32; ++q) {
              if (!(see >> q & 1)) x[c][q] = 0xff800000u;
              else if (nan >> q & 1) x[c][q] = 0x7fffffffu;
            }
          }
        }
        float top = -INFINITY;
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
          for (int q = 0; q < 32; ++q) top = fmaxf(top, __uint_as_float(x[c][q]));
        top *= sl;
        if (j == j0) {
          m = top;
        } else {
          const bool rise = valid && top > m + kLazy;
          if (__any_sync(kFull, rise)) {
            ok = bar_wait(&t.pv_done[st], (seen - 1) & 1, abort);  // the output so far is complete
            ok = __all_sync(kFull, ok);
            if (!ok) break;
            tc_after();
            const float m_new = rise ? top : m;
            const float fix = rise ? ex2_approx(m - m_new) : 1.f;
            m = m_new;
            l *= fix;
#pragma unroll
            for (int c = 0; c < DH / 32; ++c) {
              uint32_t o[32];
              tm_ld32(o, o_addr + c * 32);
              tm_wait_ld(o);
#pragma unroll
              for (int q = 0; q < 32; ++q) o[q] = __float_as_uint(__uint_as_float(o[q]) * fix);
              tm_st32(o_addr + c * 32, o);
            }
          }
        }
        __syncwarp();
        const float ref = m == -INFINITY ? 0.f : m;
        float sum0 = 0.f, sum1 = 0.f;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          uint32_t w[16];
#pragma unroll
          for (int q = 0; q < 16; ++q) {
            const float p0 = ex2_approx(fmaf(__uint_as_float(x[c][2 * q]), sl, -ref));
            const float p1 = ex2_approx(fmaf(__uint_as_float(x[c][2 * q + 1]), sl, -ref));
            sum0 += p0;
            sum1 += p1;
            w[q] = pack2<T>(p0, p1);
          }
          tm_st16(s_addr + c * 16, w);
        }
        l += sum0 + sum1;
        tm_wait_st();
        tc_before();
        __syncwarp();
        if (lane == 0) bar_arrive(&t.p_ready[st]);
        ++seen;
      }
      if (it.t1 > first_masked) tidied += it.t1 - first_masked;
      if (!ok) break;
      // ---- epilogue
      const bool mine = nt > j0;  // this stream had tiles
      if (mine) {
        ok = bar_wait(&t.pv_done[st], (seen - 1) & 1, abort);
        ok = __all_sync(kFull, ok);
        if (!ok) break;
        tc_after();
      }
      const bool join = !dual && nt > 1;
      float w0 = 1.f, w1 = 0.f;
      if (join) {
        if (st == 1) {
          t.ml[r_tile][0] = m;
          t.ml[r_tile][1] = l;
          tc_before();
          __syncwarp();
          if (lane == 0) bar_arrive(&t.other);
          continue;
        }
        ok = bar_wait(&t.other, others & 1, abort);
        ok = __all_sync(kFull, ok);
        if (!ok) break;
        ++others;
        tc_after();
        const float mo = t.ml[r_tile][0], lo = t.ml[r_tile][1];
        const float mm = fmaxf(m, mo);
        const float ref = mm == -INFINITY ? 0.f : mm;
        w0 = ex2_approx(m - ref);
        w1 = ex2_approx(mo - ref);
        l = l * w0 + lo * w1;
        m = mm;
      } else if (!mine) {
        continue;
      }
      const bool whole = it.whole();
      const int64_t tok = ch.q0 + i;
      const int h = it.kvh * geo.group + static_cast<int>(row % geo.group);
      const float inv = l > 0.f ? 1.f / l : (l == 0.f ? 0.f : NAN);
      const int64_t slot = 2 * static_cast<int64_t>(blockIdx.x) + (it.t0 == 0 ? 1 : 0);
#pragma unroll
      for (int c = 0; c < DH / 32; ++c) {
        uint32_t o[32];
        __syncwarp();
        tm_ld32(o, o_addr + c * 32);
        tm_wait_ld(o);
        if (join) {
          uint32_t y[32];
          tm_ld32(y, o_addr + kTile + c * 32);
          tm_wait_ld(y);
#pragma unroll
          for (int q = 0; q < 32; ++q)
            o[q] = __float_as_uint(__uint_as_float(o[q]) * w0 + __uint_as_float(y[q]) * w1);
        }
        if (c == DH / 32 - 1) {  // the accumulators are free for the next block
          tc_before();
          __syncwarp();
          if (lane == 0) {
            bar_arrive(&t.o_free[st]);
            if (join) bar_arrive(&t.o_free[1]);
          }
        }
        if (!valid) continue;
        if (whole) {
          uint4* out = reinterpret_cast<uint4*>(a.out + (tok * a.n_q_heads + h) * static_cast<int64_t>(DH * 2) + c * 64);
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            uint4 y;
            y.x = pack2<T>(__uint_as_float(o[8 * q]) * inv, __uint_as_float(o[8 * q + 1]) * inv);
            y.y = pack2<T>(__uint_as_float(o[8 * q + 2]) * inv, __uint_as_float(o[8 * q + 3]) * inv);
            y.z = pack2<T>(__uint_as_float(o[8 * q + 4]) * inv, __uint_as_float(o[8 * q + 5]) * inv);
            y.w = pack2<T>(__uint_as_float(o[8 * q + 6]) * inv, __uint_as_float(o[8 * q + 7]) * inv);
            out[q] = y;
          }
        } else {
          float4* out = p.part + (slot * (DH / 4) + c * 8) * (2 * kTile) + r;
#pragma unroll
          for (int q = 0; q < 8; ++q)
            out[q * 2 * kTile] = make_float4(__uint_as_float(o[4 * q]), __uint_as_float(o[4 * q + 1]),
                                             __uint_as_float(o[4 * q + 2]), __uint_as_float(o[4 * q + 3]));
        }
      }
      if (valid) {
        if (!whole) p.part_ml[slot * 2 * kTile + r] = make_float2(m, l);
        else if (a.lse != nullptr)
          a.lse[tok * a.n_q_heads + h] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
      }
    }
  }
  tc_before();
  __syncthreads();
  tc_after();
  if (warp == 9)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
  if (tid == 0 && t.abort) atomicOr(a.b.status, kStatusTimeout);
}

// Joins the parts of blocks that were cut: grid (CTAs of the first kernel, 32 rows each).
constexpr int kJoinThreads = 256;

template <typename T, int DH>
__global__ void __launch_bounds__(kJoinThreads) attention_join_kernel(const __grid_constant__ TcArgs p) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const Meta meta = p.meta[blockIdx.x];
  if (meta.parts == 0) return;
  const AttnArgs& a = p.a;
  const Geometry geo{a.n_q_heads / a.c.n_kv_heads};
  const Chunk ch = load_chunk(a.b, meta.s);
  const int rows = geo.rows(ch, meta.rb);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int r = blockIdx.y * 32 + lane;
  if (blockIdx.y * 32 >= rows) return;
  const bool valid = r < rows;
  const int64_t first = 2 * static_cast<int64_t>(blockIdx.x);
  auto slot = [first](int i) { return i == 0 ? first + 1 : first + 2 * i; };
  float m = -INFINITY;
  for (int i = 0; i < meta.parts; ++i) m = fmaxf(m, valid ? p.part_ml[slot(i) * 2 * kTile + r].x : -INFINITY);
  const float ref = m == -INFINITY ? 0.f : m;
  float l = 0.f;
  constexpr int kMine = DH / 4 / (kJoinThreads / 32);  // groups of four columns of a warp
  float4 o[kMine];
#pragma unroll
  for (int c = 0; c < kMine; ++c) o[c] = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int i = 0; i < meta.parts; ++i) {
    if (!valid) continue;
    const float2 ml = p.part_ml[slot(i) * 2 * kTile + r];
    const float w = ex2_approx(ml.x - ref);
    l = fmaf(ml.y, w, l);
#pragma unroll
    for (int c = 0; c < kMine; ++c) {
      const float4 y = p.part[(slot(i) * (DH / 4) + warp * kMine + c) * 2 * kTile + r];
      o[c].x = fmaf(y.x, w, o[c].x);
      o[c].y = fmaf(y.y, w, o[c].y);
      o[c].z = fmaf(y.z, w, o[c].z);
      o[c].w = fmaf(y.w, w, o[c].w);
    }
  }
  if (!valid) return;
  const float inv = l > 0.f ? 1.f / l : (l == 0.f ? 0.f : NAN);
  const int64_t row = static_cast<int64_t>(meta.rb) * 2 * kTile + r;
  const int64_t tok = ch.q0 + row / geo.group;
  const int h = meta.kvh * geo.group + static_cast<int>(row % geo.group);
  uint2* out = reinterpret_cast<uint2*>(a.out + (tok * a.n_q_heads + h) * static_cast<int64_t>(DH * 2)) + warp * kMine;
#pragma unroll
  for (int c = 0; c < kMine; ++c) {
    uint2 y;
    y.x = pack2<T>(o[c].x * inv, o[c].y * inv);
    y.y = pack2<T>(o[c].z * inv, o[c].w * inv);
    out[c] = y;
  }
  if (warp == 0 && a.lse != nullptr)
    a.lse[tok * a.n_q_heads + h] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
}

typedef CUresult (*EncodeFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                             const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                             CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeFn encode_fn() {
  static const EncodeFn fn = [] {
    void* f = nullptr;
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &f, cudaEnableDefault, &found) != cudaSuccess ||
        found != cudaDriverEntryPointSuccess)
      f = nullptr;
    return reinterpret_cast<EncodeFn>(f);
  }();
  return fn;
}

bool make_map(CUtensorMap* map, const AttnArgs& a, bool value, int box_rows) {
  const CacheArgs& c = a.c;
  const cuuint64_t dims[4] = {static_cast<cuuint64_t>(c.head_dim), static_cast<cuuint64_t>(c.n_kv_heads),
                              static_cast<cuuint64_t>(a.b.page_size), static_cast<cuuint64_t>(a.b.n_pages)};
  const cuuint64_t strides[3] = {static_cast<cuuint64_t>(value ? c.v_head : c.k_head),
                                 static_cast<cuuint64_t>(value ? c.v_entry : c.k_entry),
                                 static_cast<cuuint64_t>(value ? c.v_page : c.k_page)};
  const cuuint32_t box[4] = {64, 1, static_cast<cuuint32_t>(box_rows), 1};
  const cuuint32_t one[4] = {1, 1, 1, 1};
  return encode_fn()(map, c.dtype == GTO_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 4,
                     value ? c.v : c.k, dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
                     CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                     CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

size_t align_up(size_t x) { return (x + 255) & ~static_cast<size_t>(255); }

template <typename T, int DH>
cudaError_t tc_as(const TcArgs& p, int sms, cudaStream_t stream, int64_t* launches) {
  CUtensorMap km, vm;
  if (!make_map(&km, p.a, false, p.box_rows) || !make_map(&vm, p.a, true, p.box_rows)) return cudaErrorInvalidValue;
  const size_t smem = Layout<DH>::kTail + sizeof(Tail) + 1024;
  static_assert(Layout<DH>::kTail + sizeof(Tail) + 1024 <= 232448, "shared memory of an SM");
  cudaError_t e = cudaFuncSetAttribute(attention_tc_kernel<T, DH>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                       static_cast<int>(smem));
  if (e != cudaSuccess) return e;
  attention_tc_kernel<T, DH><<<sms, kThreads, smem, stream>>>(p, km, vm);
  ++*launches;
  e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(sms, 2 * kTile / 32);
  cfg.blockDim = dim3(kJoinThreads);
  cfg.stream = stream;
  cudaLaunchAttribute attr{};
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  ++*launches;
  return cudaLaunchKernelEx(&cfg, attention_join_kernel<T, DH>, p);
}

}  // namespace

bool attention_tc_serves(const gto_decode_config& c) {
  return (c.kv_dtype == GTO_BF16 || c.kv_dtype == GTO_F16) && (c.head_dim == 64 || c.head_dim == 128) &&
         c.page_size % 8 == 0 && encode_fn() != nullptr;
}

size_t attention_tc_workspace(const gto_decode_config& c, int sms) {
  const size_t slots = 2 * static_cast<size_t>(sms);
  return align_up(sizeof(Meta) * sms) + align_up(slots * 2 * kTile * sizeof(float2)) +
         slots * 2 * kTile * c.head_dim * sizeof(float);
}

cudaError_t launch_attention_tc(const AttnArgs& a, void* workspace, int sms, cudaStream_t stream, int64_t* launches) {
  TcArgs p{};
  p.a = a;
  char* ws = static_cast<char*>(workspace);
  p.meta = reinterpret_cast<Meta*>(ws);
  ws += align_up(sizeof(Meta) * sms);
  p.part_ml = reinterpret_cast<float2*>(ws);
  ws += align_up(2 * static_cast<size_t>(sms) * 2 * kTile * sizeof(float2));
  p.part = reinterpret_cast<float4*>(ws);
  p.box_rows = 8;
  while (p.box_rows < kTile && a.b.page_size % (2 * p.box_rows) == 0) p.box_rows *= 2;
  p.boxes = kTile / p.box_rows;
  if (a.c.dtype == GTO_BF16)
    return a.c.head_dim == 128 ? tc_as<Bf16, 128>(p, sms, stream, launches) : tc_as<Bf16, 64>(p, sms, stream, launches);
  return a.c.head_dim == 128 ? tc_as<F16, 128>(p, sms, stream, launches) : tc_as<F16, 64>(p, sms, stream, launches);
}

}  // namespace gto
