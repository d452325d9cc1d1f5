// gto_tree_attention on the tensor cores: 16-bit tensors, heads of 64 or 128, pages of a multiple of 8.
//
// Rows.  A query row is one token and one of the query heads that share a key head; the rows of a
// chunk and key head are cut into blocks of 256, two tiles of 128 (the M of the matrix
// instruction), so that a tile of keys and values read once serves up to 256 rows.  With 128 rows
// or fewer (single tokens, small trees) the two streams of the CTA take the even and the odd tiles
// of the same rows instead and join at the end, which halves the dependent chain product -> softmax
// -> product that a tile costs.
//
// Work.  A block of rows costs one unit for each 64 cache entries that it sees, plus kOverhead.
// All units of the call, in the order (sequence, key head, block, entries), are cut into as
// many equal spans as there are SMs; every CTA takes one.  A block that a cut goes through leaves
// its unnormalised parts in the workspace and a second, small kernel joins them in the order of
// the entries.  The lengths are read on the device; the cut depends on nothing else, so that equal
// calls give equal bits.
//
// A CTA is 12 warps.  Eight do the softmax and the epilogue, four for each of two streams, one thread a
// row.  One copies keys, one values and queries (TMA boxes out of the pages, into a ring of stages
// each: keys are free for the next tile long before the values are).  Two issue the matrix
// instructions, one a stream, so that one waits while the other issues.  Tensor memory holds for each
// stream two buffers of scores (64 columns; the weights take the first 32 of theirs) and the output
// (128): a stream's scores lie ready, two tiles ahead of its products with the values, when a softmax ends.
//
// Rounding.  Scores, maxima, sums and outputs are fp32; the weights are rounded to the 16-bit type
// to be an operand of the second product (half a step each), while their sum is taken before that
// rounding.  A row's weights are 2^(score - reference).  The reference follows the row's maximum only
// when that has risen by more than kLazy in log2 units, so that most tiles need no rescaling of the
// output.  bf16 has fp32's exponents.  fp16 has normal numbers from 2^-14 to 2^16 only: its reference lies
// kRaise below the maximum, weights go up to 2^(kRaise + kLazy) = 2^15, and those down to 2^-25 of the
// row's largest keep the half step (a long flat tail behind one large score is made of such weights);
// what is below 2^-36 of it is lost.  Scores of 2^20 and more, where fp32 knows the exponent to a tenth only,
// have their reference at the maximum: the weight of a rounding more must not pass 2^16.
//
// What bounds it (32 query heads, 8 key heads of 128; B200 at 1.7 to 1.97 GHz).  Single tokens: the copies;
// 128 sequences of 1500 to 6000 entries take 340 to 370 us by the board, 5.4 to 5.8 TB/s (83 to 90 % of the
// copy rate; the clock falls to 1.5 to 1.6 GHz).  Trees and prompts: a step of 64
// entries on 256 rows takes 2240 to 2460 cycles, where the matrix instructions need 1280 (a score
// product of N = 64 reads 6 KB of operands from shared memory in 48 cycles, which is all that it
// gives, in place of the 32 that the product would need) and the exponentials 1024: a stream's own
// chain (scores to registers and their maximum 500, exponentials 1180 where two warps of a scheduler
// have them at once, waits and hand-overs 700) is longer than either.  32 trees of 61 tokens on 1000 to 4000
// entries take 125 to 131 us, four prompts of up to 2048 tokens on up to 6000 cached ones 364 to 376 us
// (810 to 840 TFLOP/s of the products that are not masked).  One token of one sequence on 8000 entries takes
// 20.2 us: 3 until the span is known, 10 for the tiles, 6 for the join.
// Measured and slower: scores of 128 entries in one product (144 and 415 us: no second buffer), 16 warps for
// the softmax (152, 424), next scores into registers during the exponentials (149), a part of the
// exponentials as a polynomial (no gain), one warp for all matrix instructions (158).
#include <cuda.h>

#include "decode_common.cuh"

namespace gto {
namespace {

constexpr int kThreads = 384;
constexpr int kRows = 128;       // rows of a row tile (M of the matrix instruction)
constexpr int kBlock = 2 * kRows;
constexpr int kTile = 64;        // cache entries of a tile
// Cost of a block beside its tiles (queries, first scores, epilogue), in tiles.  Measured with 2, 4, 6, 8, 12: one
// token on 8000 entries 20.8, 20.2, 20.0, 19.9, 19.9 us, 32 trees 136, 134, 131, 131, 133, prompts 384, 382, 376, 379, 380.
constexpr int kOverhead = 6;
constexpr int kGoRing = 16;      // more than the value tiles that their ring can hold
// A block of no more rows is copied row by row and the rest of its tile stays zeros; a box brings the rows of other
// tokens, whose products nobody asks for but which draw power.  On long caches that lowers the clock: 128 sequences of
// one token on 5000 entries 421 us, by boxes 448; of two tokens (8 rows) 467 and 505; 64 of four on 8000 entries 381 and 400.
// On short ones a box saves the copy's latency: 64 of one token on 700 entries 73.1 and 72.1.  From 36 rows on
// boxes are no slower on either (12 tokens: 70.3 us against 70.8 row by row).
constexpr int kFewRows = 32;
// log2 units the maximum may rise before the output is rescaled, and by which the reference lies below it
template <typename T>
constexpr float kLazy = T::kNegInfElem == 0xff80u ? 8.0f : 4.0f;
template <typename T>
constexpr float kRaise = T::kNegInfElem == 0xff80u ? 0.0f : 11.0f;
constexpr uint32_t kWaitTries = 20000;  // of a tenth of a millisecond

template <int DH>
struct Layout {
  static constexpr int kTileBytes = kTile * DH * 2;    // keys or values
  static constexpr int kHalves = DH / 64;              // 128-byte columns
  static constexpr int kHalfBytes = kTile * 128;
  static constexpr int kQBytes = kRows * DH * 2;       // a row tile of queries
  static constexpr int kQHalfBytes = kRows * 128;
  static constexpr int kStages = DH == 128 ? 5 : 8;    // of the ring of keys, and of that of values
  static constexpr int kQ = 0;
  static constexpr int kKeys = 2 * kQBytes;
  static constexpr int kValues = kKeys + kStages * kTileBytes;
  static constexpr int kTail = kValues + kStages * kTileBytes;
};

// Tensor memory, columns: scores [stream][buffer][64], the weights take the first 32 of theirs;
// outputs [stream][DH].
constexpr uint32_t kOutCol = 256;
__device__ __forceinline__ constexpr uint32_t score_col(uint32_t st, uint32_t buf) { return (st * 2 + buf) * kTile; }

struct Tail {
  uint64_t full[2][8], empty[2][8];   // rings of keys and of values
  uint64_t q_full, q_empty, other;
  uint64_t s_ready[2][2], p_ready[2][2], pv_done[2][2];  // [stream][buffer]
  uint64_t o_free[2];
  // a value tile at the end of what its rows see: `go` says that it is loaded, `full` of its stage
  // only that it was issued (the product waits for the weights, which wait for `go`)
  uint64_t go[kGoRing];
  uint64_t scanned_both, scanned[2];
  float ml[kRows][2];           // reference and sum of the odd tiles' rows
  int64_t scan[kThreads / 32];
  int64_t span, each, extra;    // this CTA's units; units of a CTA, CTAs that have one more
  int64_t off;                  // where the span begins: in block (seq, kvh, rb)
  int seq, kvh, rb;
  Chunk chunk;                  // of that sequence
  uint32_t tmem;
  int abort;
  uint32_t lost[8];             // softmax warps: rows (lanes) that see a value that is not finite
};

// ------------------------------------------------------------------ instructions
__device__ __forceinline__ uint32_t smem_u32(const void* p) {
  return static_cast<uint32_t>(__cvta_generic_to_shared(p));
}
// Barriers are named by their shared-memory address.
__device__ __forceinline__ void bar_init(uint32_t b, int count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(b), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint32_t b) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(b) : "memory");
}
__device__ __forceinline__ void bar_expect(uint32_t b, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(b), "r"(bytes) : "memory");
}
// Waits until the phase of that parity has completed: kWaitTries times asleep for at most a
// tenth of a millisecond.  False if it has not.
__device__ __forceinline__ bool bar_try(uint32_t b, uint32_t parity, uint32_t tries) {
  uint32_t ok;
  asm volatile(
      "{\n .reg .pred p, q;\n .reg .u32 n;\n mov.u32 n, 0;\n"
      "WAIT:\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, 100000;\n @p bra DONE;\n"
      " add.u32 n, n, 1;\n setp.lt.u32 q, n, %3;\n @q bra WAIT;\n"
      "DONE:\n selp.u32 %0, 1, 0, p;\n}"
      : "=r"(ok)
      : "r"(b), "r"(parity), "r"(tries)
      : "memory");
  return ok != 0;
}
// The same for all roles of the kernel: false also soon after another warp has given up.
__device__ __forceinline__ bool bar_wait(uint32_t b, uint32_t parity, volatile int* abort) {
  if (bar_try(b, parity, 1)) return true;
  for (uint32_t i = 0; i < kWaitTries / 16; ++i) {
    if (bar_try(b, parity, 16)) return true;
    if (*abort) return false;
  }
  *abort = 1;
  return false;
}
__device__ __forceinline__ void fence_async() {
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
}
__device__ __forceinline__ void tc_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// The instructions below are executed by a whole warp and take effect in its leader: with all
// control flow uniform the descriptors stay in uniform registers, and one product costs the issuing
// warp a few instructions (under a branch on the lane it cost 110 to 150 cycles, more than the
// 64 that the product itself takes).
__device__ __forceinline__ uint32_t elect() {
  uint32_t e;
  asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.u32 %0, 1, 0, p;\n}" : "=r"(e));
  return e;
}
__device__ __forceinline__ void tc_commit(uint32_t b, uint32_t leader) {
  asm volatile(
      "{\n .reg .pred e;\n setp.ne.b32 e, %1, 0;\n"
      " @e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n}" ::"r"(b), "r"(leader)
      : "memory");
}
// d (+)= a b: operands as the low words of their descriptors, the high word is the same for all
__device__ __forceinline__ void mma_ss(uint32_t d, uint32_t a, uint32_t b, uint32_t hi, uint32_t idesc, uint32_t acc,
                                       uint32_t leader) {
  asm volatile(
      "{\n .reg .pred p, e;\n .reg .b64 x, y;\n setp.ne.b32 p, %5, 0;\n setp.ne.b32 e, %6, 0;\n"
      " mov.b64 x, {%1, %3};\n mov.b64 y, {%2, %3};\n"
      " @e tcgen05.mma.cta_group::1.kind::f16 [%0], x, y, %4, p;\n}" ::"r"(d), "r"(a), "r"(b), "r"(hi), "r"(idesc),
      "r"(acc), "r"(leader)
      : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint32_t b, uint32_t hi, uint32_t idesc, uint32_t acc,
                                       uint32_t leader) {
  asm volatile(
      "{\n .reg .pred p, e;\n .reg .b64 y;\n setp.ne.b32 p, %5, 0;\n setp.ne.b32 e, %6, 0;\n"
      " mov.b64 y, {%2, %3};\n"
      " @e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], y, %4, p;\n}" ::"r"(d), "r"(a), "r"(b), "r"(hi), "r"(idesc),
      "r"(acc), "r"(leader)
      : "memory");
}
__device__ __forceinline__ void tma_3d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(
          dst),
      "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
      : "memory");
}
__device__ __forceinline__ void tma_4d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, int w,
                                       uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], "
      "[%6];" ::"r"(dst),
      "l"(map), "r"(x), "r"(y), "r"(z), "r"(w), "r"(bar)
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

// Shared-memory operand, 128-byte swizzle.  Low word: start and leading byte offset over 16; high
// word: stride byte offset over 16 (eight rows of 128 bytes), the version bit of this generation,
// swizzle mode 2.
constexpr uint32_t kDescHi = (1024u >> 4) | (1u << 14) | (2u << 29);
__device__ __forceinline__ uint32_t desc_lo(uint32_t addr, uint32_t leading) {
  return ((addr >> 4) & 0x3fffu) | ((leading >> 4) << 16);
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

// ---- two fp32 values in one instruction
__device__ __forceinline__ uint64_t pair(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void unpair(uint64_t r, float& a, float& b) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(r));
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
// ------------------------------------------------------------------ work
// Rows of a call fit 30 bits (checked when the context is made).
struct Geometry {
  int group;  // query heads of a key head
  __device__ __forceinline__ int blocks(const Chunk& c) const {
    return c.ok ? (c.n * group + kBlock - 1) / (kBlock) : 0;
  }
  __device__ __forceinline__ int rows(const Chunk& c, int rb) const {
    return min(c.n * group - rb * kBlock, kBlock);
  }
  __device__ __forceinline__ int last_token(const Chunk& c, int rb) const {
    return (rb * kBlock + rows(c, rb) - 1) / group;
  }
  __device__ __forceinline__ int tiles(const Chunk& c, int rb) const {
    return (kv_end(c, last_token(c, rb)) + kTile - 1) / kTile;
  }
};

struct Item {
  int s, kvh, rb, rows;
  int t0, t1, n;       // tiles [t0, t1) of n
  int first;           // first token of the block
  int end;             // entries that any row of the block sees
  int common;          // entries that every row sees
  bool alike;          // all rows see the same entries
  int after;           // units of the block that later CTAs do
  __device__ __forceinline__ bool whole() const { return t0 == 0 && t1 == n; }
  __device__ __forceinline__ bool dual() const { return rows > kRows; }
  __device__ __forceinline__ bool masked(int t) const { return (t + 1) * kTile > common; }
};

// Goes through the blocks of a CTA's span; every role of the CTA does so by itself.
struct Walk {
  const BatchArgs& b;
  Geometry g;
  int heads;
  int s, kvh, rb, nrb, off;
  int64_t left;
  Chunk c;
  Chunk chunk;  // of the item that next() gave

  __device__ __forceinline__ Walk(const BatchArgs& batch, Geometry geo, int n_kv_heads, const Tail& t)
      : b(batch), g(geo), heads(n_kv_heads), s(t.seq), kvh(t.kvh), rb(t.rb), nrb(0),
        off(static_cast<int>(t.off)), left(t.span) {
    if (left <= 0) return;
    c = t.chunk;
    nrb = g.blocks(c);
  }
  __device__ bool next(Item& it) {
    while (left > 0 && s < b.S) {
      it.rows = g.rows(c, rb);
      it.first = rb * kBlock / g.group;
      const int last = (rb * kBlock + it.rows - 1) / g.group;
      it.end = kv_end(c, last);
      it.n = (it.end + kTile - 1) / kTile;
      const int u = it.n + kOverhead - off;  // units of the block from here on
      const int take = left < u ? static_cast<int>(left) : u;
      it.s = s;
      it.kvh = kvh;
      it.rb = rb;
      it.t0 = max(off - kOverhead, 0);
      it.t1 = max(off + take - kOverhead, 0);
      it.common = it.first < c.lead ? c.base + it.first + 1 : c.base + c.lead;
      it.alike = it.first == last && it.first < c.lead;
      it.after = u - take;
      chunk = c;
      left -= take;
      off = 0;
      if (++rb == nrb) {
        rb = 0;
        if (++kvh == heads) {
          kvh = 0;
          nrb = 0;
          while (nrb == 0 && left > 0 && ++s < b.S) {
            c = load_chunk(b, s);
            nrb = g.blocks(c);
          }
        }
      }
      if (it.t1 > it.t0) return true;
    }
    return false;
  }
};

struct Meta {  // of a block whose first part a CTA did
  int64_t tok0;                   // its chunk's first token
  int32_t row0, rows, kvh, parts; // first of its rows in the chunk, ...; parts = 0: no such block
};

struct TcArgs {
  AttnArgs a;
  Meta* meta;
  float4* part;   // [slot][DH/4][256]
  float2* part_ml;  // [slot][256]
  int box_rows;   // entries of a TMA box
  int box_shift;  // log2 of the boxes that make up a tile's rows
  int page_shift; // log2 of the page size, -1 where it is no power of two
  int q_tokens;   // tokens of a row tile where the query heads of a key head divide 128, else 0
  uint32_t group_magic;  // ceil(2^16 / group): x / group = x * group_magic >> 16 for x < 512
};

// Every thread of the CTA: units of the call, this CTA's span and where it begins.
__device__ __forceinline__ void plan(const BatchArgs& b, Geometry g, int heads, Tail& t) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  // a thread owns a run of sequences
  const int per = (b.S + kThreads - 1) / kThreads;
  const int s0 = min(tid * per, b.S), s1 = min(s0 + per, b.S);
  auto units_of = [&](const Chunk& c) {  // of one key head
    const int nrb = g.blocks(c);
    int64_t u = 0;
    for (int i = 0; i < nrb; ++i) u += g.tiles(c, i) + kOverhead;
    return u;
  };
  int64_t mine, run;
  Chunk head{};  // of the run's first sequence
  for (int seqs = b.S;;) {  // once, or again without the sequences from the first decrease of q_start on
    int fall = seqs;
    mine = 0;
    for (int s = s0; s < min(s1, seqs); ++s) {
      const Chunk c = load_chunk(b, s);
      if (s == s0) head = c;
      if (!c.ok && blockIdx.x == 0) atomicOr(b.status, kStatusBadIndex);
      if (!c.ok && falls(b, s)) fall = min(fall, s);
      mine += units_of(c) * heads;
    }
    run = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t y = __shfl_up_sync(kFull, run, o);
      if (lane >= o) run += y;
    }
    if (lane == 31) t.scan[warp] = run;
    if (tid == 0) {
      t.span = 0;
      t.seq = seqs;
    }
    if (!__syncthreads_or(fall < seqs)) break;
    atomicMin(&t.seq, fall);
    __syncthreads();
    seqs = t.seq;
    __syncthreads();  // (read by all before it is written again)
  }
  int64_t units = 0;
  for (int w = 0; w < kThreads / 32; ++w) {
    if (w < warp) run += t.scan[w];
    units += t.scan[w];
  }
  // CTA c takes `each` units, the first `extra` CTAs one more
  const uint32_t ctas = gridDim.x, cta = blockIdx.x;
  const int64_t each = units >> 32 ? units / ctas : static_cast<uint32_t>(units) / ctas;
  const int64_t extra = units - each * ctas;
  const int64_t from = each * cta + min(static_cast<int64_t>(cta), extra), span = each + (cta < extra ? 1 : 0);
  const int64_t begin = run - mine;
  if (span > 0 && from >= begin && from < run) {
    int64_t off = from - begin;
    for (int s = s0; s < s1; ++s) {
      const Chunk c = s == s0 ? head : load_chunk(b, s);
      const int64_t u = units_of(c);
      if (off >= u * heads) {
        off -= u * heads;
        continue;
      }
      int kvh = 0, rb = 0;
      if (off >= u) {
        kvh = static_cast<int>(off >> 32 ? off / u : static_cast<uint32_t>(off) / static_cast<uint32_t>(u));
        off -= u * kvh;
      }
      for (int n = g.tiles(c, 0) + kOverhead; off >= n; n = g.tiles(c, ++rb) + kOverhead) off -= n;
      t.seq = s;
      t.chunk = c;
      t.kvh = kvh;
      t.rb = rb;
      t.off = off;
      t.span = span;
      t.each = each;
      t.extra = extra;
      break;
    }
  }
  __syncthreads();
}

// ------------------------------------------------------------------ the kernel
template <typename T, int DH>
__global__ void __launch_bounds__(kThreads, 1)
    attention_tc_kernel(const __grid_constant__ TcArgs p, const __grid_constant__ CUtensorMap k_map,
                        const __grid_constant__ CUtensorMap v_map, const __grid_constant__ CUtensorMap q_map) {
  using L = Layout<DH>;
  extern __shared__ unsigned char s_dyn[];
  unsigned char* smem = s_dyn + ((1024u - (smem_u32(s_dyn) & 1023u)) & 1023u);
  Tail& t = *reinterpret_cast<Tail*>(smem + L::kTail);
  const uint32_t q_base = smem_u32(smem + L::kQ), keys = smem_u32(smem + L::kKeys), values = smem_u32(smem + L::kValues);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const AttnArgs& a = p.a;
  const Geometry geo{a.n_q_heads / a.c.n_kv_heads};
  volatile int* abort = &t.abort;
  const uint32_t tail = q_base + L::kTail;
#define GTO_BAR(member) (tail + static_cast<uint32_t>(offsetof(Tail, member)))

  if (tid == 0) {
    for (int i = 0; i < 16; ++i) {
      bar_init(GTO_BAR(full) + i * 8, 1);
      bar_init(GTO_BAR(empty) + i * 8, 2);
    }
    bar_init(GTO_BAR(q_full), 32);
    bar_init(GTO_BAR(q_empty), 2);
    bar_init(GTO_BAR(other), 4);
    for (int i = 0; i < 2; ++i) {
      for (int b = 0; b < 2; ++b) {
        bar_init(GTO_BAR(s_ready) + ((i) * 2 + (b)) * 8, 1);
        bar_init(GTO_BAR(p_ready) + ((i) * 2 + (b)) * 8, 4);
        bar_init(GTO_BAR(pv_done) + ((i) * 2 + (b)) * 8, 1);
      }
      bar_init(GTO_BAR(o_free) + (i) * 8, 4);
      bar_init(GTO_BAR(scanned) + (i) * 8, 4);
    }
    bar_init(GTO_BAR(scanned_both), 8);
    for (int i = 0; i < kGoRing; ++i) bar_init(GTO_BAR(go) + (i) * 8, 1);
    t.abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  // Rows that a block does not have are zeros where it has few: a tile of 128 costs its time in the
  // tensor cores all the same, but less power.
  for (int i = tid; i < L::kQBytes / 16; i += kThreads) reinterpret_cast<uint4*>(smem + L::kQ)[i] = make_uint4(0, 0, 0, 0);
  fence_async();
  if (tid == 256) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(&k_map) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&v_map) : "memory");
    if (p.q_tokens) asm volatile("prefetch.tensormap [%0];" ::"l"(&q_map) : "memory");
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

  Walk walk(a.b, geo, a.c.n_kv_heads, t);
  Item it;
  if (warp == 8 || warp == 11) {
    // ---- a warp for the keys, one for the values and the queries: TMA boxes into their ring
    const bool value = warp == 11;
    const uint32_t full = GTO_BAR(full) + (value ? 64 : 0), empty = GTO_BAR(empty) + (value ? 64 : 0);
    uint32_t st = 0, phase = 1;  // a stage's first use waits for nothing
    uint32_t slot = 0, gone = 0, items = 0;
    bool kept = false;  // whether this CTA began a block that others end
    bool ok = true;
    const int half = lane >> p.box_shift, e_off = (lane & ((1 << p.box_shift) - 1)) * p.box_rows;
    const uint32_t my_dst = (value ? values : keys) + half * L::kHalfBytes + e_off * 128;
    const bool my_box = half < L::kHalves;
    while (ok && walk.next(it)) {
      if (value) {  // before a block's values, its queries
        if (items > 0) ok = bar_wait(GTO_BAR(q_empty), (items - 1) & 1, abort);
        ok = __all_sync(kFull, ok);
        if (!ok) break;
        ++items;
        const Chunk& ch = walk.chunk;
        if (p.q_tokens && it.rows > kFewRows) {
          // rows are tokens x heads in memory order: a box each for a row tile's halves (rows behind
          // the chunk's last bring what lies there, and nobody reads them)
          if (lane == 0) {
            const int tiles = it.dual() ? 2 : 1;
            bar_expect(GTO_BAR(q_full), tiles * L::kQBytes);
            for (int i = 0; i < tiles; ++i)
              for (int half = 0; half < L::kHalves; ++half)
                tma_3d(q_base + i * L::kQBytes + half * L::kQHalfBytes, &q_map, half * 64, it.kvh * geo.group,
                       ch.q0 + it.first + i * p.q_tokens, GTO_BAR(q_full));
          } else {
            bar_arrive(GTO_BAR(q_full));
          }
        } else {
          // a thread copies one 16-byte column of every second or fourth row
          constexpr int kCols = DH / 8, kStep = 32 / kCols;
          const int c = lane % kCols;
          const int h0 = it.rb * kBlock - it.first * geo.group;  // head of row 0 within its token
          const char* src0 = a.q + (static_cast<int64_t>(ch.q0) + it.first) * a.q_stride +
                             static_cast<int64_t>(it.kvh) * geo.group * (DH * 2) + c * 16;
          const uint32_t dst0 = q_base + (c / 8) * L::kQHalfBytes;
  #pragma unroll 4
          for (int r = lane / kCols; r < it.rows; r += kStep) {
            const uint32_t x = h0 + r, i = x * p.group_magic >> 16;
            const char* src = src0 + i * a.q_stride + (x - i * geo.group) * (DH * 2);
            const uint32_t dst = dst0 + (r >> 7) * L::kQBytes + (r & 127) * 128 + (((c & 7) ^ (r & 7)) << 4);
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
          }
          asm volatile("cp.async.wait_all;" ::: "memory");
          fence_async();
          bar_arrive(GTO_BAR(q_full));
        }
        if (lane == 0 && it.t0 == 0 && it.t1 < it.n) {
          int parts = 1;
          int64_t after = it.after;
          for (int64_t c = blockIdx.x + 1; after > 0; ++c, ++parts) after -= t.each + (c < t.extra ? 1 : 0);
          p.meta[blockIdx.x] = Meta{ch.q0, it.rb * kBlock, it.rows, it.kvh, parts};
          kept = true;
        }
      }
      const int32_t* table = a.b.page_table + static_cast<int64_t>(it.s) * a.b.max_pages;
      auto page_index = [&](int e) { return p.page_shift >= 0 ? e >> p.page_shift : e / a.b.page_size; };
      int e = it.t0 * kTile + e_off, index = page_index(e);
      int page = my_box && e < it.end ? table[index] : -1;
      for (int tile = it.t0; tile < it.t1; ++tile) {
        const int place = e - index * a.b.page_size;
        bool mine = my_box && e < it.end;
        if (mine && (page < 0 || page >= a.b.n_pages)) {
          atomicOr(a.b.status, kStatusBadIndex);
          mine = false;
        }
        const int now = page;
        e += kTile;
        index = page_index(e);
        if (my_box && e < it.end && tile + 1 < it.t1) page = table[index];  // of the next tile, on its way
        const uint32_t bytes = __popc(__ballot_sync(kFull, mine)) * p.box_rows * 128;
        ok = __all_sync(kFull, bar_wait(empty + st * 8, phase, abort));
        if (!ok) break;
        const bool apart = value && it.masked(tile);
        const uint32_t bar = apart ? GTO_BAR(go) + gone % kGoRing * 8 : full + st * 8;
        if (lane == 0) {
          bar_expect(bar, bytes);
          if (apart) bar_arrive(full + st * 8);
        }
        __syncwarp();
        if (mine) tma_4d(my_dst + st * L::kTileBytes, value ? &v_map : &k_map, half * 64, it.kvh, place, now, bar);
        if (apart) ++gone;
        ++slot;
        if (++st == L::kStages) {
          st = 0;
          phase ^= 1;
        }
      }
    }
    // copies in flight end before the CTA does
    for (uint32_t i = slot > L::kStages ? slot - L::kStages : 0; i < slot; ++i)
      bar_try(full + i % L::kStages * 8, i / L::kStages & 1, kWaitTries);
    for (uint32_t i = gone > kGoRing ? gone - kGoRing : 0; i < gone; ++i)
      bar_try(GTO_BAR(go) + i % kGoRing * 8, i / kGoRing & 1, kWaitTries);
    if (value) {
      if (items > 0) bar_try(GTO_BAR(q_full), (items - 1) & 1, kWaitTries);
      if (lane == 0 && !kept) p.meta[blockIdx.x] = Meta{0, 0, 0, 0, 0};
    }
  } else if (warp == 9 || warp == 10) {
    // ---- matrix instructions: a warp for each stream, so that one waits while the other issues (the
    // tensor core takes few instructions ahead)
    constexpr bool kBf16 = T::kNegInfElem == 0xff80u;
    constexpr uint32_t kIdQk = instr_desc(kBf16, kTile, false), kIdPv = instr_desc(kBf16, DH, true);
    const uint32_t leader = elect();
    const uint32_t st = __shfl_sync(kFull, static_cast<uint32_t>(warp - 9), 0);
    const uint32_t tm = __shfl_sync(kFull, tmem, 0);
    const uint32_t q_lo = __shfl_sync(kFull, desc_lo(q_base, 16), 0);
    const uint32_t k_lo = __shfl_sync(kFull, desc_lo(keys, 16), 0);
    const uint32_t v_lo = __shfl_sync(kFull, desc_lo(values, L::kHalfBytes), 0);
    const uint32_t k_full = GTO_BAR(full), k_empty = GTO_BAR(empty), v_full = k_full + 64, v_empty = k_empty + 64;
    const uint32_t s_ready = GTO_BAR(s_ready) + st * 16, p_ready = GTO_BAR(p_ready) + st * 16,
                   pv_done = GTO_BAR(pv_done) + st * 16;
    const uint32_t s_col = tm + score_col(st, 0), o_col = tm + kOutCol + st * kRows;
    uint32_t k_at = 0, k_ph = 0, v_at = 0, v_ph = 0;  // stages of the next key and value tile, their phases
    uint32_t items = 0, qk_buf = 0, pv_buf = 0, p_ph = 0, fin = 0;
    bool ok = true;
    auto advance = [](uint32_t& at, uint32_t& ph) {
      if (++at == L::kStages) {
        at = 0;
        ph ^= 1;
      }
    };
    // a tile of the other stream is waited for and released like one's own, so that no phase of a
    // stage is missed
    auto pass_key = [&] {
      ok = __all_sync(kFull, ok && bar_wait(k_full + k_at * 8, k_ph, abort));
      if (ok && leader) bar_arrive(k_empty + k_at * 8);
      advance(k_at, k_ph);
    };
    auto pass_value = [&] {
      ok = __all_sync(kFull, ok && bar_wait(v_full + v_at * 8, v_ph, abort));
      if (ok && leader) bar_arrive(v_empty + v_at * 8);
      advance(v_at, v_ph);
    };
    auto qk = [&](uint32_t qa, bool last) {
      ok = __all_sync(kFull, ok && bar_wait(k_full + k_at * 8, k_ph, abort));
      if (!ok) return;
      tc_after();
      const uint32_t d = s_col + qk_buf * kTile, ka = k_lo + k_at * (L::kTileBytes >> 4);
#pragma unroll
      for (int k = 0; k < DH / 16; ++k)
        mma_ss(d, qa + (k / 4) * (L::kQHalfBytes >> 4) + (k % 4) * 2, ka + (k / 4) * (L::kHalfBytes >> 4) + (k % 4) * 2,
               kDescHi, kIdQk, k > 0, leader);
      tc_commit(s_ready + qk_buf * 8, leader);
      tc_commit(k_empty + k_at * 8, leader);
      if (last) tc_commit(GTO_BAR(q_empty), leader);
      qk_buf ^= 1;
      advance(k_at, k_ph);
    };
    auto pv = [&](int left, bool first) {
      ok = ok && bar_wait(v_full + v_at * 8, v_ph, abort);
      if (first) {  // the block before this one has left its accumulator
        if (fin > 0) ok = ok && bar_wait(GTO_BAR(o_free) + st * 8, (fin - 1) & 1, abort);
        ++fin;
      }
      ok = __all_sync(kFull, ok && bar_wait(p_ready + pv_buf * 8, p_ph, abort));
      if (!ok) return;
      tc_after();
      const uint32_t va = v_lo + v_at * (L::kTileBytes >> 4), pa = s_col + pv_buf * kTile;
#pragma unroll
      for (int k = 0; k < kTile / 16; ++k)
        if (k == 0 || left > k * 16) mma_ts(o_col, pa + k * 8, va + k * (2048 >> 4), kDescHi, kIdPv, k > 0 || !first, leader);
      tc_commit(pv_done + pv_buf * 8, leader);
      tc_commit(v_empty + v_at * 8, leader);
      p_ph ^= pv_buf;
      pv_buf ^= 1;
      advance(v_at, v_ph);
    };
    while (ok && walk.next(it)) {
      const int nt = it.t1 - it.t0, left = it.end - it.t0 * kTile;
      ok = bar_wait(GTO_BAR(q_full), items & 1, abort);
      ++items;
      // A stream's scores run two of its tiles ahead of its products with the values, one in each
      // buffer: the next ones lie ready when a softmax ends.
      if (it.dual()) {  // two row tiles: both streams take every tile
        const uint32_t qa = q_lo + st * (L::kQBytes >> 4);
        qk(qa, nt == 1);
        if (nt > 1) qk(qa, nt == 2);
#pragma unroll 1
        for (int j = 0; j < nt && ok; ++j) {
          pv(left - j * kTile, j == 0);
          if (j + 2 < nt) qk(qa, j + 3 == nt);
        }
      } else {  // one: the streams take the even and the odd tiles
        const int first = static_cast<int>(st);
        int keys_done = 0, values_done = 0;
        auto qk_of = [&](int j) {
          for (; keys_done < j; ++keys_done) pass_key();
          qk(q_lo, j + 2 >= nt);
          ++keys_done;
        };
        if (first < nt) qk_of(first);
        else tc_commit(GTO_BAR(q_empty), leader);
        if (first + 2 < nt) qk_of(first + 2);
#pragma unroll 1
        for (int j = first; j < nt && ok; j += 2) {
          for (; values_done < j; ++values_done) pass_value();
          pv(left - j * kTile, j == first);
          ++values_done;
          if (j + 4 < nt) qk_of(j + 4);
        }
        for (; keys_done < nt; ++keys_done) pass_key();
        for (; values_done < nt; ++values_done) pass_value();
      }
    }
    if (!ok) {  // given up: matrix instructions in flight end before tensor memory is freed
      const long long t0 = clock64();
      while (clock64() - t0 < (1ll << 22)) {
      }
    }
    __syncwarp();
  } else {
    // ---- softmax and epilogue: one thread a row
    const int st = warp >> 2;                 // stream: a row tile, or the even / odd tiles
    const int r_tile = tid & 127;
    const uint32_t lanes = static_cast<uint32_t>(warp & 3) << 21;  // first tensor-memory row of the warp
    const uint32_t s_addr = tmem + lanes + score_col(st, 0), o_addr = tmem + lanes + kOutCol + st * kRows;
    const float sl = a.scale * kLog2e;
    const uint64_t sl2 = pair(sl, sl);
    uint32_t seen = 0, tiles = 0, gone = 0, others = 0, scans[2] = {0, 0};
    bool ok = true;
    while (ok && walk.next(it)) {
      const bool dual = it.dual();
      const Chunk& ch = walk.chunk;
      const int r = (dual ? st * kRows : 0) + r_tile;
      const bool valid = r < it.rows;
      const uint32_t row = it.rb * kBlock - it.first * geo.group + (valid ? r : 0);  // from the block's first token on
      const int i = it.first + static_cast<int>(row * p.group_magic >> 16);
      // what the row sees: entries before `free_end`, and the nodes of its mask
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
      const int first_masked = max(it.common / kTile, it.t0);  // tiles from here on are masked
      float m = -INFINITY, l = 0.f;  // reference and sum
      if (lane == 0) t.lost[warp] = 0;
      if (it.alike && !__any_sync(kFull, valid)) {
        // a warp of rows that do not exist: their scores and weights may stay what they are
        for (int j = j0; j < nt && ok; j += step, ++seen) {
          const uint32_t buf = seen & 1;
          ok = __all_sync(kFull, bar_wait(GTO_BAR(s_ready) + (st * 2 + buf) * 8, (seen >> 1) & 1, abort));
          if (ok && lane == 0) bar_arrive(GTO_BAR(p_ready) + (st * 2 + buf) * 8);
        }
      } else if (j0 < nt) {
        uint32_t x[2][32];
        // Scores of a tile at the end of what the rows see: what a row does not see becomes -inf.
        auto mask = [&](int tile) {
          const uint32_t no = gone + (tile - first_masked);
          ok = __all_sync(kFull, bar_wait(GTO_BAR(go) + no % kGoRing * 8, no / kGoRing & 1, abort));
          if (!ok) return;
          unsigned char* v = smem + L::kValues + (tiles + tile - it.t0) % L::kStages * L::kTileBytes;
          const int n = min(kTile, it.end - tile * kTile);
          // rows of the last instruction's 16 that hold no entry: a weight 0 times NaN is NaN
          const int n16 = (n + 15) & ~15;
          for (int q = lane; q < (n16 - n) * L::kHalves * 8; q += 32)
            *reinterpret_cast<uint4*>(v + (q / 8 % L::kHalves) * L::kHalfBytes + (n + q / (8 * L::kHalves)) * 128 +
                                      q % 8 * 16) = make_uint4(0, 0, 0, 0);
          // Entries that some rows do not see must be finite for those: where they are not they
          // become 0, and the rows that see them get NaN in the end.  Every warp looks at all of them,
          // and nobody writes before all have looked.
          uint32_t bad0 = 0, bad1 = 0;
          if (!it.alike) {
            constexpr uint32_t kAbs = 0x7fff7fffu, kOne = T::kNegInfElem == 0xff80u ? 0x00800080u : 0x04000400u;
            const int r0 = max(0, it.common - tile * kTile);
#pragma unroll 4
            for (int q = r0 * L::kHalves * 8 + lane; q < n * L::kHalves * 8; q += 32) {
              const int vr = q / (8 * L::kHalves);
              const uint4 y = *reinterpret_cast<const uint4*>(v + (q / 8 % L::kHalves) * L::kHalfBytes + vr * 128 + q % 8 * 16);
              // an exponent of all ones carries into the sign
              const uint32_t any = ((y.x & kAbs) + kOne) | ((y.y & kAbs) + kOne) | ((y.z & kAbs) + kOne) | ((y.w & kAbs) + kOne);
              if (any & 0x80008000u) {
                if (vr < 32) bad0 |= 1u << vr;
                else bad1 |= 1u << (vr - 32);
              }
            }
            bad0 = __reduce_or_sync(kFull, bad0);
            bad1 = __reduce_or_sync(kFull, bad1);
            if (bad0 | bad1) {
              const uint32_t bar = dual ? GTO_BAR(scanned_both) : GTO_BAR(scanned) + st * 8;
              if (lane == 0) bar_arrive(bar);
              ok = __all_sync(kFull, bar_wait(bar, scans[dual ? 0 : 1]++ & 1, abort));
              if (!ok) return;
              for (int vr = 0; vr < n; ++vr)
                if ((vr < 32 ? bad0 >> vr : bad1 >> (vr - 32)) & 1)
                  for (int q = lane; q < L::kHalves * 8; q += 32)
                    *reinterpret_cast<uint4*>(v + (q / 8) * L::kHalfBytes + vr * 128 + q % 8 * 16) = make_uint4(0, 0, 0, 0);
            }
          }
          fence_async();
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            const int before = free_end - (tile * kTile + c * 32);  // visible entries at the start of these 32
            uint32_t see;
            if (before >= 32) {
              see = 0xffffffffu;
            } else {
              see = before > 0 ? (1u << before) - 1 : 0u;
              if (node) {
                // bits of the mask from node -before on
                const int sh = -before;
                uint64_t bits;
                if (sh <= 0) bits = m0 << -sh;
                else if (sh < 64) bits = (m0 >> sh) | m1 << (64 - sh);
                else bits = sh < 128 ? m1 >> (sh - 64) : 0;
                see |= static_cast<uint32_t>(bits);
              }
            }
            const uint32_t bad = c ? bad1 : bad0;
            if (bad != 0) {
              const uint32_t rows = __ballot_sync(kFull, (see & bad) != 0);
              if (lane == 0) t.lost[warp] |= rows;
            }
#pragma unroll
            for (int q = 0; q < 32; ++q)
              if (!(see >> q & 1)) x[c][q] = 0xff800000u;
          }
        };
        auto max_of = [](const uint32_t (&y)[32]) {
          float a0 = fmaxf(__uint_as_float(y[0]), __uint_as_float(y[1])), a1 = fmaxf(__uint_as_float(y[2]), __uint_as_float(y[3]));
#pragma unroll
          for (int q = 4; q < 32; q += 4) {
            a0 = max3(a0, __uint_as_float(y[q]), __uint_as_float(y[q + 1]));
            a1 = max3(a1, __uint_as_float(y[q + 2]), __uint_as_float(y[q + 3]));
          }
          return fmaxf(a0, a1);
        };
#pragma unroll 1
        for (int j = j0; j < nt; j += step) {
          const int tile = it.t0 + j;
          const uint32_t buf = seen & 1, x_addr = s_addr + buf * kTile;
          ok = __all_sync(kFull, bar_wait(GTO_BAR(s_ready) + (st * 2 + buf) * 8, (seen >> 1) & 1, abort));
          if (!ok) break;
          tc_after();
          tm_ld32(x[0], x_addr);
          tm_ld32(x[1], x_addr + 32);
          tm_wait_ld(x[0]);
          tm_after_wait(x[1]);
          if (tile >= first_masked) {
            mask(tile);
            if (!ok) break;
          }
          float top = fmaxf(max_of(x[0]), max_of(x[1])) * sl;  // to be the reference of these scores
          if (kRaise<T> != 0.f) top -= fabsf(top) < 0x1p20f ? kRaise<T> : 0.f;
          if (j == j0) {
            m = top;
          } else {
            const bool rise = valid && top > m + kLazy<T>;
            if (__any_sync(kFull, rise)) {
              // the product with the last weights is complete (those before it are: these scores were
              // issued after them)
              ok = __all_sync(kFull, bar_wait(GTO_BAR(pv_done) + (st * 2 + (buf ^ 1)) * 8, (seen - 1) >> 1 & 1, abort));
              if (!ok) break;
              tc_after();
              const float m_new = rise ? top : m;
              const float fix = rise ? ex2_approx(m - m_new) : 1.f;
              m = m_new;
              l *= fix;
#pragma unroll 1
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
          const uint64_t ref2 = pair(-ref, -ref);
          uint64_t sum_a = pair(0.f, 0.f), sum_b = sum_a;
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            uint32_t w[16];
#pragma unroll
            for (int q = 0; q < 16; ++q) {
              float p0, p1;
              unpair(fma2(pair(__uint_as_float(x[c][2 * q]), __uint_as_float(x[c][2 * q + 1])), sl2, ref2), p0, p1);
              p0 = ex2_approx(p0);
              p1 = ex2_approx(p1);
              if (q & 1) sum_b = add2(sum_b, pair(p0, p1));
              else sum_a = add2(sum_a, pair(p0, p1));
              w[q] = pack2<T>(p0, p1);
            }
            tm_st16(x_addr + c * 16, w);
          }
          float u0, u1;
          unpair(add2(sum_a, sum_b), u0, u1);
          l += u0 + u1;
          tm_wait_st();
          tc_before();
          __syncwarp();
          if (lane == 0) bar_arrive(GTO_BAR(p_ready) + (st * 2 + buf) * 8);
          ++seen;
        }
      }
      tiles += nt;
      if (it.t1 > first_masked) gone += it.t1 - first_masked;
      if (!ok) break;
      // ---- epilogue
      const bool mine = nt > j0;  // this stream had tiles
      if (mine) {
        ok = bar_wait(GTO_BAR(pv_done) + ((st) * 2 + ((seen - 1) & 1)) * 8, (seen - 1) >> 1 & 1, abort);
        ok = __all_sync(kFull, ok);
        if (!ok) break;
        tc_after();
      }
      // a sum below zero (or -0) says that the row's output is lost; its magnitude is the sum
      __syncwarp();
      if (t.lost[warp] >> lane & 1) l = -l;
      const bool join = !dual && nt > 1;
      float w0 = 1.f, w1 = 0.f;
      if (join) {
        if (st == 1) {
          t.ml[r_tile][0] = m;
          t.ml[r_tile][1] = l;
          tc_before();
          __syncwarp();
          if (lane == 0) bar_arrive(GTO_BAR(other));
          continue;
        }
        ok = bar_wait(GTO_BAR(other), others & 1, abort);
        ok = __all_sync(kFull, ok);
        if (!ok) break;
        ++others;
        tc_after();
        const float mo = t.ml[r_tile][0], lo = t.ml[r_tile][1];
        const float mm = fmaxf(m, mo);
        const float ref = mm == -INFINITY ? 0.f : mm;
        w0 = ex2_approx(m - ref);
        w1 = ex2_approx(mo - ref);
        const float sum = fabsf(l) * w0 + fabsf(lo) * w1;
        l = signbit(l) || signbit(lo) ? -sum : sum;
        m = mm;
      } else if (!mine) {
        continue;
      }
      const bool whole = it.whole();
      const int64_t tok = ch.q0 + i;
      const int h = it.kvh * geo.group + static_cast<int>(row) - (i - it.first) * geo.group;
      const float sum = fabsf(l);
      const float inv = signbit(l) ? NAN : sum > 0.f ? 1.f / sum : (sum == 0.f ? 0.f : NAN);
      const int64_t slot = 2 * static_cast<int64_t>(blockIdx.x) + (it.t0 == 0 ? 1 : 0);
      uint4* out = reinterpret_cast<uint4*>(a.out + (tok * a.n_q_heads + h) * static_cast<int64_t>(DH * 2));
      float4* part = p.part + slot * (DH / 4) * kBlock + r;
#pragma unroll 1
      for (int c = 0; c < DH / 32; ++c) {
        uint32_t o[32];
        __syncwarp();
        tm_ld32(o, o_addr + c * 32);
        if (join) {
          uint32_t y[32];
          tm_ld32(y, o_addr + kRows + c * 32);
          tm_wait_ld(o);
          tm_after_wait(y);
#pragma unroll
          for (int q = 0; q < 32; ++q)
            o[q] = __float_as_uint(__uint_as_float(o[q]) * w0 + __uint_as_float(y[q]) * w1);
        } else {
          tm_wait_ld(o);
        }
        if (c == DH / 32 - 1) {  // the accumulators are free for the next block
          tc_before();
          __syncwarp();
          if (lane == 0) {
            bar_arrive(GTO_BAR(o_free) + (st) * 8);
            if (join) bar_arrive(GTO_BAR(o_free) + (1) * 8);
          }
        }
        if (valid && whole) {
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            uint4 y;
            y.x = pack2<T>(__uint_as_float(o[8 * q]) * inv, __uint_as_float(o[8 * q + 1]) * inv);
            y.y = pack2<T>(__uint_as_float(o[8 * q + 2]) * inv, __uint_as_float(o[8 * q + 3]) * inv);
            y.z = pack2<T>(__uint_as_float(o[8 * q + 4]) * inv, __uint_as_float(o[8 * q + 5]) * inv);
            y.w = pack2<T>(__uint_as_float(o[8 * q + 6]) * inv, __uint_as_float(o[8 * q + 7]) * inv);
            out[c * 4 + q] = y;
          }
        } else if (valid) {
#pragma unroll
          for (int q = 0; q < 8; ++q)
            part[(c * 8 + q) * kBlock] = make_float4(__uint_as_float(o[4 * q]), __uint_as_float(o[4 * q + 1]),
                                                     __uint_as_float(o[4 * q + 2]), __uint_as_float(o[4 * q + 3]));
        }
      }
      if (valid) {
        if (!whole) p.part_ml[slot * kBlock + r] = make_float2(m, l);
        else if (a.lse != nullptr)
          a.lse[tok * a.n_q_heads + h] = sum == 0.f ? -INFINITY : (m + log2f(sum)) * 0.6931471805599453f;
      }
    }
  }
  tc_before();
  __syncthreads();
  tc_after();
  if (warp == 9)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
  if (tid == 0 && t.abort) atomicOr(a.b.status, kStatusTimeout);
#undef GTO_BAR
}

// Joins the parts of blocks that were cut: grid (CTAs of the first kernel, 32 rows each).  Latency
// is all there is: the weights of all parts are formed at once, then a thread has four parts in
// flight for its row and four columns.
constexpr int kJoinThreads = 256;
constexpr int kJoinRows = 32;
constexpr int kMaxCtas = 256;

template <typename T, int DH>
__global__ void __launch_bounds__(kJoinThreads) attention_join_kernel(const __grid_constant__ TcArgs p) {
  __shared__ float s_w[kMaxCtas + 1][kJoinRows];  // weight of a part's row
  __shared__ float s_m[kJoinThreads / 32][kJoinRows], s_l[kJoinThreads / 32][kJoinRows];
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const Meta meta = p.meta[blockIdx.x];
  const int first_row = blockIdx.y * kJoinRows;
  if (first_row >= meta.rows || meta.parts == 0) return;
  const AttnArgs& a = p.a;
  const int group = a.n_q_heads / a.c.n_kv_heads;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int n_rows = min(kJoinRows, meta.rows - first_row);
  const int64_t first = 2 * static_cast<int64_t>(blockIdx.x);
  auto slot = [first](int i) { return i == 0 ? first + 1 : first + 2 * i; };
  // A thread has four columns of a row, eight rows of 128 columns at a time; its first parts are asked for
  // before the weights are.
  constexpr int kRowsAtOnce = kJoinThreads / (DH / 4), kFlight = 8;
  constexpr int64_t kSlot = (DH / 4) * kBlock;
  const int r8 = threadIdx.x % kRowsAtOnce, c = threadIdx.x / kRowsAtOnce;
  const float4* part = p.part + static_cast<int64_t>(c) * kBlock + first_row;
  float4 y[kFlight];
  const auto fetch = [&](int r, int i0) {
#pragma unroll
    for (int q = 0; q < kFlight; ++q)
      if (i0 + q < meta.parts) y[q] = part[slot(i0 + q) * kSlot + r];
  };
  if (r8 < n_rows) fetch(r8, 0);
  // ---- a row's reference and sum over the parts: lane = row, the warps share the parts
  float m = -INFINITY, l = 0.f;
  for (int i = warp; i < meta.parts; i += kJoinThreads / 32) {
    const float2 ml = lane < n_rows ? p.part_ml[slot(i) * kBlock + first_row + lane] : make_float2(-INFINITY, 0.f);
    const float top = fmaxf(m, ml.x);
    const float ref = top == -INFINITY ? 0.f : top;
    l = l * ex2_approx(m - ref) + fabsf(ml.y) * ex2_approx(ml.x - ref);
    m = top;
    s_w[i][lane] = signbit(ml.y) ? NAN : ml.x;  // (a row whose output is lost)
  }
  s_m[warp][lane] = m;
  s_l[warp][lane] = l;
  __syncthreads();
  m = -INFINITY;
#pragma unroll
  for (int w = 0; w < kJoinThreads / 32; ++w) m = fmaxf(m, s_m[w][lane]);
  const float ref = m == -INFINITY ? 0.f : m;
  l = 0.f;
#pragma unroll
  for (int w = 0; w < kJoinThreads / 32; ++w) l = fmaf(s_l[w][lane], ex2_approx(s_m[w][lane] - ref), l);
  const float inv = l > 0.f ? 1.f / l : (l == 0.f ? 0.f : NAN);
  for (int i = warp; i < meta.parts; i += kJoinThreads / 32) s_w[i][lane] = ex2_approx(s_w[i][lane] - ref) * inv;
  if (warp == 0 && lane < n_rows && a.lse != nullptr) {
    const int row = meta.row0 + first_row + lane;
    a.lse[(meta.tok0 + row / group) * a.n_q_heads + meta.kvh * group + row % group] =
        l == 0.f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
  }
  __syncthreads();
  // ---- outputs
  for (int r = r8; r < n_rows; r += kRowsAtOnce) {
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    if (r != r8) fetch(r, 0);
    for (int i = 0; i < meta.parts; i += kFlight) {
      if (i > 0) fetch(r, i);
#pragma unroll
      for (int q = 0; q < kFlight; ++q)
        if (i + q < meta.parts) {
          const float w = s_w[i + q][r];
          o.x = fmaf(y[q].x, w, o.x);
          o.y = fmaf(y[q].y, w, o.y);
          o.z = fmaf(y[q].z, w, o.z);
          o.w = fmaf(y[q].w, w, o.w);
        }
    }
    const int row = meta.row0 + first_row + r;
    const int64_t at = (meta.tok0 + row / group) * a.n_q_heads + meta.kvh * group + row % group;
    uint2 packed;
    packed.x = pack2<T>(o.x, o.y);
    packed.y = pack2<T>(o.z, o.w);
    reinterpret_cast<uint2*>(a.out + at * static_cast<int64_t>(DH * 2))[c] = packed;
  }
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

// queries as [token][head][element]: a box is half a row tile
bool make_q_map(CUtensorMap* map, const AttnArgs& a, int tokens) {
  const cuuint64_t dims[3] = {static_cast<cuuint64_t>(a.c.head_dim), static_cast<cuuint64_t>(a.n_q_heads),
                              static_cast<cuuint64_t>(a.b.T)};
  const cuuint64_t strides[2] = {static_cast<cuuint64_t>(a.c.head_dim) * 2, static_cast<cuuint64_t>(a.q_stride)};
  const cuuint32_t box[3] = {64, static_cast<cuuint32_t>(a.n_q_heads / a.c.n_kv_heads), static_cast<cuuint32_t>(tokens)};
  const cuuint32_t one[3] = {1, 1, 1};
  return encode_fn()(map, a.c.dtype == GTO_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3,
                     const_cast<char*>(a.q), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
                     CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                     CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

size_t align_up(size_t x) { return (x + 255) & ~static_cast<size_t>(255); }

template <typename T, int DH>
cudaError_t tc_as(const TcArgs& p, int sms, cudaStream_t stream, int64_t* launches) {
  CUtensorMap km, vm, qm = {};
  if (p.q_tokens && !make_q_map(&qm, p.a, p.q_tokens)) return cudaErrorInvalidValue;
  if (!make_map(&km, p.a, false, p.box_rows) || !make_map(&vm, p.a, true, p.box_rows)) return cudaErrorInvalidValue;
  const size_t smem = Layout<DH>::kTail + sizeof(Tail) + 1024;
  static_assert(Layout<DH>::kTail + sizeof(Tail) + 1024 <= 232448, "shared memory of an SM");
  cudaError_t e = cudaFuncSetAttribute(attention_tc_kernel<T, DH>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                       static_cast<int>(smem));
  if (e != cudaSuccess) return e;
  sms = sms < kMaxCtas ? sms : kMaxCtas;
  attention_tc_kernel<T, DH><<<sms, kThreads, smem, stream>>>(p, km, vm, qm);
  ++*launches;
  e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(sms, kBlock / kJoinRows);
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
  return align_up(sizeof(Meta) * sms) + align_up(slots * kBlock * sizeof(float2)) +
         slots * kBlock * c.head_dim * sizeof(float);
}

cudaError_t launch_attention_tc(const AttnArgs& a, void* workspace, int sms, cudaStream_t stream, int64_t* launches) {
  TcArgs p{};
  p.a = a;
  char* ws = static_cast<char*>(workspace);
  p.meta = reinterpret_cast<Meta*>(ws);
  ws += align_up(sizeof(Meta) * sms);
  p.part_ml = reinterpret_cast<float2*>(ws);
  ws += align_up(2 * static_cast<size_t>(sms) * kBlock * sizeof(float2));
  p.part = reinterpret_cast<float4*>(ws);
  p.box_rows = 8;
  while (p.box_rows < kTile && a.b.page_size % (2 * p.box_rows) == 0) p.box_rows *= 2;
  p.box_shift = 0;
  while (p.box_rows << p.box_shift < kTile) ++p.box_shift;
  p.page_shift = -1;
  if ((a.b.page_size & (a.b.page_size - 1)) == 0)
    for (p.page_shift = 0; 1 << p.page_shift < a.b.page_size;) ++p.page_shift;
  const uint32_t group = a.n_q_heads / a.c.n_kv_heads;
  p.group_magic = (65536 + group - 1) / group;
  // a stride of a tensor map is below 2^40 bytes
  p.q_tokens = kRows % group == 0 && a.q_stride < (1ll << 40) ? kRows / group : 0;
  if (a.c.dtype == GTO_BF16)
    return a.c.head_dim == 128 ? tc_as<Bf16, 128>(p, sms, stream, launches) : tc_as<Bf16, 64>(p, sms, stream, launches);
  return a.c.head_dim == 128 ? tc_as<F16, 128>(p, sms, stream, launches) : tc_as<F16, 64>(p, sms, stream, launches);
}

}  // namespace gto
