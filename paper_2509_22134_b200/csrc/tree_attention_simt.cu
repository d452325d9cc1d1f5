// gto_tree_attention on the fp32 units: fp32 tensors, and the head sizes and page sizes that the
// tensor-core kernel does not take.
//
// Online softmax over tiles of 32 cache entries.  A CTA owns 16 query rows of one key head (a row is
// one token and one of the query heads that share the key head), so that a tile is read once for
// all query heads of the group; a cluster of two, four or eight CTAs splits the entries of the same
// rows, since few rows and a long cache is what decoding is, and joins (maximum, sum, output) through
// distributed shared memory in a fixed order.  All arithmetic is fp32.  A tile is a chain: its keys
// and values (0.8 us; their pages were looked up during the tile before), scores, softmax, output;
// small calls are bound by that chain, large ones by shared-memory reads, a float4 for four
// fused multiply-adds: 42 rows of 8 heads on 300 entries of 64 take 15.4 to 17 us by the clock, 1000 prompt tokens of
// 32 heads on up to 1000 entries of 128 take 1.0 ms (12 TFLOP/s).
#include <cooperative_groups.h>

#include "decode_common.cuh"

namespace gto {
namespace {

namespace cg = cooperative_groups;

constexpr int kThreads = 128;
constexpr int kRows = 16;    // query rows of a CTA; eight threads each
constexpr int kTile = 32;    // entries of a tile
constexpr int kCols = 8;     // threads of a row
constexpr int kMaxQuads = kMaxHeadDim / (4 * kCols);

// Sequence that work unit `unit` belongs to, where sequence s has units(chunk of s) of them; the
// unit's number inside the sequence in *rest.  Called by the whole CTA; -1 past the last unit.  Sequences from
// the first decrease of q_start on have none.
template <typename F>
__device__ int find_unit(const BatchArgs& b, int64_t unit, F units, int64_t* rest) {
  __shared__ int64_t s_scan[kThreads / 32];
  __shared__ int s_found, s_fall;
  __shared__ int64_t s_rest;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if (tid == 0) {
    s_found = -1;
    s_fall = b.S;
  }
  int64_t before = 0;
  for (int s0 = 0; s0 < b.S; s0 += kThreads) {
    const int s = s0 + tid;
    int64_t n = 0;
    bool fall = false;
    if (s < b.S) {
      const Chunk c = load_chunk(b, s);
      if (c.ok) n = units(c);
      else atomicOr(b.status, kStatusBadIndex);
      fall = !c.ok && falls(b, s);
    }
    int64_t run;
    const auto scan = [&] {
      run = n;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int64_t y = __shfl_up_sync(kFull, run, o);
        if (lane >= o) run += y;
      }
      __syncthreads();
      if (lane == 31) s_scan[warp] = run;
    };
    scan();
    if (fall) atomicMin(&s_fall, s);
    __syncthreads();
    const bool last = s_fall < b.S;
    if (last) {  // once more without the sequences that are skipped
      if (s >= s_fall) n = 0;
      scan();
      __syncthreads();
    }
    int64_t total = 0;
    for (int w = 0; w < kThreads / 32; ++w) {
      if (w < warp) run += s_scan[w];
      total += s_scan[w];
    }
    run += before;
    if (unit < run && unit >= run - n) {
      s_found = s;
      s_rest = unit - (run - n);
    }
    before += total;
    __syncthreads();
    if (s_found >= 0 || last) break;
  }
  *rest = s_rest;
  return s_found;
}

template <typename T, int kSplit>
__global__ void __launch_bounds__(kThreads) attention_simt_kernel(AttnArgs a) {
  constexpr int E = T::kPerVec;
  extern __shared__ __align__(16) float s_mem[];
  cg::cluster_group cluster = cg::this_cluster();
  const int rank = static_cast<int>(cluster.block_rank());
  const int tid = threadIdx.x;
  const int Dh = a.c.head_dim, group = a.n_q_heads / a.c.n_kv_heads;
  const int ld = Dh + 4;  // rows 16 bytes apart modulo the banks
  float* s_q = s_mem;                    // [kRows][Dh]
  float* s_k = s_q + kRows * Dh;         // [kTile][ld]
  float* s_v = s_k + kTile * ld;         // [kTile][ld]
  float* s_o = s_v + kTile * ld;         // [kRows][Dh], for the join
  __shared__ float s_p[kRows][kTile + 1];
  __shared__ float s_ml[kRows][2];
  __shared__ int s_page[2][kTile];  // of this tile's entries and of the next one's

  int64_t rest;
  const int s = find_unit(a.b, blockIdx.x / kSplit, [group](const Chunk& c) {
    return (static_cast<int64_t>(c.n) * group + kRows - 1) / kRows;
  }, &rest);
  if (s < 0) return;  // the whole cluster has the same unit
  const Chunk ch = load_chunk(a.b, s);
  const int kvh = blockIdx.y;
  const int64_t row0 = rest * kRows;
  const int64_t rows_all = static_cast<int64_t>(ch.n) * group;
  const int rows = static_cast<int>(rows_all - row0 < kRows ? rows_all - row0 : kRows);

  for (int v = tid; v < kRows * (Dh / E); v += kThreads) {
    const int r = v / (Dh / E), c = v % (Dh / E);
    float f[E];
#pragma unroll
    for (int e = 0; e < E; ++e) f[e] = 0.f;
    if (r < rows) {
      const int64_t row = row0 + r;
      const int64_t tok = ch.q0 + row / group;
      const int h = kvh * group + static_cast<int>(row % group);
      T::unpack(*reinterpret_cast<const uint4*>(a.q + tok * a.q_stride +
                                                (static_cast<int64_t>(h) * Dh) * T::kBytes + c * 16), f);
    }
#pragma unroll
    for (int e = 0; e < E; ++e) s_q[r * Dh + c * E + e] = f[e];
  }

  const int r = tid / kCols, col = tid % kCols;
  const int i = r < rows ? static_cast<int>((row0 + r) / group) : 0;
  const int end = kv_end(ch, static_cast<int>((row0 + rows - 1) / group));
  const float sl = a.scale * kLog2e;
  float m = -INFINITY, l = 0.f;
  float4 o[kMaxQuads];
#pragma unroll
  for (int j = 0; j < kMaxQuads; ++j) o[j] = make_float4(0.f, 0.f, 0.f, 0.f);

  const auto look_up = [&](int e0) {  // thread tid < kTile: the page of entry e0 + tid
    int page = -1;
    if (tid < end - e0) {
      page = page_of(a.b, s, e0 + tid);
      if (page < 0) atomicOr(a.b.status, kStatusBadIndex);
    }
    return page;
  };
  int buf = 0;
  if (tid < kTile) s_page[0][tid] = look_up(rank * kTile);
  for (int e0 = rank * kTile; e0 < end; e0 += kSplit * kTile, buf ^= 1) {
    const int n = min(kTile, end - e0);
    __syncthreads();
    const int next = tid < kTile ? look_up(e0 + kSplit * kTile) : 0;  // on its way while the tile is
    for (int v = tid; v < kTile * (Dh / E); v += kThreads) {
      const int e = v / (Dh / E), c = v % (Dh / E);
      const int page = s_page[buf][e];
      uint4 xk = make_uint4(0, 0, 0, 0), xv = xk;
      if (page >= 0) {
        const int64_t slot = (e0 + e) % a.b.page_size;
        xk = *reinterpret_cast<const uint4*>(a.c.k + page * a.c.k_page + slot * a.c.k_entry + kvh * a.c.k_head + c * 16);
        xv = *reinterpret_cast<const uint4*>(a.c.v + page * a.c.v_page + slot * a.c.v_entry + kvh * a.c.v_head + c * 16);
      }
      float fk[E], fv[E];
      T::unpack(xk, fk);
      T::unpack(xv, fv);
#pragma unroll
      for (int q = 0; q < E; ++q) {
        s_k[e * ld + c * E + q] = fk[q];
        s_v[e * ld + c * E + q] = fv[q];
      }
    }
    if (tid < kTile) s_page[buf ^ 1][tid] = next;
    __syncthreads();
    float x[kTile / kCols];
#pragma unroll
    for (int j = 0; j < kTile / kCols; ++j) x[j] = 0.f;
    for (int d = 0; d < Dh; d += 4) {
      const float4 q4 = *reinterpret_cast<const float4*>(s_q + r * Dh + d);
#pragma unroll
      for (int j = 0; j < kTile / kCols; ++j) {
        const float4 k4 = *reinterpret_cast<const float4*>(s_k + (col + j * kCols) * ld + d);
        x[j] = fmaf(q4.x, k4.x, fmaf(q4.y, k4.y, fmaf(q4.z, k4.z, fmaf(q4.w, k4.w, x[j]))));
      }
    }
    float top = -INFINITY;
#pragma unroll
    for (int j = 0; j < kTile / kCols; ++j) {
      const int e = col + j * kCols;
      const bool see = r < rows && e < n && s_page[buf][e] >= 0 && sees(a.b, s, ch, i, e0 + e);
      x[j] = see ? x[j] * sl : -INFINITY;
      top = fmaxf(top, x[j]);
    }
#pragma unroll
    for (int q = 1; q < kCols; q <<= 1) top = fmaxf(top, __shfl_xor_sync(kFull, top, q));
    const float m_new = fmaxf(m, top);
    const float ref = m_new == -INFINITY ? 0.f : m_new;
    const float fix = exp2f(m - ref);
    float sum = 0.f;
#pragma unroll
    for (int j = 0; j < kTile / kCols; ++j) {
      const float p = exp2f(x[j] - ref);
      sum += p;
      s_p[r][col + j * kCols] = p;
    }
    l = l * fix + sum;  // this thread's share of the row's sum
    m = m_new;
    __syncwarp();  // a row's eight threads are in one warp
#pragma unroll
    for (int j = 0; j < kMaxQuads; ++j) {
      o[j].x *= fix; o[j].y *= fix; o[j].z *= fix; o[j].w *= fix;
    }
    // (weights behind the last entry are 0, and the tile is filled up)
    for (int e = 0; e < n; e += 4) {
      float p[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) p[u] = s_p[r][e + u];
#pragma unroll
      for (int j = 0; j < kMaxQuads; ++j) {
        const int d = (j * kCols + col) * 4;
        if (d < Dh) {
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            const float4 v4 = *reinterpret_cast<const float4*>(s_v + (e + u) * ld + d);
            if (p[u] != 0.f) {  // an entry that the row does not see may hold anything, NaN too
              o[j].x = fmaf(p[u], v4.x, o[j].x);
              o[j].y = fmaf(p[u], v4.y, o[j].y);
              o[j].z = fmaf(p[u], v4.z, o[j].z);
              o[j].w = fmaf(p[u], v4.w, o[j].w);
            }
          }
        }
      }
    }
  }
#pragma unroll
  for (int q = 1; q < kCols; q <<= 1) l += __shfl_xor_sync(kFull, l, q);
  if (col == 0) {
    s_ml[r][0] = m;
    s_ml[r][1] = l;
  }
#pragma unroll
  for (int j = 0; j < kMaxQuads; ++j) {
    const int d = (j * kCols + col) * 4;
    if (d < Dh) *reinterpret_cast<float4*>(s_o + r * Dh + d) = o[j];
  }
  cluster.sync();
  // ---- join: CTA `rank` finishes kMine of the rows
  constexpr int kMine = kRows / kSplit;
  const int jr = rank * kMine + tid / (kThreads / kMine);
  const int t0 = tid % (kThreads / kMine);
  if (jr < rows) {
    float top = -INFINITY, w[kSplit], total = 0.f;
    for (int q = 0; q < kSplit; ++q) top = fmaxf(top, cluster.map_shared_rank(&s_ml[0][0], q)[jr * 2]);
    for (int q = 0; q < kSplit; ++q) {
      const float* ml = cluster.map_shared_rank(&s_ml[0][0], q) + jr * 2;
      w[q] = ml[0] == -INFINITY ? 0.f : exp2f(ml[0] - top);
      total = fmaf(w[q], ml[1], total);
    }
    const float inv = total > 0.f ? 1.f / total : (total == 0.f ? 0.f : NAN);
    const int64_t row = row0 + jr;
    const int64_t tok = ch.q0 + row / group;
    const int h = kvh * group + static_cast<int>(row % group);
    char* out = a.out + (tok * a.n_q_heads + h) * static_cast<int64_t>(Dh) * T::kBytes;
    for (int c = t0; c < Dh / E; c += kThreads / kMine) {
      float f[E];
#pragma unroll
      for (int e = 0; e < E; ++e) f[e] = 0.f;
      for (int q = 0; q < kSplit; ++q) {
        const float* po = cluster.map_shared_rank(s_o, q) + jr * Dh + c * E;
        if (w[q] != 0.f) {
#pragma unroll
          for (int e = 0; e < E; ++e) f[e] = fmaf(w[q], po[e], f[e]);
        }
      }
#pragma unroll
      for (int e = 0; e < E; ++e) f[e] *= inv;
      *reinterpret_cast<uint4*>(out + c * 16) = T::pack(f);
    }
    if (a.lse != nullptr && t0 == 0)
      a.lse[tok * a.n_q_heads + h] =
          total == 0.f ? -INFINITY : (top + log2f(total)) * 0.6931471805599453f;
  }
  cluster.sync();  // nobody leaves while its rows are read
}

template <typename T, int kSplit>
cudaError_t simt_as(const AttnArgs& a, int64_t units, cudaStream_t stream) {
  const int Dh = a.c.head_dim;
  const size_t smem = sizeof(float) * (2 * kRows * Dh + 2 * kTile * (Dh + 4));
  cudaError_t e = cudaFuncSetAttribute(attention_simt_kernel<T, kSplit>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                       static_cast<int>(sizeof(float) * (2 * kRows * kMaxHeadDim + 2 * kTile * (kMaxHeadDim + 4))));
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(static_cast<unsigned>(units * kSplit), a.c.n_kv_heads);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr{};
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = kSplit;
  attr.val.clusterDim.y = 1;
  attr.val.clusterDim.z = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, attention_simt_kernel<T, kSplit>, a);
}

template <typename T>
cudaError_t simt_as(const AttnArgs& a, int sms, cudaStream_t stream) {
  // the lengths are on the device: as many units as T tokens in S chunks can make
  const int group = a.n_q_heads / a.c.n_kv_heads;
  const int64_t units = (static_cast<int64_t>(a.b.T) * group + kRows - 1) / kRows + a.b.S;
  // Few units: more CTAs for each shorten the walk over its entries (one token on 2000 entries 45 us with
  // eight, 84 with four; 14 tree rows on 300 entries 15.7 and 18.2).  More: the join costs what it
  // shortens (100 tokens on 200 entries 18.5 us with four, 27 with eight; 500 tokens on 1000 entries,
  // 2016 units, 1015 with two, 1090 with four).
  const int64_t all = units * a.c.n_kv_heads;
  if (all <= sms / 2) return simt_as<T, 8>(a, units, stream);
  if (all <= 8ll * sms) return simt_as<T, 4>(a, units, stream);
  return simt_as<T, 2>(a, units, stream);
}

}  // namespace

cudaError_t launch_attention_simt(const AttnArgs& a, int sms, cudaStream_t stream, int64_t* launches) {
  ++*launches;
  if (a.c.dtype == GTO_BF16) return simt_as<Bf16>(a, sms, stream);
  if (a.c.dtype == GTO_F16) return simt_as<F16>(a, sms, stream);
  return simt_as<F32>(a, sms, stream);
}

}  // namespace gto
