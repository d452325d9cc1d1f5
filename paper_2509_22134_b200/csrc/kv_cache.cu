// Paged key / value cache: gto_kv_append (rotation, optional norms, placement) and gto_kv_commit
// (the accepted tokens of a verified tree moved together).  Both move bytes and nothing else
// bounds them: append reads and writes (n_q + 2 n_kv) * head_dim values a token once, commit reads
// and writes 2 * n_kv * head_dim values an accepted token and layer once.
//
// Measured, heads of 128: eight prompts of up to 4000 tokens, 40 query and 40 key heads, 185 us (97 % of the
// copy rate); 64 trees of 61 tokens, 32 and 8 heads, 25.1 us, of which 14.9 are the bytes and the rest
// the chain place -> position -> rotation of three waves of CTAs.  Asking for the rows before that
// chain cost more in registers than it hid (26 to 32 us), prefetching them into L2 too (26 us);
// 42 registers a thread for a wave less gave 181 and 24.9 us, and 4.0 instead of 3.6 for one token.
// Commit: 64 sequences, 32 layers 13.8 to 14.2 us (9.1 for the bytes).
#include "decode_common.cuh"

namespace gto {
namespace {

constexpr int kAppendThreads = 128;
constexpr int kMaxHalf = kMaxHeadDim / 2;  // rotated pairs of a head

// cos and sin of position * inv_freq.  The angle is formed and reduced to a fraction of a turn in
// fp64 (at position 100 000 an fp32 angle is off by 0.004 rad); the reduced fraction is below 1/2
// and its rounding to fp32 costs half a step of 2^-24 turns.
__device__ __forceinline__ void turn(double position, double inv_freq, float& c, float& s) {
  const double turns = position * inv_freq * 0.15915494309189535;
  const float f = static_cast<float>(turns - rint(turns));
  sincospif(2.0f * f, &s, &c);
}

// One CTA per token, and one that looks at all sequences for those that contradict themselves.  A group
// of `lanes` lanes (a power of two, at least half the 16-byte vectors of a head) takes one head at a
// time; a lane holds the two vectors whose elements rotate into one another.
template <typename T, bool kInterleaved>
__global__ void __launch_bounds__(kAppendThreads) kv_append_kernel(AppendArgs a, int lanes) {
  constexpr int E = T::kPerVec;
  __shared__ float s_cos[kMaxHalf], s_sin[kMaxHalf];
  __shared__ int s_seq;
  const int tid = threadIdx.x, t = blockIdx.x;
  if (t == a.b.T) {
    for (int s = tid; s < a.b.S; s += kAppendThreads)
      if (!load_chunk(a.b, s).ok) atomicOr(a.b.status, kStatusBadIndex);
    return;
  }
  if (tid == 0) s_seq = -1;
  __syncthreads();
  bool fall = false;
  for (int s = tid; s < a.b.S; s += kAppendThreads) {
    const int q0 = a.b.q_start[s], q1 = a.b.q_start[s + 1];
    if (q0 <= t && t < q1) s_seq = s;
    fall |= q1 < q0;
  }
  if (__syncthreads_or(fall)) {  // several sequences may have the token: the first counts, if q_start has not decreased before
    if (tid == 0) {
      s_seq = -1;
      for (int s = 0; s < a.b.S && !falls(a.b, s); ++s)
        if (a.b.q_start[s] <= t && t < a.b.q_start[s + 1]) s_seq = s;
    }
    __syncthreads();
  }
  const int s = s_seq;
  if (s < 0) return;  // a token of no sequence, or of one that is skipped
  const Chunk ch = load_chunk(a.b, s);
  const int i = t - ch.q0;
  int page = -1, pos = 0;
  bool ok = ch.ok && i >= 0 && i < ch.n;
  if (ok) {
    page = page_of(a.b, s, ch.base + i);
    pos = ch.base + i;
    if (i >= ch.lead)
      pos = ch.base + ch.lead - 1 + a.b.node_depth[static_cast<int64_t>(s) * a.b.g + i - ch.lead];
    ok = page >= 0;
  }
  if (!ok) {
    if (tid == 0) atomicOr(a.b.status, kStatusBadIndex);
    return;
  }
  const int half = a.rope_dims / 2;
  for (int f = tid; f < half; f += kAppendThreads)
    turn(static_cast<double>(pos), a.inv_freq[f], s_cos[f], s_sin[f]);
  __syncthreads();

  const int Dh = a.c.head_dim, hq = a.q ? a.n_q_heads : 0, hkv = a.c.n_kv_heads;
  const int pairs = Dh / (2 * E), rot_pairs = a.rope_dims / (2 * E);
  const int lane = tid & (lanes - 1);
  const int groups = kAppendThreads / lanes;
  const int64_t entry = (ch.base + i) % a.b.page_size;
  char* krow = a.c.k + page * a.c.k_page + entry * a.c.k_entry;
  char* vrow = a.c.v + page * a.c.v_page + entry * a.c.v_entry;
  const int head_bytes = Dh * T::kBytes;
  const bool mine = lane < pairs;
  // vectors of this lane: (x_i, x_{i+half}) lie half apart; pairs (2i, 2i+1), and values that
  // are not rotated, lie side by side
  int v0, v1;
  if (kInterleaved || lane >= rot_pairs) {
    v0 = 2 * lane;
    v1 = v0 + 1;
  } else {
    v0 = lane;
    v1 = lane + rot_pairs;
  }
  const int heads = hq + 2 * hkv;
  const int rounds = (heads + groups - 1) / groups;  // the same for every lane: shuffles inside
  for (int r = 0; r < rounds; ++r) {
    const int h = r * groups + tid / lanes;
    const char* src = nullptr;
    char* dst = nullptr;
    const char* w = nullptr;
    bool rotate = false;
    if (h < hq) {
      src = a.q + t * a.q_stride + static_cast<int64_t>(h) * head_bytes;
      dst = a.q_out + (static_cast<int64_t>(t) * hq + h) * head_bytes;
      w = a.q_norm;
      rotate = true;
    } else if (h < hq + hkv) {
      src = a.k + t * a.k_stride + static_cast<int64_t>(h - hq) * head_bytes;
      dst = krow + (h - hq) * a.c.k_head;
      w = a.k_norm;
      rotate = true;
    } else if (h < heads) {
      src = a.v + t * a.v_stride + static_cast<int64_t>(h - hq - hkv) * head_bytes;
      dst = vrow + (h - hq - hkv) * a.c.v_head;
    }
    uint4 x0 = make_uint4(0, 0, 0, 0), x1 = x0;
    const bool live = mine && src != nullptr;
    if (live) {
      x0 = *reinterpret_cast<const uint4*>(src + v0 * 16);
      x1 = *reinterpret_cast<const uint4*>(src + v1 * 16);
    }
    float f0[E], f1[E];
    T::unpack(x0, f0);
    T::unpack(x1, f1);
    if (w != nullptr || a.q_norm != nullptr || a.k_norm != nullptr) {
      float ss = 0.f;
#pragma unroll
      for (int e = 0; e < E; ++e) ss = fmaf(f0[e], f0[e], fmaf(f1[e], f1[e], ss));
      for (int o = lanes >> 1; o > 0; o >>= 1) ss += __shfl_xor_sync(kFull, ss, o);
      if (w != nullptr && live) {
        const float rs = rsqrtf(ss / Dh + a.norm_eps);
        float w0[E], w1[E];
        T::unpack(*reinterpret_cast<const uint4*>(w + v0 * 16), w0);
        T::unpack(*reinterpret_cast<const uint4*>(w + v1 * 16), w1);
#pragma unroll
        for (int e = 0; e < E; ++e) {
          f0[e] *= rs * w0[e];
          f1[e] *= rs * w1[e];
        }
      }
    }
    if (!live) continue;
    if (rotate) {
      if (kInterleaved) {
#pragma unroll
        for (int e = 0; e < E; e += 2) {
          const int p0 = (v0 * E + e) >> 1, p1 = (v1 * E + e) >> 1;
          if (p0 < half) {
            const float c = s_cos[p0], sn = s_sin[p0], u = f0[e], y = f0[e + 1];
            f0[e] = u * c - y * sn;
            f0[e + 1] = y * c + u * sn;
          }
          if (p1 < half) {
            const float c = s_cos[p1], sn = s_sin[p1], u = f1[e], y = f1[e + 1];
            f1[e] = u * c - y * sn;
            f1[e + 1] = y * c + u * sn;
          }
        }
      } else if (lane < rot_pairs) {
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const float c = s_cos[lane * E + e], sn = s_sin[lane * E + e], u = f0[e], y = f1[e];
          f0[e] = u * c - y * sn;
          f1[e] = y * c + u * sn;
        }
      }
      x0 = T::pack(f0);
      x1 = T::pack(f1);
    }
    *reinterpret_cast<uint4*>(dst + v0 * 16) = x0;
    *reinterpret_cast<uint4*>(dst + v1 * 16) = x1;
  }
}

// One CTA per (sequence, layer); a thread owns a 16-byte column of the entries and carries it along
// the path.  In-place is safe in any order of columns: entry j is written after entry path[j] >= j
// was read, and later sources lie above j; within a chunk of eight all loads precede the stores.
constexpr int kCommitThreads = 256;
constexpr int kCommitBatch = 8;

__global__ void __launch_bounds__(kCommitThreads) kv_commit_kernel(CommitArgs a) {
  const int s = blockIdx.x, layer = blockIdx.y, tid = threadIdx.x;
  const Chunk ch = load_chunk(a.b, s);
  const int accepted = a.accept_len[s];
  const int len = ch.ok && ch.nodes > 0 ? accepted : 0;
  const bool ok = ch.ok && len >= 0 && len <= a.D;
  __shared__ int64_t s_ksrc[kMaxDepth], s_kdst[kMaxDepth], s_vsrc[kMaxDepth], s_vdst[kMaxDepth];
  bool bad = !ok, behind = false;
  static_assert(kMaxDepth <= 32, "the first warp looks up the path, the others the rest meanwhile");
  if (tid >= 32) {
    // a decrease of q_start, which the CTA of the sequence there reports
    for (int j = tid - 32; j < s; j += kCommitThreads - 32) behind |= falls(a.b, j);
    if (ok && ch.lead + len > 0) {
      // the pages of all entries that stay: without one, append has left the token out
      const int last = (ch.base + ch.lead + len - 1) / a.b.page_size;
      for (int p = ch.base / a.b.page_size + tid - 32; p <= last; p += kCommitThreads - 32)
        bad |= page_of(a.b, s, p * a.b.page_size) < 0;
    }
  } else if (ok && tid < len) {
    const int32_t* path = a.path_node + static_cast<int64_t>(s) * a.D;
    const int p = path[tid];
    const int before = tid > 0 ? path[tid - 1] : -1;
    bool good = p > before && p >= tid && p < ch.nodes;
    if (good) {
      const int e0 = ch.base + ch.lead + p, e1 = ch.base + ch.lead + tid;
      const int64_t p0 = page_of(a.b, s, e0), p1 = page_of(a.b, s, e1);
      const int64_t r0 = e0 % a.b.page_size, r1 = e1 % a.b.page_size;
      good = p0 >= 0 && p1 >= 0;
      s_ksrc[tid] = p0 * a.c.k_page + r0 * a.c.k_entry;
      s_kdst[tid] = p1 * a.c.k_page + r1 * a.c.k_entry;
      s_vsrc[tid] = p0 * a.c.v_page + r0 * a.c.v_entry;
      s_vdst[tid] = p1 * a.c.v_page + r1 * a.c.v_entry;
    }
    bad = !good;
  }
  if (__syncthreads_or(bad || behind)) {
    if (!__syncthreads_or(behind) && tid == 0) atomicOr(a.b.status, kStatusBadIndex);
    return;
  }
  if (layer == 0 && tid == 0) a.kv_len_out[s] = ch.base + ch.lead + len;
  const int per_head = a.c.head_dim * (a.c.dtype == GTO_F32 ? 4 : 2) / 16;
  const int cols = a.c.n_kv_heads * per_head;
  for (int c = tid; c < 2 * cols; c += kCommitThreads) {
    const bool key = c < cols;
    const int cc = key ? c : c - cols;
    const int64_t at = (cc / per_head) * (key ? a.c.k_head : a.c.v_head) + (cc % per_head) * 16;
    char* base = (key ? a.c.k + layer * a.c.k_layer : a.c.v + layer * a.c.v_layer) + at;
    const int64_t* src = key ? s_ksrc : s_vsrc;
    const int64_t* dst = key ? s_kdst : s_vdst;
    for (int j0 = 0; j0 < len; j0 += kCommitBatch) {
      uint4 x[kCommitBatch];
#pragma unroll
      for (int j = 0; j < kCommitBatch; ++j)
        if (j0 + j < len) x[j] = *reinterpret_cast<const uint4*>(base + src[j0 + j]);
#pragma unroll
      for (int j = 0; j < kCommitBatch; ++j)
        if (j0 + j < len && src[j0 + j] != dst[j0 + j])
          *reinterpret_cast<uint4*>(base + dst[j0 + j]) = x[j];
    }
  }
}

template <typename T>
cudaError_t append_as(const AppendArgs& a, cudaStream_t stream) {
  int lanes = 1;
  while (lanes < a.c.head_dim / (2 * T::kPerVec)) lanes *= 2;
  if (a.interleaved)
    kv_append_kernel<T, true><<<a.b.T + 1, kAppendThreads, 0, stream>>>(a, lanes);
  else
    kv_append_kernel<T, false><<<a.b.T + 1, kAppendThreads, 0, stream>>>(a, lanes);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_kv_append(const AppendArgs& a, cudaStream_t stream, int64_t* launches) {
  ++*launches;
  if (a.c.dtype == GTO_BF16) return append_as<Bf16>(a, stream);
  if (a.c.dtype == GTO_F16) return append_as<F16>(a, stream);
  return append_as<F32>(a, stream);
}

cudaError_t launch_kv_commit(const CommitArgs& a, cudaStream_t stream, int64_t* launches) {
  ++*launches;
  kv_commit_kernel<<<dim3(a.b.S, a.c.n_layers), kCommitThreads, 0, stream>>>(a);
  return cudaGetLastError();
}

}  // namespace gto
