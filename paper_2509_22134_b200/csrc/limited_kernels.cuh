// gto_sample_tokens and gto_verify_tree_limited: tokens drawn from softmax(z / temperature) of which top-k,
// top-p and min-p leave a part.
//
// With w_i = exp((z_i - max z) / temperature) and the tokens in the order (z descending, id ascending), every
// limit keeps a prefix of that order, so that what stays is "no lower than a border", a pair (value, id); the token
// is then the first id at which the cumulative sum of what stays passes u times the whole.
//
// A row is shared by a cluster of one to eight CTAs and read once.  On the way every thread leaves the maximum of
// each of its slots (some 32 logits), and the warps leave sums of fp32 weights where the row's whole mass will
// be needed.  From the slots' maxima it follows about how many tokens, and which mass, a value and all above it
// hold (a slot is a bucket that tokens fall into by chance: with J of B slots reaching the value, about
// -B ln(1 - J/B) tokens do), and so a value that all that stays lies above.  The few slots that reach it are
// read again, their tokens above it make a list, and the list is sorted, summed in fp64 and cut.  Rows of which
// more stays than the list holds are counted into 2048 bins, summed in fp64 above the bin of the border, and only that bin's
// tokens are listed (Row::wide); where these are too many as well, the interval is narrowed (Row::wide_border).
//
// Decisions are those of fp64 sums.  The whole mass is summed in fp32 with a bound on its error (kSlack); a decision that
// it could turn is taken again after the row has been summed in fp64.
//
// Many rows have a CTA each, which leaves to a second kernel's clusters what the list or the fp32 sums cannot tell.
//
// What bounds it, as measured on a B200: a row of 128 256 bf16 of which a list's worth stays takes 13 to 20 us with its launch (eight
// CTAs: 3 us of reading, then a chain of some ten barriers and exchanges of 0.5 us each); one of which thousands stay 35 us,
// most of it two more passes, one of shared-memory atomics and one of fp64 (64 lanes a cycle and SM, 20 instructions a
// token).  512 such rows with mixed limits take 101 to 109 us (131 MB at 1.2 TB/s): the first kernel about 50 us, of which 20 us
// is the reading at 6.6 TB/s and 8 us the exponentials, the second about 55 us for the few per cent of rows that it is left.
#pragma once

#include <algorithm>

#include "limited_row.cuh"

namespace gto {

constexpr int kLater = -2;  // token of a row that is left to the second kernel

// Marks a row as left, and lists it where there is room.
__device__ __forceinline__ void leave(const LimitedArgs& a, int s) {
  a.token[s] = kLater;
  const int at = atomicAdd(a.left, 1);
  if (at < kMaxLeft) a.left[kLeftRows + at] = s;
}

// What a kernel serves: rows that a list or the warps' sums can tell, the others are left; all; those that were left.
enum Mode { kEasy, kAll, kLeft };

// Row (kTree: tree) s, by the CTAs of a cluster.
template <typename T, int kCluster, int kThreads, bool kTree, Mode kMode>
__device__ __forceinline__ void serve(const LimitedArgs& a, Shared<kCluster, kThreads, kMode != kEasy>& sh, int s, int rank) {
  constexpr bool kServesAll = kMode != kEasy;
  using R = Row<T, kCluster, kThreads, kServesAll>;
  constexpr int kNodes = kTree ? kMaxNodes : 1;
  constexpr int kChunks = kMaxNodes / 32;
  __shared__ int s_id[kNodes], s_parent[kNodes], s_removed[kNodes];
  __shared__ float s_u[kNodes];
  __shared__ double s_p[kNodes];
  __shared__ int s_child, s_removed_n, s_close;
  const int tid = threadIdx.x, lane = tid & 31;
  R row(sh, a.V, rank);
  row.alone = kMode == kAll;  // (kLeft: its kernel has waited)
  const bool first = row.rank == 0 && tid == 0;
  if constexpr (kServesAll) row.fill_table();  // (read behind a barrier)

  const float heat = a.temperature[s];
  const bool greedy = heat == 0.f;
  const int ask_k = a.top_k ? a.top_k[s] : 0;
  const float top_p = a.top_p ? a.top_p[s] : 1.f, min_p = a.min_p ? a.min_p[s] : 0.f;
  const bool sound = heat >= 0.f && heat < INFINITY && top_p == top_p && min_p == min_p;
  const int top_k = ask_k > 0 && ask_k < a.V ? ask_k : 0;
  const float floor = fminf(fmaxf(min_p, 0.f), 1.f);
  const double scale = greedy ? 0.0 : 1.4426950408889634 / static_cast<double>(heat);
  const float c2 = static_cast<float>(scale);
  const bool hot = !(c2 < 1e30f && c2 > 1e-8f);  // (a temperature next to 0, or far above the logits, is beyond fp32)
  const bool limited = top_k > 0 || top_p < 1.f || floor > 0.f;
  const bool sums = kMode != kLeft && !greedy && !hot && (!limited || (top_p < 1.f && top_k == 0));
  row.scale_to(scale);
  const auto unit = [](float u) { return static_cast<double>(fminf(fmaxf(u, 0.f), 0.99999994f)); };
  const double u_last = unit(a.u[s]);

  int64_t at_row = s;
  bool lost = false;  // no such row
  if (!kTree && a.rows) {
    at_row = a.rows[s];
    lost = at_row < 0 || at_row >= a.n_rows;
    if (lost && first) atomicOr(a.status, kStatusBadIndex);
  }
  if (kTree) {
    int nodes = a.n_nodes ? a.n_nodes[s] : a.g;
    bool report = nodes < 0 || nodes > a.g;
    if (report) nodes = 0;
    for (int n = tid; n < kMaxNodes; n += kThreads) {
      int id = -1, parent = -2;  // no context's child
      if (n < nodes) {
        const int64_t at = static_cast<int64_t>(s) * a.g + n;
        const int tok = a.node_token[at], par = a.node_parent[at];
        if (tok >= 0 && tok < a.V_draft) id = a.d2t ? a.d2t[tok] : tok;
        if (id >= 0 && id < a.V && par >= -1 && par < n) parent = par;
        else report = true;
        s_u[n] = a.u_node[at];
      }
      s_id[n] = id;
      s_parent[n] = parent;
    }
    if (report && row.rank == 0) atomicOr(a.status, kStatusBadIndex);
    at_row = static_cast<int64_t>(s) * a.rows_of_tree;
    __syncthreads();
  }

  int len = 0, cur = -1, last = -1;
  bool later = false;  // more than this kernel does
  bool drawn = false;  // the last token, by the lane that found it
  if (!sound && first) atomicOr(a.status, kStatusNonFinite);
  int64_t here = at_row;
  bool go = sound && !lost;
  while (go) {
    go = false;
    row.z = a.logits + here * a.row_stride;
    double mass = 0.0;
    bool masked = !kTree && !limited && a.n_kept;
    bool bad;
    if (kMode != kLeft && sums) bad = row.template stream<true>(&mass, &masked);
    else bad = row.template stream<false>(&mass, &masked);
    if (bad || !(fabsf(row.M) < INFINITY)) {
      if (first) atomicOr(a.status, kStatusNonFinite);
      break;
    }
    int best = -1;
    // What stays: the border, how the sums were made, the mass.
    uint64_t border = 0;
    bool listed = false, exact = false;
    typename R::Wide wide;
    wide.ok = wide.near = false;
    double total = 1.0;
    int n_stay = 1;
    if (greedy) {
      best = row.best();
    } else if (!limited) {
      total = mass;
      exact = hot || kMode == kLeft;
      if (hot) {
        if constexpr (kMode == kEasy) {
          later = true;
          break;
        } else if constexpr (kTree) {
          total = row.whole();
        }
      }
      n_stay = a.V;
      if (masked) {
        int n = 0;
        row.each([&](float x, int id) { n += x > -INFINITY; });
        n_stay = row.reduce(0.0, 0.0, n, 0).n;
      }
    } else {
      if constexpr (kMode != kLeft) {
        if (!(hot && top_p < 1.f && top_k == 0)) {
          float tau;
          const int n = row.aim_at(top_k, top_p, mass, floor, &tau) ? row.gather(tau) : R::kList + 1;
          if (n <= R::kList) {
            Cut cut = row.cut(n, top_k, top_p, mass, sums ? kSlack * mass : 0.0, floor, tau);
            if constexpr (kServesAll) {
              if (cut.close) {
                mass = row.whole();
                cut = row.cut(n, top_k, top_p, mass, 0.0, floor, tau);
              }
            }
            listed = exact = cut.enough && (kServesAll || !cut.close);
            if (listed) {
              border = cut.border;
              total = cut.total;
              n_stay = cut.n;
            }
          }
        }
      }
      if constexpr (!kServesAll) {
        if (!listed) {
          later = true;
          break;
        }
      } else if (!listed) {
        exact = true;
        row.wide(top_k, top_p, floor, &wide);
        if (wide.ok) {
          border = wide.border;
          total = wide.total;
          n_stay = wide.n;
        }
      }
      if constexpr (kServesAll) {
        if (!listed && !wide.ok) {
          const float from = row.near_from();
#pragma unroll 1
          for (int kind = 0; kind < 2; ++kind) {
            if (kind == 0 ? top_k == 0 : !(top_p < 1.f)) continue;
            double goal = wide.goal;
            if (kind == 1 && !wide.near) {
              double m = 0.0;
              row.each([&](float x, int id) { m += x > -INFINITY && make_key(x, id) >= border ? row.raw_any(x, from) : 0.0; });
              goal = static_cast<double>(top_p) * row.reduce(m, 0.0, 0, 0).a;
            }
            border = row.wide_border(border, kind == 0 ? top_k : 0, goal, wide);
          }
          const double least = static_cast<double>(floor);
          double m = 0.0;
          int n = 0;
          uint32_t low = 0xffffffffu;  // the lowest value that min-p leaves
          row.each([&](float x, int id) {
            if (x == -INFINITY || make_key(x, id) < border) return;
            const double w = row.raw_any(x, from);
            if (w < least) return;
            m += w;
            ++n;
            low = min(low, orderable(x));
          });
          const auto r = row.reduce(m, 0.0, n, 0);
          uint32_t unused = 0;
          row.least_most(&low, &unused);
          total = r.a;
          n_stay = r.n;
          if (floor > 0.f) {
            const uint64_t f = static_cast<uint64_t>(low) << 32;  // with any id
            border = f > border ? f : border;
          }
        }
      }
    }
    const auto weight = [&](float x, int id) { return x > -INFINITY && make_key(x, id) >= border ? row.raw(x) : 0.0; };
    int removed = 0;
    if constexpr (kTree) {
      // ---- the children of the context, in list order (the same in every CTA)
      for (;;) {
        __syncthreads();
        if (tid < 32) {
          int child = -1, gone_n = 0;
          bool close = false;
          const double slack = exact ? 0.0 : kSlack * total;
          double gone = 0.0;
#pragma unroll 1
          for (int c = 0; c < kChunks; ++c) {
            const int n = c * 32 + lane;
            const bool is = s_parent[n] == cur;
            if (!__any_sync(kFull, is) || child >= 0 || close) continue;
            const int id = s_id[n];
            if (greedy) {
              const unsigned hit = __ballot_sync(kFull, is && id == best);
              if (hit) child = c * 32 + __ffs(hit) - 1;
              continue;
            }
            // All children of the chunk at once: each as if those before it had been refused; the first
            // that is accepted is the child.  The token of an earlier sibling has nothing left.
            const unsigned same = __match_any_sync(kFull, is ? id : -1 - lane);
            bool again = (same & ((1u << lane) - 1)) != 0;
            for (int r = 0; r < gone_n; ++r) again |= s_removed[r] == id;
            const bool tried = is && !again;
            const double p = tried ? weight(T::load1(row.z, id), id) : 0.0;
            const double upto = scan_warp(p, lane);
            const double aim = tried ? unit(s_u[n]) * (total - gone - (upto - p)) : 0.0;
            const unsigned yes = __ballot_sync(kFull, tried && aim < p);
            const unsigned near = __ballot_sync(kFull, tried && p > 0.0 && fabs(aim - p) < slack);
            const int at = yes ? __ffs(yes) - 1 : 31;
            close = (near & (0xffffffffu >> (31 - at))) != 0;
            if (yes) {
              child = c * 32 + at;
            } else {
              const unsigned out = __ballot_sync(kFull, tried);
              if (tried) {
                const int r = gone_n + __popc(out & ((1u << lane) - 1));
                s_removed[r] = id;
                s_p[r] = p;
              }
              gone_n += __popc(out);
              gone += __shfl_sync(kFull, upto, 31);
              __syncwarp();
            }
          }
          if (lane == 0) {
            s_child = child;
            s_removed_n = gone_n;
            s_close = close;
          }
        }
        __syncthreads();
        if (!s_close) break;
        total = row.whole();
        exact = true;
      }
      removed = s_removed_n;
      const int child = s_child;
      if (child >= 0) {
        if (len == a.D) {  // a tree deeper than it may be
          if (first) atomicOr(a.status, kStatusBadIndex);
          break;
        }
        if (first) {
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
            if (first) atomicOr(a.status, kStatusBadIndex);
            break;
          }
          here = at_row + 1 + (depth - 1) * a.k + slot;
        } else {
          here = at_row + 1 + child;
        }
        row.cluster_sync();  // (what the others may still read of this row)
        go = true;
        continue;
      }
    }
    if (greedy) {
      last = best;
      break;
    }
    const auto out = [&](int id) {
      if (kTree)
        for (int r = 0; r < removed; ++r)
          if (s_removed[r] == id) return true;
      return false;
    };
    const auto taken = [&](int lo, int hi) {
      double g = 0.0;
      if (kTree)
        for (int r = 0; r < removed; ++r)
          if (s_removed[r] >= lo && s_removed[r] < hi) g += s_p[r];
      return g;
    };
    const auto left = [&](float x, int id) { return out(id) ? 0.0 : weight(x, id); };
    const auto write = [&](const Found& f, double whole) {
      if (!f.mine) return;
      if (kTree) {
        a.token[static_cast<int64_t>(s) * (a.D + 1) + len] = f.id;
      } else {
        a.token[s] = f.id;
        if (a.logp) a.logp[s] = f.id < 0 ? 0.f : static_cast<float>(log(f.weight / whole));
        if (a.n_kept) a.n_kept[s] = f.id < 0 ? 0 : n_stay;
      }
    };
    drawn = true;
    if (listed) {
      write(row.draw_listed(n_stay, u_last, out), total);
      break;
    }
    if constexpr (kServesAll) {
      if (wide.ok) {
        write(row.draw_wide(wide, u_last, taken, left), total);
        break;
      }
    }
    bool close = exact;
    if constexpr (kMode != kLeft) {
      if (!exact) {
        const Found f = row.draw_all(u_last, total, taken, out);
        if constexpr (kMode == kEasy) {
          if (f.mine && f.close) leave(a, s);
          else write(f, total);
        } else {
          Mail m{};
          m.n = __any_sync(kFull, f.mine && f.close);
          const Mail* all = row.post(m);
          bool some = false;
#pragma unroll
          for (int r = 0; r < R::kMailRounds; ++r)
            if (r * 32 + lane < R::kMails) some |= all[r * 32 + lane].n != 0;
          close = __any_sync(kFull, some);
          if (!close) write(f, total);
        }
      }
    }
    if constexpr (kServesAll) {
      if (close) {
        Found f;
        if (!kTree && !limited) f = row.locate_all(u_last);
        else f = row.locate(left, u_last, 0.0);
        write(f, f.total);
      }
    }
  }
  if (kCluster > 1) {
    row.meet();          // (where no row was read)
    row.cluster_sync();  // nobody leaves while its shared memory is read
  }
  if (row.rank != 0) return;
  if (kTree) {
    if (tid == 0) {
      a.accept_len[s] = len;
      if (!drawn) a.token[static_cast<int64_t>(s) * (a.D + 1) + len] = last;
    }
    for (int j = len + tid; j < a.D; j += kThreads) a.path_node[static_cast<int64_t>(s) * a.D + j] = -1;
    for (int j = len + 1 + tid; j <= a.D; j += kThreads) a.token[static_cast<int64_t>(s) * (a.D + 1) + j] = -1;
  } else if (tid == 0 && later) {
    leave(a, s);
  } else if (tid == 0 && !drawn) {
    a.token[s] = last;
    if (a.logp) a.logp[s] = 0.f;
    if (a.n_kept) a.n_kept[s] = last < 0 ? 0 : 1;
  }
}

// Row of CTA i of N.  An SM has the CTAs i, i + 148, i + 296, ..., and settings often repeat every 2, 4 or 8 rows: rows in
// their own order gave some SMs nothing but rows whose weights are summed (exponential units busy 61 % of the time on one SM, 2 % on another;
// 512 mixed rows of 128 256 bf16: 117 us, so 108).
__device__ __forceinline__ int spread(int i, int N) { return (i & ~15) + 16 <= N ? (i & ~15) | ((i + (i >> 4)) & 15) : i; }

// One CTA a row, for many rows: what a list of the likeliest tokens, or the sums of the warps, can tell.
template <typename T, int kThreads>
__global__ void __launch_bounds__(kThreads, 1280 / kThreads) many_rows_kernel(LimitedArgs a) {
  __shared__ Shared<1, kThreads, false> sh;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");  // (the next kernel may get ready)
  serve<T, 1, kThreads, false, kEasy>(a, sh, spread(static_cast<int>(blockIdx.x), a.N), 0);
}

constexpr int kClusterThreads = 256;

// A cluster a row or tree, for whatever the limits leave.
template <typename T, int kCluster, bool kTree>
__global__ void __launch_bounds__(kClusterThreads, 2) limited_kernel(LimitedArgs a) {
  __shared__ Shared<kCluster, kClusterThreads, true> sh;
  Row<T, kCluster, kClusterThreads, true>::begun();
  serve<T, kCluster, kClusterThreads, kTree, kAll>(a, sh, static_cast<int>(blockIdx.x / kCluster), static_cast<int>(blockIdx.x % kCluster));
}

// The rows that many_rows_kernel has left.
template <typename T, int kCluster>
__global__ void __launch_bounds__(kClusterThreads, 2) left_rows_kernel(LimitedArgs a) {
  __shared__ Shared<kCluster, kClusterThreads, true> sh;
  using R = Row<T, kCluster, kClusterThreads, true>;
  R::begun();
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int rank = static_cast<int>(blockIdx.x % kCluster), clusters = static_cast<int>(gridDim.x / kCluster);
  const int left = a.left[0];
  R::wait_for_others();
  __syncthreads();  // (all of the CTA have read the count before thread 0 says so below)
  if (left <= kMaxLeft) {
    for (int i = blockIdx.x / kCluster; i < left; i += clusters) {
      const int s = a.left[kLeftRows + i];
      // (always, unless calls that share the workspace ran at once)
      if (s >= 0 && s < a.N) serve<T, kCluster, kClusterThreads, false, kLeft>(a, sh, s, rank);
    }
  }
  // the last one to have read the count sets it to 0 for the next call
  if (threadIdx.x == 0) {
    __threadfence();
    if (atomicAdd(a.left + 1, 1) == static_cast<int>(gridDim.x) - 1) a.left[0] = a.left[1] = 0;
  }
  if (left <= kMaxLeft) return;
  // (more than the list holds: every cluster looks at its share of the rows.  A row's mark is only changed by its own
  // cluster, behind a barrier of all its CTAs)
  for (int64_t s = blockIdx.x / kCluster; s < a.N; s += clusters) {
    const bool mine = a.token[s] == kLater;
    if (kCluster > 1) asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
    if (mine) serve<T, kCluster, kClusterThreads, false, kLeft>(a, sh, static_cast<int>(s), rank);
  }
}

template <typename K>
cudaError_t launch(K kernel, const LimitedArgs& a, int64_t rows, int cluster, int threads, bool after, cudaStream_t stream,
                   int64_t* launches) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(static_cast<unsigned>(rows * cluster));
  cfg.blockDim = dim3(static_cast<unsigned>(threads));
  cfg.stream = stream;
  cudaLaunchAttribute attr[2] = {};
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = static_cast<unsigned>(cluster);
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  // (its CTAs may be placed while the kernel before it ends, for which they wait themselves)
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = after ? 2 : 1;
  ++*launches;
  return cudaLaunchKernelEx(&cfg, kernel, a);
}

template <typename T>
cudaError_t limited_as(const LimitedArgs& a, bool tree, int sms, cudaStream_t stream, int64_t* launches) {
  if (tree) return launch(limited_kernel<T, 8, true>, a, a.N, 8, kClusterThreads, false, stream, launches);
  // As many CTAs a row as fit the device twice over; one where there are rows enough, and then the few that need more than it can
  // tell by clusters.  A cluster's exchanges cost more than its CTAs save where the row is short.  Measured, in us, for rows that
  // mix limits (in brackets: all top-k 50):
  //   of 128 256 bf16     8: 55 (16) by eight, 66 (16) by four, 82 (31) by one; 37: 51 (27), 64 (18), 84 (31);
  //                       74: 59 (39), 66 (29), 100 (31); 148: 102 (61), 84 (41), 107 (31); 300: 170 (117), 119 (68), 113 (35)
  //   of 32 000 f16       8: 45 (14), 29 (14), 45 (21); 74: 57 (35), 35 (23), 49 (21); 148: 94 (57), 47 (33), 59 (21); 300: by one 74 (23)
  const bool brief = a.V <= (128 << 10) / static_cast<int>(16 / T::kPerVec);
  if (!brief && a.N * 8ll <= 2ll * sms) return launch(limited_kernel<T, 8, false>, a, a.N, 8, kClusterThreads, false, stream, launches);
  if (a.N * 4ll <= 2ll * sms) return launch(limited_kernel<T, 4, false>, a, a.N, 4, kClusterThreads, false, stream, launches);
  // Ten small CTAs an SM where they have work and only the rows' sums to make, else five with as many loads on their way: of
  // 128 256 bf16 1000 rows without limits take 92 us with 128 threads and 109 with 256, with top-k 50 82 and 74.
  const bool small = a.N > 5ll * sms && !a.top_k && !a.top_p && !a.min_p;
  const cudaError_t e = small ? launch(many_rows_kernel<T, 128>, a, a.N, 1, 128, false, stream, launches)
                              : launch(many_rows_kernel<T, 256>, a, a.N, 1, 256, false, stream, launches);
  if (e != cudaSuccess) return e;
  // What is left, by clusters of two where rows are short and of four where they are long: 512 mixed rows of 32 000 f16 take 74
  // and 88 us, 148 of 128 256 bf16 131 and 107.  (An odd number of clusters: settings that repeat fall to all of them.)
  if (brief) return launch(left_rows_kernel<T, 2>, a, std::max(sms * 2 / 2 - 1, 1), 2, kClusterThreads, true, stream, launches);
  return launch(left_rows_kernel<T, 4>, a, std::max(sms * 2 / 4 - 1, 1), 4, kClusterThreads, true, stream, launches);
}

}  // namespace gto
