/*
 * gto.h - C ABI of the B200 draft-tree pass of Group Tree Optimization (GTO).
 *
 * One training micro-batch holds B positions.  For every position there are G = 2
 * draft trees: t = 0 built from the current draft model's logits, t = 1 from the
 * frozen reference draft's.  Logit rows are inputs (one V-wide row per context):
 *
 *   draft  [G, B, D, k, V_draft]   row [t,b,0,0,:] is the root context; row [t,b,d,j,:]
 *                                  (1 <= d < D) is the context reached through frontier
 *                                  slot j of depth d; rows [t,b,0,1..k-1,:] are never read.
 *   target [G, B, R, V_target]     R = 1 + (D-1)*k; row 0 = root context, row
 *                                  1 + (d-1)*k + j = frontier slot j of depth d.
 *
 * Logits are bf16, fp16 (the paper trains under FP16 autocast, App. B) or fp32, row-major,
 * contiguous; V_draft and V_target must make a row a
 * multiple of 16 bytes.  All pointers in the structs below are DEVICE pointers owned by
 * the caller, 16-byte aligned, dense row-major with the shapes given.  The library
 * allocates memory only in gto_create (its device workspace and a page-locked host copy of
 * the row list for gto_tree_reward_host) and gto_decode_create (its workspace) and keeps no caller pointer
 * after a call returns.  Calls enqueue work on `stream` (a cudaStream_t passed as void*)
 * and return without synchronising; argument errors are returned at once and launch
 * nothing.  Data faults (a non-finite row sum, an index out of range in a caller's table) are recorded
 * in a device status word read by gto_device_status.  A context is not thread-safe;
 * use one per host thread and device.  No entry point writes to stdout or throws.
 */
#ifndef GTO_H_
#define GTO_H_

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct gto_ctx gto_ctx; /* opaque; owns the workspace only */

typedef enum {
  GTO_OK = 0,
  GTO_ERR_INVALID_ARG = 1, /* null pointer, bad shape, misaligned pointer               */
  GTO_ERR_UNSUPPORTED = 2, /* shape outside the compiled limits (see gto_create)        */
  GTO_ERR_WORKSPACE = 3,   /* workspace allocation failed                                */
  GTO_ERR_CUDA = 4,        /* a CUDA runtime call failed                                 */
  GTO_ERR_NONFINITE = 5,   /* device status: a row's log-sum-exp was not finite          */
  GTO_ERR_TIMEOUT = 6,     /* device status: a wait inside gto_tree_attention or gto_verify_tree
                              ran out; the outputs of that attention are unspecified, a
                              sequence that could not be verified has accept_len -1        */
  GTO_ERR_TOO_LARGE = 7,   /* gto_build_tree_noalloc: batch exceeds the fixed scratch    */
  GTO_ERR_BAD_INDEX = 8    /* device status: an index in a caller's table (d2t, a tree's
                              rows, tokens or parents, a path's rows, a page table, the
                              lengths of a batch) was out of range; the
                              entry was skipped, results that depend on it are unspecified  */
} gto_status;

typedef enum { GTO_F32 = 0, GTO_BF16 = 1, GTO_F16 = 2 } gto_dtype;

/* Reward aggregation over the tree's sequences: Eq. 5 (log-sum-exp smooth max, the
 * default) or the two alternatives of the aggregation ablation in Sec. 4.2. */
typedef enum { GTO_AGG_LSE = 0, GTO_AGG_MAX = 1, GTO_AGG_MEAN = 2 } gto_agg;

enum {
  GTO_FLAG_STD_UNBIASED = 1u, /* Eq. 10 with the sample std (divide by m-1)             */
  GTO_FLAG_NO_DEBIAS = 2u,    /* Eq. 9 switched off: R_i = r(T_i) (debiasing ablation)  */
  GTO_FLAG_FORCE_ROW_SPLIT = 16u, /* always split a logit row over a thread-block cluster (the
                                  library does so by itself where it pays: few, long rows);
                                  for tests and tuning                                      */
  GTO_FLAG_SEQ_ALL_NODES = 8u, /* Eq. 5 over the root-to-node sequence of every selected node
                                  instead of the root-to-leaf sequences only                 */
  GTO_FLAG_PATH_MAX_EXPECTED = 32u, /* the "longest accepted sequence" of Sec. 3.2 read as the
                                  candidate sequence with the largest expected acceptance length
                                  L_i of Eq. 3 (lowest list position on ties), reported whole, root
                                  to its last node; default: the greedy-target verification walk */
  GTO_FLAG_GRAD_LIVE_ROWS = 4u /* gto_group_surrogate_grad writes only the rows that carry a
                                  gradient (j < path_len[b] and coeff[b] != 0) and leaves the
                                  rest of grad untouched, instead of filling it with zeros   */
};

typedef struct {
  int32_t B;        /* positions; a multiple of m                                       */
  int32_t G;        /* trees per position; must be 2                                    */
  int32_t D;        /* maximum tree depth d of Sec. 3.1                                 */
  int32_t k;        /* top-k per node expansion and per layer (App. B: 10)              */
  int32_t g;        /* nodes kept by the global prune, root excluded (App. B: 60)       */
  int32_t m;        /* group size of Eq. 6 (App. B: 8); groups are consecutive positions */
  int32_t V_draft;  /* draft vocabulary                                                  */
  int32_t V_target; /* target vocabulary                                                 */
  int32_t logit_dtype; /* gto_dtype of draft, target and grad                           */
  int32_t reward_agg;  /* gto_agg                                                       */
  float eta;        /* smooth-max temperature of Eq. 5 (App. B: 1)                      */
  float clip_eps;   /* epsilon of Eq. 12                                                */
  float std_delta;  /* delta of Eq. 10                                                  */
  float grad_scale; /* factor on the summed group losses (a trainer passes omega / K)   */
  uint32_t flags;
} gto_config;

/* The pruned draft trees (Sec. 3.1, tree policy G).  Node lists hold g nodes per tree in
 * ascending pool index (depth-major candidate number), so a parent precedes its children. */
typedef struct {
  int32_t* node_token;   /* [G,B,g] draft-vocabulary id                                  */
  int32_t* node_parent;  /* [G,B,g] list position of the parent, -1 = child of the root  */
  int32_t* node_depth;   /* [G,B,g] 1..D                                                 */
  int32_t* node_ctx_row; /* [G,B,g] context row (0..R-1) the token was proposed from     */
  int32_t* node_slot;    /* [G,B,g] frontier slot of the node at its depth, -1 = not expanded */
  int32_t* node_pool;    /* [G,B,g] pool index: c at depth 1, k + (d-2)k^2 + j*k + c later */
  float* node_logp;      /* [G,B,g] draft log-probability of the edge into the node      */
  double* node_score;    /* [G,B,g] global acceptance score: sum of node_logp on the path */
  uint64_t* node_mask;   /* [G,B,g,W] W = ceil(g/64): bit a of row n = a is n or an ancestor */
  double* row_lse;       /* [G,B,R] log-sum-exp of every draft context row               */
} gto_tree;

/* Draft Tree Reward (Eq. 3-5) and the longest accepted sequence (Sec. 3.2) of tree 0. */
typedef struct {
  double* reward;        /* [G,B] r = R(T; eta)                                          */
  double* etree;         /* [G,B] sum over nodes of the path product (exact expected
                                  accepted tokens under target sampling; auxiliary)      */
  int32_t* n_leaves;     /* [G,B] number N of sequences (leaves) in Eq. 5                */
  float* node_ptarget;   /* [G,B,g] target probability of the node's token in its context */
  float* node_pathprod;  /* [G,B,g] Eq. 4: product of node_ptarget from the root         */
  float* node_L;         /* [G,B,g] Eq. 3 for the sequence ending at the node            */
  double* row_lse_t;     /* [G,B,R] target log-sum-exp; NaN for rows no node uses        */
  int32_t* row_argmax_t; /* [G,B,R] greedy target token (lowest id on ties); -1 likewise */
  int32_t* path_len;     /* [B] l_i: accepted draft tokens of tree 0 under the greedy target */
  int32_t* path_node;    /* [B,D] list positions of the accepted nodes; -1 beyond l_i    */
  int32_t* path_row;     /* [B,D] context row of each step (the draft row that produced it) */
  int32_t* path_token;   /* [B,D] draft token ids                                        */
  float* path_logp;      /* [B,D] draft log-probability of each step; 0 beyond l_i       */
} gto_reward;

/* Group statistics and surrogate of Eq. 9-12. */
typedef struct {
  double* R;        /* [B] debiased reward, Eq. 9                                        */
  double* adv;      /* [B] standardised advantage, Eq. 10                                */
  double* ratio;    /* [B] s_i of Eq. 11                                                 */
  double* coeff;    /* [B] factor on (onehot - softmax) for every step of position i     */
  int32_t* active;  /* [B] 1 if the unclipped branch of Eq. 12 is the minimum            */
  double* loss;     /* [B/m] group losses of Eq. 12                                      */
} gto_grad_stats;

/* Validates the configuration and allocates the workspace on `device`.
 * Limits: G == 2; 1 <= k and k*k <= 128; 1 <= g <= min(128, k + (D-1)k^2); 1 <= D <= 16;
 * B % m == 0; G*B <= 65535; k <= V_draft; V * sizeof(logit) a multiple of 16 for both vocabularies.
 * Returns GTO_ERR_UNSUPPORTED outside them. */
gto_status gto_create(gto_ctx** ctx, const gto_config* cfg, int device);
gto_status gto_destroy(gto_ctx* ctx);

/* Tree policy G of Sec. 3.1 for all G*B trees: per context row the draft log-softmax and
 * its k best tokens (value descending, id ascending); layer-wise expansion keeping the k
 * best of the k*k candidates of each layer by cumulative log-probability (Fig. 1 caption:
 * path confidence is the product of edge probabilities); global top-g over all
 * k + (D-1)k^2 candidates.  Every tie goes to the lower index.  Writes every array of *out. */
gto_status gto_build_tree(gto_ctx* ctx, const void* draft_logits, const gto_tree* out,
                          void* stream);

/* Largest G*B*R*k (draft context rows times top-k) gto_build_tree_noalloc accepts: its
 * scratch is a fixed array of 8 bytes per entry (8 MiB) inside the library image. */
#define GTO_NOALLOC_MAX_ENTRIES (1 << 20)

/* gto_build_tree for callers that must not allocate device memory (no counterpart in the
 * paper: it is an integration aid).  A trainer that routes every device byte through its own
 * allocator, a process living inside a fixed memory budget, or a thread that cannot afford
 * the device-wide stall an allocation may cause, cannot create a gto_ctx, because gto_create
 * calls cudaMalloc.  This call needs no context: it takes the configuration directly and
 * keeps the per-row top-k tables in a fixed device array that ships with the library (every
 * GPU that loads the library holds those 8 MiB until the process ends).  It never calls
 * cudaMalloc, cudaFree or any allocating routine.
 *   - Computes exactly what gto_build_tree computes and writes every array of *out; only
 *     B, G, D, k, g, V_draft and logit_dtype of *cfg are used.
 *   - Returns GTO_ERR_TOO_LARGE when G*B*R*k > GTO_NOALLOC_MAX_ENTRIES: split the batch.
 *   - The first call on a device looks up the array's device address (one
 *     cudaGetSymbolAddress, cached per device); make that first call outside any stream
 *     capture.
 *   - All calls on a device share the one array and it keeps the last call's contents; the
 *     call clears what it needs cleared.  Two calls whose kernels can overlap on the GPU
 *     (different streams, no dependency between them) race on it: order them.
 *   - There is no status word to read back: a row with non-finite logits shows as a
 *     non-finite entry of out->row_lse. */
gto_status gto_build_tree_noalloc(const gto_config* cfg, int device, const void* draft_logits,
                                  const gto_tree* out, void* stream);

/* Draft Tree Reward, Eq. 3-5, and the longest accepted sequence of Sec. 3.2.  Reads only
 * the target rows that are the context of a selected node.  d2t maps draft ids to target
 * ids ([V_draft] int32, device, injective); NULL means identity and needs
 * V_draft == V_target.  Writes every array of *out. */
gto_status gto_tree_reward(gto_ctx* ctx, const gto_tree* tree, const void* target_logits,
                           const int32_t* d2t, const gto_reward* out, void* stream);

/* gto_tree_reward for target logits that live in HOST memory (Eq. 3-5 and Sec. 3.2 as
 * above).  Only the target rows that are the context of a selected node are needed
 * (about a fifth of them at the paper's tree shape), so only those cross the bus: the call
 * builds the row list on the device, reads it back (it SYNCHRONISES `stream` once), copies
 * each run of adjacent needed rows from target_host to the same offset of target_dev, and
 * then proceeds as gto_tree_reward on target_dev.  target_host: HOST [G,B,R,V_target],
 * should be page-locked for the copies to be asynchronous; target_dev: DEVICE scratch of the
 * same shape owned by the caller, rows that are not needed are left untouched.
 * *rows_copied (optional, host) receives the number of rows copied. */
gto_status gto_tree_reward_host(gto_ctx* ctx, const gto_tree* tree, const void* target_host,
                                void* target_dev, const int32_t* d2t, const gto_reward* out,
                                void* stream, int64_t* rows_copied);

/* Eq. 9-12 and the derivative of the summed group losses with respect to the draft logits:
 * grad[b,j,:] = coeff_b * (onehot(path_token[b,j]) - softmax(draft row path_row[b,j] of
 * tree 0)) for j < path_len[b], zero otherwise (also when the ratio is clipped).  With
 * GTO_FLAG_GRAD_LIVE_ROWS the zero rows are not written (a trainer that scatters the rows
 * into its logit gradient by path_row reads only the live ones).
 * old_logp [B,D] fp32: log-probabilities of the accepted tokens under the old / reference
 * draft (entries beyond path_len ignored).  grad [B,D,V_draft] in the logit dtype. */
gto_status gto_group_surrogate_grad(gto_ctx* ctx, const void* draft_logits,
                                    const gto_tree* tree, const gto_reward* reward,
                                    const float* old_logp, void* grad,
                                    const gto_grad_stats* out, void* stream);

/* Token-level loss of Eq. 13 / App. B. */
typedef struct {
  double* loss;   /* [B] H(p_T, p_M) of the position's prefix                              */
  double* lse_t;  /* [B] log-sum-exp of the target logits over the (mapped) draft vocabulary */
} gto_token_stats;

/* Token-level loss L_token of Eq. 13 (defined in App. B): for every position b the
 * cross-entropy H(p_T, p_M) = -sum_v p_T(v) log p_M(v) from the target's next-token
 * distribution to the draft's under the same teacher-forced prefix, i.e. on the root context
 * rows draft[0,b,0,0,:] and target[0,b,0,:].  With a reduced draft vocabulary p_T is the
 * softmax of the target logits at the mapped ids d2t[0..V_draft) (NULL = identity).  Writes
 * out->loss[b] and grad_root[b,:] = weight * (p_M - p_T), the derivative of weight * H with
 * respect to the draft logits of that row ([B, V_draft], logit dtype, every entry written);
 * a trainer passes weight = 1 / (number of supervised positions).  Needs tree->row_lse from
 * gto_build_tree on the same draft logits.  Any d2t with entries in [0, V_target) is served;
 * an increasing one (a vocabulary subset listed in id order) reads every 32-byte sector of
 * the target row once.  An entry outside the target vocabulary is reported in the device
 * status word (GTO_ERR_BAD_INDEX) and counts as probability 0. */
gto_status gto_token_loss(gto_ctx* ctx, const void* draft_logits, const void* target_logits,
                          const int32_t* d2t, const gto_tree* tree, float weight,
                          void* grad_root, const gto_token_stats* out, void* stream);

/* The total loss of Sec. 3.2, L = L_token + omega * L_GTO, as ONE gradient buffer: the same
 * computation as gto_token_loss, with the root-row gradient weight * (p_M - p_T) of position b
 * going into slice grad[b,0,:] of the buffer gto_group_surrogate_grad filled ([B,D,V_draft]).
 * Step 0 of an accepted path is always taken from the root row, so where that slice already
 * holds a surrogate gradient (path_len[b] > 0 and coeff[b] != 0) the token gradient is added
 * to it, and elsewhere the slice is overwritten.  Afterwards grad[b,0,:] is the derivative of
 * weight * H_b + grad_scale * (sum of the group losses) with respect to the root row of
 * position b, for every b (also where path_row[b,0] is -1).  Call it after
 * gto_group_surrogate_grad on the same stream, with that call's reward and stats. */
gto_status gto_token_loss_accumulate(gto_ctx* ctx, const void* draft_logits,
                                     const void* target_logits, const int32_t* d2t,
                                     const gto_tree* tree, const gto_reward* reward,
                                     const gto_grad_stats* stats, float weight, void* grad,
                                     const gto_token_stats* out, void* stream);

/* SampleGroups of Algorithm 1 under Eq. 6-7: K non-overlapping groups of m adjacent positions
 * of a sequence of length s; start indices are 1-based, 1 <= t_k <= s - m + 1 and
 * t_{k+1} >= t_k + m.  Host-only (no device work): `u` is a HOST array of K uniforms in
 * [0, 1) supplied by the caller, `starts` a HOST array that receives t_1 < ... < t_K.  The
 * paper fixes no law for the draw; this one turns the K uniforms into K independent offsets
 * in [0, s - K m], sorts them and shifts the k-th (0-based) by k m.  Every admissible
 * placement can occur, but not equally often: its weight is the number of orderings of its
 * offsets, so placements with groups packed back to back (equal offsets) are rarer.  Returns
 * GTO_ERR_INVALID_ARG when K*m > s or an argument is out of range. */
gto_status gto_sample_groups(int32_t s, int32_t m, int32_t K, const double* u, int32_t* starts);

/* Synchronises `stream`, then reads and clears the device status word:
 * *host_code = GTO_OK, GTO_ERR_NONFINITE or GTO_ERR_BAD_INDEX.  Kernels check
 * every index they take from a caller's table before using it as an address. */
gto_status gto_device_status(gto_ctx* ctx, void* stream, int32_t* host_code);

/* Number of kernel launches the library has enqueued through this context. */
int64_t gto_launch_count(const gto_ctx* ctx);

/* Kernels of one pass, in launch order (index into the arrays of gto_kernel_times). */
enum {
  GTO_K_DRAFT_ROWS = 0,  /* Sec. 3.1 (i): log-softmax + top-k of every draft row          */
  GTO_K_TREE_BUILD = 1,  /* Sec. 3.1 (i)-(ii): layer-wise expansion, global top-g         */
  GTO_K_REWARD_PLAN = 2, /* list of target rows that are the context of a selected node   */
  GTO_K_TARGET_ROWS = 3, /* Eq. 4: log-sum-exp and greedy token of every listed target row */
  GTO_K_TREE_REWARD = 4, /* Eq. 3-5 and the longest accepted sequence                      */
  GTO_K_GROUP_STATS = 5, /* Eq. 9-12 per group                                             */
  GTO_K_GRAD_ROWS = 6,   /* derivative of Eq. 12 into the draft rows of the accepted path  */
  GTO_K_TOKEN_LOSS = 7,  /* Eq. 13 / App. B: cross-entropy and its gradient on the root rows */
  GTO_K_COUNT = 8
};

/* Per-kernel device timing, off by default.  While enabled, every launch is bracketed by
 * two CUDA events on the caller's stream (host memory only; no device allocation). */
gto_status gto_kernel_timing(gto_ctx* ctx, int enable);

/* Synchronises `stream`, adds up the recorded launches since the last call and clears the
 * record: total_ms[i] = summed device time of kernel i, launches[i] = how many.  Both
 * arrays are HOST arrays of GTO_K_COUNT entries. */
gto_status gto_kernel_times(gto_ctx* ctx, void* stream, double* total_ms, int64_t* launches);

/* ------------------------------------------------------------------------------------------
 * One decoding step over a draft tree (Sec. 2 of the paper: the target verifies the tree that
 * policy G built, in one forward pass under the tree's mask).
 *
 *   gto_kv_append       puts the keys and values of a chunk of new tokens into a paged cache,
 *                       with the rotation of their positions
 *   gto_tree_attention  attention of the chunk over the cache and over itself
 *   gto_verify_tree     which drafted tokens the target accepts, and the token after them
 *   gto_kv_commit       moves the accepted tokens' cache entries together
 *
 * A batch has S sequences.  Sequence s brings a chunk of n = q_start[s+1] - q_start[s] tokens;
 * kv_len[s] = L counts its cache entries, the chunk's among them, so the chunk owns entries
 * base .. L-1 with base = L - n.  Without a tree the chunk's tokens follow one another (one
 * token: plain decoding; many: a piece of a prompt).  With a tree the last n_nodes[s] tokens of
 * the chunk are the nodes of a draft tree in the order of gto_tree's node lists, and the
 * lead = n - n_nodes[s] tokens before them follow one another; the first level of the tree hangs
 * below the last of them (or, with lead = 0, below entry base - 1).
 * Entry t of sequence s lies in place t % page_size of page page_table[s][t / page_size].
 *
 * The functions take a gto_decode_ctx, which owns the workspace (for bf16 / fp16 caches with heads of 64 or 128 about
 * 20 / 39 MB, whatever the other sizes are) and a status word.  Calls
 * through one context share them: order them (one stream, events), and give every stream or
 * captured graph that may run at the same time a context of its own.  The calls can be
 * captured into a CUDA graph, which the context has to outlive; lengths, tables and trees are
 * read on the device at replay.
 * Every index is checked on the device before it is followed.  A sequence whose q_start, kv_len or
 * n_nodes contradict one another or the limits is reported (GTO_ERR_BAD_INDEX) and skipped; where
 * q_start decreases, so are all sequences from there on.  A page_table entry that names no page is
 * reported when it is needed: gto_kv_append leaves that token out, the rows of gto_tree_attention
 * that look there are unspecified, gto_kv_commit skips the sequence if one of its new entries would lie there. */

typedef struct gto_decode_ctx gto_decode_ctx;

enum {
  GTO_DECODE_ROPE_INTERLEAVED = 1u, /* rotate the pairs (2i, 2i+1) instead of (i, i + rope_dims/2) */
  GTO_DECODE_CONTEXT_ROWS = 2u /* gto_verify_tree reads target rows in the layout of
                                  gto_tree_reward, [S, R, V_target] with R = 1 + (D-1)k, through
                                  node_depth and node_slot; default: [S, 1+g, V_target], row 0
                                  after the root, row 1 + n after node n                        */
};

typedef struct {
  int32_t S;          /* most sequences of a call                                         */
  int32_t T;          /* most tokens of a call                                            */
  int32_t g;          /* nodes of a draft tree (row length of the node arrays); 0: none   */
  int32_t D;          /* most levels of a tree                                            */
  int32_t k;          /* frontier slots per level, with GTO_DECODE_CONTEXT_ROWS only       */
  int32_t n_q_heads, n_kv_heads, head_dim;  /* n_kv_heads = 0: no cache (verification only) */
  int32_t page_size, n_pages, max_pages;    /* entries of a page, pages, row of page_table  */
  int32_t kv_dtype;   /* gto_dtype of queries, keys, values, cache and output             */
  int32_t rope_dims;  /* leading dimensions of a head that are rotated; 0: none            */
  int32_t V_draft, V_target, logit_dtype;   /* V_target = 0: no verification               */
  float softmax_scale;
  float norm_eps;     /* epsilon of the optional query / key norms                         */
  uint32_t flags;
} gto_decode_config;

/* Device pointers of a batch. */
typedef struct {
  int32_t S, T;               /* sequences; tokens the token arrays have room for           */
  const int32_t* q_start;     /* [S+1] first token of every chunk; tokens from q_start[S] on
                                 belong to no sequence and are left alone                   */
  const int32_t* kv_len;      /* [S]                                                        */
  const int32_t* page_table;  /* [S, max_pages]                                             */
  const int32_t* n_nodes;     /* [S] tree nodes of each chunk, 0..g; NULL: g everywhere     */
  const uint64_t* node_mask;  /* [S, g, ceil(g/64)] as in gto_tree; NULL: no trees          */
  const int32_t* node_depth;  /* [S, g] as in gto_tree, for gto_kv_append; NULL: no trees   */
} gto_batch;

/* Paged keys and values.  Element (layer, page, entry, head, :) starts at the sum of the
 * indices times the strides; the head_dim values of a head are contiguous.  Strides count
 * elements, multiples of 16 bytes.  No two elements share memory, and the token arrays of a call share none
 * with the cache. */
typedef struct {
  void* k;
  void* v;
  int64_t k_page, k_entry, k_head, k_layer;
  int64_t v_page, v_entry, v_head, v_layer;
  int32_t n_layers;  /* gto_kv_commit works on all of them; the other calls on layer 0      */
} gto_kv_cache;

/* Trees to verify: arrays of gto_tree, restricted to the S trees (row length g). */
typedef struct {
  int32_t S;
  const int32_t* node_token;   /* [S, g] */
  const int32_t* node_parent;  /* [S, g] */
  const int32_t* node_depth;   /* [S, g] with GTO_DECODE_CONTEXT_ROWS, else NULL */
  const int32_t* node_slot;    /* [S, g] with GTO_DECODE_CONTEXT_ROWS, else NULL */
  const int32_t* n_nodes;      /* [S] nodes of each tree, 0..g; NULL: g */
} gto_draft_tree;

typedef struct {
  int32_t* accept_len;  /* [S] accepted drafted tokens; -1: a wait ran out (GTO_ERR_TIMEOUT), the
                           sequence's path_node and token are unspecified                   */
  int32_t* path_node;   /* [S, D] their list positions; -1 beyond accept_len                */
  int32_t* token;       /* [S, D+1] their target-vocabulary ids, then the token that follows
                           them (-1 if the last node has no target row); -1 beyond          */
} gto_verdict;

/* Limits: 0 <= g <= 128; 1 <= D <= 16; n_q_heads a multiple of n_kv_heads, at most 128 of
 * them per key head; head_dim a multiple of 16, at most 256; rope_dims a multiple of 16, at
 * most head_dim; max_pages * page_size <= 2^31 - 256; V * sizeof(logit) a multiple of 16 for the target
 * vocabulary and at most 1.5 MB; g <= V_draft <= V_target. */
gto_status gto_decode_create(gto_decode_ctx** ctx, const gto_decode_config* cfg, int device);
gto_status gto_decode_destroy(gto_decode_ctx* ctx);

/* Keys and values of the batch into the cache, queries rotated on the way.  q, k, v: rows of
 * n_heads * head_dim contiguous elements, row t at t * stride (elements, a multiple of 16
 * bytes: they may be slices of one projection); q_out: dense [T, n_q_heads, head_dim], may be
 * q itself where q is dense, and overlaps neither k nor v; q and q_out may both be NULL.  Token i of the lead has position
 * base + i, node a of the tree base + lead - 1 + node_depth[a].
 * q_norm / k_norm ([head_dim], kv_dtype, or NULL): the head is first scaled to unit mean
 * square and multiplied by the weights.  Then the pair (x_i, x_{i + rope_dims/2}) is rotated by
 * the angle position * inv_freq[i] (inv_freq: [rope_dims/2] fp64; the angle is formed in fp64,
 * so that far positions keep their phase).  Everything in fp32, rounded once.  Values are
 * copied.  No two tokens of the batch may own the same cache entry. */
gto_status gto_kv_append(gto_decode_ctx* ctx, const gto_batch* batch, const gto_kv_cache* cache,
                         const void* q, int64_t q_stride, const void* k, int64_t k_stride,
                         const void* v, int64_t v_stride, void* q_out, const double* inv_freq,
                         const void* q_norm, const void* k_norm, void* stream);

/* out[t] = sum over visible entries e of softmax_e(softmax_scale q_t . k_e) v_e, for every token
 * of the batch and every query head (query head h reads key head h / (n_q_heads / n_kv_heads)).
 * A token of the lead sees the entries up to its own; node a of a tree sees every entry before
 * the tree and the nodes in row a of node_mask.  A row that sees nothing gives zeros.  q as in
 * gto_kv_append; out: dense [T, n_q_heads, head_dim]; lse ([T, n_q_heads] fp32 or NULL) receives
 * the log-sum-exp of the row's scaled scores, -inf for a row that sees nothing.  Rows of tokens
 * that belong to no sequence are left as they were.  out and lse overlap neither q nor each other.  A
 * value (of v) that is not finite can make the outputs of a row that sees it not finite in all dimensions,
 * not in its own alone; rows that do not see it, and every lse, are not touched by it. */
gto_status gto_tree_attention(gto_decode_ctx* ctx, const gto_batch* batch, const gto_kv_cache* cache,
                              const void* q, int64_t q_stride, void* out, float* lse, void* stream);

/* Verification of drafted tokens against the target's probabilities.  The walk starts at the root.
 * At a context with target logits z let p = softmax(z / temperature[s]) and M = 1; the drafted
 * children x_1, x_2, ... of the context are tried in list order: child x is accepted if
 * u_node[x] * M < p(x), else p(x) is taken out: M -= p(x), p(x) = 0 (a child with the token of an
 * earlier one therefore cannot be accepted).  An accepted child becomes the context.  When none
 * is accepted the step's last token is drawn from what is left: the smallest id v with
 * sum_{w <= v} p(w) > u_bonus[s] * M.  The drafted tokens are point proposals (policy G takes
 * the k best, it does not sample), so the accepted tokens and the last one together follow the
 * target's distribution exactly.  temperature 0: a child is accepted if its token is the
 * arg-max (lowest id on ties), and the last token is the arg-max.
 * target: [S, 1+g, V_target] (see GTO_DECODE_CONTEXT_ROWS); d2t: [V_draft] or NULL (identity,
 * needs V_draft == V_target); temperature, u_bonus: [S] fp32; u_node: [S, g] fp32; the uniforms
 * are given by the caller, in [0, 1) (clamped to it).  The decisions are those of fp64 sums (a
 * row is first summed in fp32 with a bound on its error, and again in fp64 where a decision lies
 * within that bound of its border).  A sequence whose visited
 * rows hold NaN or +inf, or nothing but -inf, or whose temperature is negative or not finite,
 * is reported (GTO_ERR_NONFINITE); it keeps what was accepted before and gets the last token -1.  Where a
 * CTA of a sequence is not heard of within about two seconds, GTO_ERR_TIMEOUT is reported and the
 * sequence's accept_len is -1, which gto_kv_commit skips.  The arrays of *out overlap neither one another
 * nor what the call reads. */
gto_status gto_verify_tree(gto_decode_ctx* ctx, const gto_draft_tree* tree, const void* target,
                           const int32_t* d2t, const float* temperature, const float* u_node,
                           const float* u_bonus, const gto_verdict* out, void* stream);

/* Keeps the accepted nodes of every sequence: cache entry base + lead + path_node[s][j] is copied
 * to base + lead + j for j < accept_len[s], in all layers, and kv_len_out[s] = base + lead +
 * accept_len[s] (base + n for a sequence without a tree in this batch; untouched for one that is
 * skipped).  batch is the step's, T among it: a sequence that gto_kv_append skipped for lying behind its T
 * tokens is skipped here too.  kv_len_out overlaps neither batch->kv_len, which the whole call reads, nor
 * another table of the batch or the verdict.  path_node must
 * increase along the path, as gto_verify_tree writes it; a sequence where it does not, or whose accept_len is
 * negative or above D, is reported and skipped. */
gto_status gto_kv_commit(gto_decode_ctx* ctx, const gto_batch* batch, const gto_verdict* verdict,
                         const gto_kv_cache* cache, int32_t* kv_len_out, void* stream);

/* As gto_device_status and gto_launch_count, for a decoding context. */
gto_status gto_decode_status(gto_decode_ctx* ctx, void* stream, int32_t* host_code);
int64_t gto_decode_launch_count(const gto_decode_ctx* ctx);

const char* gto_status_string(gto_status s);

#ifdef __cplusplus
}
#endif
#endif /* GTO_H_ */
