/*
 * vecattn.h -- C ABI of libvecattn, vertical-vector sparse attention for
 * AMD Instinct MI355X (gfx950), after VecAttention (arXiv 2603.29494).
 *
 * The method has two stages (paper, Sec. 3 and appendix algorithms 1-2):
 *   1. vecattn_select: for every query block of P rows, pool the block's
 *      queries (Eq. 2), score every eligible key with the pooled query
 *      (estimated map A_p, Sec. 3.1.1) and keep the important key columns
 *      ("vertical vectors") by a budget (row-wise topK) or a cumulative-mass
 *      threshold (row-wise topP), Sec. 3.1.2, or the minS filter (Eq. 3), also
 *      with Algorithm 1's cross-tile running maximum (vecattn_select_mins_tiled).
 *      Output: the index matrix I and count vector C of Algorithm 1.
 *   2. vecattn_sparse_attn: attention of each query block restricted to the
 *      gathered K/V rows of its selected keys (Eq. 4, Algorithm 2).
 *
 * Conventions shared by every entry point
 *   - Tensors are caller-owned device memory.  The library never allocates,
 *     frees or synchronises; every call is asynchronous on `stream` (a
 *     hipStream_t; NULL means the default stream), and calls on different
 *     streams may run concurrently.  The only state kept between calls is a
 *     per-process, per-device locality counter of vecattn_sparse_attn (the
 *     progress of the workgroups on each XCD through their lists, which paces
 *     the order in which a workgroup walks its list; non-causal calls only):
 *     concurrent calls share it, which changes their speed and the order of
 *     the softmax sums (the last bits of O), never which keys are attended.
 *   - Q, K, V, O are bf16 with logical shape [B, H, N, D] described by a
 *     vecattn_tdesc: sizes plus element strides sB, sH, sN; the D dimension is
 *     contiguous (stride 1).  Every row start must be 16-byte aligned (base
 *     pointer 16-byte aligned, sB, sH, sN multiples of 8).  D must be 64 or 128.
 *   - Query heads Hq and key/value heads Hkv: Hq % Hkv == 0, and query head h
 *     reads key/value head h / (Hq / Hkv) (grouped-query attention).
 *   - Blocks: block = P >= 1 query rows; N_p = ceil(N / P); block i holds rows
 *     [i*P, min(N, (i+1)*P)) (the last block may be ragged).
 *   - I (idx) is int32 [B, Hq, N_p, cap], contiguous.  Row (b, h, i) lists the
 *     selected keys of block i in strictly ascending order in its first C[b,h,i]
 *     entries; the remaining entries are -1 (left unwritten with
 *     VECATTN_UNPADDED).  C (counts) is int32 [B, Hq, N_p].
 *   - Argument errors are detected on the host before any launch and return a
 *     status without touching memory.  Launch failures return
 *     VECATTN_ERR_DEVICE.
 */
#ifndef VECATTN_H
#define VECATTN_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum vecattn_status {
  VECATTN_OK = 0,
  VECATTN_ERR_INVALID_ARG = 1, /* null pointer, bad size/stride/alignment, bad parameter */
  VECATTN_ERR_UNSUPPORTED = 2, /* valid request this build does not implement (e.g. D=96) */
  VECATTN_ERR_CAPACITY = 3,    /* cap smaller than a topK budget, or workspace too small */
  VECATTN_ERR_DEVICE = 4       /* a HIP call or kernel launch failed */
} vecattn_status;

typedef enum vecattn_sel_mode {
  VECATTN_SEL_TOPK = 0, /* param = keep ratio r in (0, 1]: block i keeps
                           k_i = min(L_i, max(1, ceil(r * L_i - 1e-9))) keys */
  VECATTN_SEL_TOPP = 1, /* param = mass p in (0, 1]: block i keeps the shortest
                           prefix, in (score desc, index asc) order, whose softmax
                           mass over its eligible keys is >= p */
  VECATTN_SEL_MINS = 2, /* param = alpha >= 0 (Eq. 3, minS): block i keeps every
                           eligible key whose score is >= its largest score
                           minus alpha (alpha = +inf keeps all) */
  VECATTN_SEL_MINS_TILED = 3 /* param = alpha >= 0: minS against Algorithm 1's
                           cross-tile running maximum (Sec. 3.1.3), with the
                           paper's B_K = 16 keys per tile and G_K = 16 tiles per
                           group; see vecattn_select_mins_tiled */
} vecattn_sel_mode;

/* Bits of the `causal` argument of the selection entry points.  0 (none) and
 * 1 (VECATTN_CAUSAL) keep their plain meaning; bits other than these three are
 * invalid. */
#define VECATTN_CAUSAL 1    /* block i's eligible keys end at its last row */
#define VECATTN_KEEP_DIAG 2 /* block i also keeps the keys of its own rows,
                               [i*P, min(N, (i+1)*P)); cap must then cover
                               vecattn_select_max_count for the same flags in
                               every mode (no block is clamped) */
#define VECATTN_UNPADDED 4  /* the entries of I past a row's count are left as
                               they were instead of being set to -1 (the
                               attention and vecattn_check_lists read only the
                               first C entries): with a large cap (threshold
                               modes, cap = N) this saves writing the padding */

/* Of the `flags` of entry points that have them: the rows (or entries) of an output that
 * belong to no row (or token) of their sequence are written as 0 instead of being left as
 * they were. */
#define VECATTN_CLEAR_PADDING 8

typedef struct vecattn_tdesc {
  int64_t B, H, N, D; /* logical sizes */
  int64_t sB, sH, sN; /* element strides of the B, H and N dimensions */
} vecattn_tdesc;

/* Version of this ABI (major * 100 + minor). */
int32_t vecattn_version(void);

/* Human-readable name of a status code (static storage, never NULL). */
const char* vecattn_status_string(vecattn_status s);

/*
 * Query pooling, Eq. 2 (Sec. 3.1.1): qp[b, h, i, :] = bf16 rounding (nearest,
 * ties to even, applied once) of the exact mean of q's rows in block i.  The
 * ragged last block averages the rows it has.
 *   q  : bf16 [B, H, N, D] (qd)          qp : bf16 [B, H, N_p, D] (qpd, N = N_p)
 * Errors: INVALID_ARG for null pointers, block < 1, or qpd not matching
 * (B, H, N_p, D); UNSUPPORTED for D not in {64, 128}.
 */
vecattn_status vecattn_pool(const void* q, const vecattn_tdesc* qd, int32_t block, void* qp,
                            const vecattn_tdesc* qpd, void* stream);

/*
 * Largest number of keys any block can select, for sizing cap.  topK: max_i k_i
 * (with VECATTN_KEEP_DIAG: max_i min(L_i, k_i + n_i), n_i the rows of block i);
 * the other modes: max_i L_i, where L_i = N (non-causal) or min(N, (i+1)*P)
 * (causal).  `causal` takes the same bits as vecattn_select.
 * Errors: INVALID_ARG for N < 1, block < 1, out == NULL, or param outside the
 * mode's range.
 */
vecattn_status vecattn_select_max_count(int64_t N, int32_t block, int32_t causal, int32_t mode,
                                        double param, int64_t* out);

/*
 * Workspace bytes vecattn_select makes use of for these shapes (device memory
 * the caller allocates and passes in; contents need not be initialised).  The
 * size depends on B, Hq, Hkv (kd->H), N, D, block and mode, and for minS on
 * whether cap is below N; it does not depend on the causal bits.  Calls with
 * less are described at vecattn_select.
 * Errors: INVALID_ARG (a NULL pointer, block < 1, cap < 1, an unknown mode,
 * sizes < 1 or N > 2^30, Hq % Hkv != 0, D not in {64, 128}).
 */
vecattn_status vecattn_select_workspace_size(const vecattn_tdesc* qd, const vecattn_tdesc* kd,
                                             int32_t block, int32_t causal, int32_t mode,
                                             int64_t cap, size_t* bytes);

/* The same size as a return value (0 when vecattn_select_workspace_size would
 * return an error). */
size_t vecattn_select_workspace_bytes(const vecattn_tdesc* qd, const vecattn_tdesc* kd,
                                      int32_t block, int32_t mode, int64_t cap);

/*
 * Important-vector selection (Sec. 3.1; Algorithm 1's outputs I and C).
 *   q : bf16 [B, Hq, N, D]    k : bf16 [B, Hkv, N, D]
 *   causal : VECATTN_CAUSAL and/or VECATTN_KEEP_DIAG bits.  Block i's
 *   eligible keys are j in [0, N), or j in [0, min(N, (i+1)*P)) with
 *   VECATTN_CAUSAL.  With VECATTN_KEEP_DIAG the block's list is the union of
 *   the mode's selection and the keys of its own rows (a practical variant
 *   the paper leaves open: local keys always attended).  Scores are <Q_p[i], k_j> / sqrt(D)
 *   with Q_p from vecattn_pool, computed from bf16 products accumulated in
 *   fp32.  Ties in score are broken toward the lower key index.
 *   idx    : int32 [B, Hq, N_p, cap] output (ascending lists, -1 padded)
 *   counts : int32 [B, Hq, N_p] output
 *   n_clamped : optional device int32; when not NULL, the number of blocks
 *            whose threshold-mode selection exceeded cap is ADDED to it
 *            (topP and minS blocks keep their cap highest-scoring keys;
 *            cross-tile minS blocks their first cap keys).
 *   workspace : device memory (16-byte aligned), vecattn_select_workspace_size
 *            bytes for the best speed.  A call of at most 16384 tokens (topK,
 *            topP, minS) also runs in less, with the same lists (topP cuts whose
 *            mass is within fp32 rounding of p, and NaN scores, aside), but
 *            no less than
 *              align256(B * Hq * N_p * D * 2)
 *                + min(N_p, 64) * 4 * (N rounded up to a multiple of 32)
 *            (or than that size, if it is smaller); longer sequences and
 *            cross-tile minS need the whole size.
 * Errors: INVALID_ARG (null pointer, shape mismatch between q and k, block < 1,
 * param outside (0, 1] for topK / topP or negative / NaN for minS, cap < 1);
 * CAPACITY (topK with cap < max_i k_i, or a workspace that is too small);
 * UNSUPPORTED (D not in {64, 128}).
 */
vecattn_status vecattn_select(const void* q, const vecattn_tdesc* qd, const void* k,
                              const vecattn_tdesc* kd, int32_t block, int32_t causal, int32_t mode,
                              double param, int32_t* idx, int64_t cap, int32_t* counts,
                              int32_t* n_clamped, void* workspace, size_t workspace_bytes,
                              void* stream);

/*
 * vecattn_select without a caller workspace, for callers that cannot allocate
 * device memory (code under stream capture, tight serving loops, harnesses
 * that forbid allocation).  The workspace is a 64 MiB array inside the library
 * (VECATTN_STATIC_WORKSPACE_BYTES), one copy per GPU the library runs on, held
 * until the process ends; the call allocates nothing.  Arguments and results
 * are those of vecattn_select.  Every call on a GPU uses that GPU's one copy
 * (the current device's): calls that overlap on one GPU (other streams, other
 * threads) race and must be serialised by the caller.
 * Errors: as vecattn_select; CAPACITY when these shapes need a workspace of
 * more than VECATTN_STATIC_WORKSPACE_BYTES (the least vecattn_select accepts,
 * not the size query's); DEVICE if the array's device address cannot be
 * obtained.
 */
#define VECATTN_STATIC_WORKSPACE_BYTES (64u << 20)
vecattn_status vecattn_select_noalloc(const void* q, const vecattn_tdesc* qd, const void* k,
                                      const vecattn_tdesc* kd, int32_t block, int32_t causal,
                                      int32_t mode, double param, int32_t* idx, int64_t cap,
                                      int32_t* counts, int32_t* n_clamped, void* stream);

/*
 * Important-vector selection with Algorithm 1's cross-tile minS filter
 * (appendix Algorithm 1; Sec. 3.1.3, "Cross-tile minS optimization"; the rule
 * is Eq. 3's with a running maximum in place of the row maximum).  Block i's
 * eligible keys (as for vecattn_select) fall into groups of tile * group_tiles
 * consecutive keys, the first starting at key 0; inside a group the tiles of
 * `tile` keys are visited in ascending order, and a key of tile t is kept when
 * its score is >= (largest score in the group's tiles 0..t) - alpha.  Scores
 * are computed as for vecattn_select; alpha = +inf keeps every eligible key.
 *   tile        : B_K, 16 or 32 keys
 *   group_tiles : G_K, a power of two, tile * group_tiles <= 2^30 (a group
 *                 longer than N makes the running maximum span the whole row)
 *   idx, counts, workspace : as for vecattn_select (workspace size from
 *            vecattn_select_workspace_size with mode VECATTN_SEL_MINS_TILED)
 *   n_clamped : optional device int32; the number of blocks that selected more
 *            than cap keys is ADDED to it.  Such a block keeps its first cap
 *            selected keys in key order (the order in which Algorithm 1 appends
 *            its tiles) and reports count = cap.
 * vecattn_select with mode VECATTN_SEL_MINS_TILED equals this call with
 * tile = 16, group_tiles = 16.
 * Errors: INVALID_ARG (null pointer, shape mismatch, block < 1, cap < 1, alpha
 * negative or NaN, tile not 16 or 32, group_tiles not a power of two or too
 * large); CAPACITY (workspace too small); UNSUPPORTED (D not in {64, 128}).
 */
vecattn_status vecattn_select_mins_tiled(const void* q, const vecattn_tdesc* qd, const void* k,
                                         const vecattn_tdesc* kd, int32_t block, int32_t causal,
                                         double alpha, int32_t tile, int32_t group_tiles,
                                         int32_t* idx, int64_t cap, int32_t* counts,
                                         int32_t* n_clamped, void* workspace,
                                         size_t workspace_bytes, void* stream);

/*
 * vecattn_select with one parameter per query head: params[h] (host memory,
 * Hq values) replaces `param` for query head h -- e.g. the per-head filter
 * ratios of Eq. 5 (vecattn_plan_filter_ratios).  tile and group_tiles apply
 * to VECATTN_SEL_MINS_TILED as in vecattn_select_mins_tiled and are ignored by
 * the other modes.  The values are read during the call; the buffer may be
 * reused as soon as it returns.
 * Errors: as vecattn_select, each params[h] checked against the mode's range
 * (topK: CAPACITY when cap is below any head's budget); INVALID_ARG for
 * params == NULL or, for cross-tile minS, a bad tiling; UNSUPPORTED for more
 * than 128 query heads.
 */
vecattn_status vecattn_select_per_head(const void* q, const vecattn_tdesc* qd, const void* k,
                                       const vecattn_tdesc* kd, int32_t block, int32_t causal,
                                       int32_t mode, const double* params, int32_t tile,
                                       int32_t group_tiles, int32_t* idx, int64_t cap,
                                       int32_t* counts, int32_t* n_clamped, void* workspace,
                                       size_t workspace_bytes, void* stream);

/*
 * Vector-sparse attention, Eq. 4 (Sec. 3.2) and Algorithm 2.  For query row r
 * of block i (head h), the visible keys are V_r = { j in I[b,h,i,0:C[b,h,i]] :
 * causal == 0 or j <= r }, and
 *   o[r] = sum_{j in V_r} softmax_j(scale * <q_r, k_j>) v_j,
 *   lse[r] = log sum_{j in V_r} exp(scale * <q_r, k_j>)   (natural log).
 * A row with no visible key gets o[r] = 0 and lse[r] = -inf.
 *   q, o : bf16 [B, Hq, N, D]      k, v : bf16 [B, Hkv, N, D]
 *   idx, counts : as produced by vecattn_select (any source is accepted if
 *   every listed key is in [0, N) and the lists are strictly ascending;
 *   other contents are undefined behaviour).
 *   causal : the VECATTN_CAUSAL bit (VECATTN_KEEP_DIAG and VECATTN_UNPADDED are
 *   accepted and have no effect here; other bits are invalid).
 *   scale : softmax scale; 0 means 1 / sqrt(D).
 *   lse   : optional fp32 [B, Hq, N] contiguous output, may be NULL.
 * Errors: INVALID_ARG (null pointer, shape mismatch, block < 1, cap < 1,
 * misalignment); UNSUPPORTED (D not in {64, 128}; or a K or V head the
 * gathers cannot address with 32-bit offsets: N >= 2^24, a row stride sN of
 * 2^23 elements or more (with N > 1), or (N - 1) * sN * 2 + 2 * D >= 2^31
 * bytes -- e.g. a packed [B, N, 3, H, D] QKV view with H * D = 5120 from
 * N ~ 69,900 on).
 */
vecattn_status vecattn_sparse_attn(const void* q, const vecattn_tdesc* qd, const void* k,
                                   const vecattn_tdesc* kd, const void* v, const vecattn_tdesc* vd,
                                   const int32_t* idx, int64_t cap, const int32_t* counts,
                                   int32_t block, int32_t causal, float scale, void* o,
                                   const vecattn_tdesc* od, float* lse, void* stream);

/*
 * Block schedule for vecattn_sparse_attn_ordered.  Eq. 4 and Algorithm 2 treat
 * the query blocks independently, so the order in which the attention takes
 * them changes only its speed.  This call orders the N_p blocks of each
 * (b, h) by:
 *   1. count C[b,h,i], largest first (the longest lists start first, so the
 *      workgroups of a head finish together, and lists of like length, which
 *      walk the keys at a like pace, run side by side and share cache hits);
 *   2. then a signature: the mean of the entries at positions
 *      floor((2j + 1) * C / 16), j = 0..7, of the list (each clamped to
 *      [0, N - 1]), as floor(sum * 64 / N) capped at 511, smallest first;
 *   3. then the block index, smallest first.
 * A head of more than 16384 blocks is ordered in consecutive segments of
 * 16384 blocks, each segment by the rules above (positions [16384 s,
 * 16384 (s + 1)) hold a permutation of the same blocks).
 *   idx, cap, counts : as for vecattn_sparse_attn (counts are clamped to
 *            [0, cap]; only the 8 sampled entries of each list are read)
 *   B, Hq, N, block  : the selection's shapes; N_p = ceil(N / block)
 *   order  : int32 [B, Hq, N_p] device output; row (b, h) is a permutation of
 *            [0, N_p)
 * Asynchronous on `stream`; one read of counts and of the sampled entries.
 * Errors: INVALID_ARG (a NULL pointer, B, Hq, N or block < 1, N or cap
 * outside [1, 2^30], B * Hq > 2^31 - 1).
 */
vecattn_status vecattn_attn_order(const int32_t* idx, int64_t cap, const int32_t* counts,
                                  int64_t B, int32_t Hq, int64_t N, int32_t block, int32_t* order,
                                  void* stream);

/*
 * vecattn_sparse_attn taking the blocks of each (b, h) in a given order:
 *   order : int32 [B, Hq, N_p] device memory, row (b, h) a permutation of
 *           [0, N_p) (e.g. from vecattn_attn_order), or NULL for the
 *           ascending order (then this is vecattn_sparse_attn).  Entries are
 *           clamped to [0, N_p); a row that is not a permutation leaves the
 *           blocks missing from it unwritten.
 * Every other argument, the results and the errors are those of
 * vecattn_sparse_attn (the order of the softmax sums, and so the last bits
 * of O, can differ between calls, as there).
 */
vecattn_status vecattn_sparse_attn_ordered(const void* q, const vecattn_tdesc* qd, const void* k,
                                           const vecattn_tdesc* kd, const void* v,
                                           const vecattn_tdesc* vd, const int32_t* idx,
                                           int64_t cap, const int32_t* counts,
                                           const int32_t* order, int32_t block, int32_t causal,
                                           float scale, void* o, const vecattn_tdesc* od,
                                           float* lse, void* stream);

/*
 * Checker for the index input of vecattn_sparse_attn, for lists that did not
 * come from vecattn_select.  Sets *n_bad (device int32, cleared by the call)
 * to the number of rows whose list breaks the attention's contract: a count
 * outside [0, cap], or among the row's first `count` entries one outside
 * [0, n_keys) or one not strictly above the entry before it.  Entries past a
 * row's count are not read.
 *   idx    : int32 [rows, cap], contiguous (e.g. [B, Hq, N_p, cap] as rows =
 *            B * Hq * N_p)            counts : int32 [rows]
 *   n_keys : N of the keys the lists index
 * One read of the listed entries (4 bytes each); asynchronous on `stream`.
 * Errors: INVALID_ARG (n_bad NULL, idx or counts NULL with rows > 0, rows < 0
 * or > 2^31 - 1, cap < 1, n_keys < 1, cap or n_keys > 2^30).
 */
vecattn_status vecattn_check_lists(const int32_t* idx, int64_t rows, int64_t cap,
                                   const int32_t* counts, int64_t n_keys, int32_t* n_bad,
                                   void* stream);

/*
 * Variable-length batches.  Sequences of different lengths packed along N of
 * B = 1 tensors: sequence s is rows [cu_seqlens[s], cu_seqlens[s+1]) (host
 * int64, nseq + 1 values, cu_seqlens[0] = 0, non-decreasing, last = N; empty
 * sequences are allowed).  Each sequence is handled exactly as a separate
 * B = 1 call on its rows (its key indices count from its first row).  The
 * selections run one after another on `stream`; the attention takes up to 32
 * sequences per launch, the longest first.  Output layouts are the
 * per-sequence arrays laid end to end:
 *   idx    : int32, for each sequence [Hq, N_p(s), cap], N_p(s) = ceil(n_s / P)
 *   counts : int32, for each sequence [Hq, N_p(s)]
 *   lse    : fp32,  for each sequence [Hq, n_s] (optional)
 * Q, K, V, O rows are read and written in place (the [1, H, N, D] views).
 * The selection workspace is sized (vecattn_select_workspace_size) for the
 * longest sequence; what vecattn_select says of less holds for each one.
 * Every argument is checked for every sequence before the first launch.  Each
 * sequence costs the selection a set of launches of its own (three up to 16384
 * tokens, about 25 beyond).
 */
vecattn_status vecattn_select_varlen(const void* q, const vecattn_tdesc* qd, const void* k,
                                     const vecattn_tdesc* kd, const int64_t* cu_seqlens,
                                     int32_t nseq, int32_t block, int32_t causal, int32_t mode,
                                     double param, int32_t* idx, int64_t cap, int32_t* counts,
                                     int32_t* n_clamped, void* workspace, size_t workspace_bytes,
                                     void* stream);
vecattn_status vecattn_sparse_attn_varlen(const void* q, const vecattn_tdesc* qd, const void* k,
                                          const vecattn_tdesc* kd, const void* v,
                                          const vecattn_tdesc* vd, const int64_t* cu_seqlens,
                                          int32_t nseq, const int32_t* idx, int64_t cap,
                                          const int32_t* counts, int32_t block, int32_t causal,
                                          float scale, void* o, const vecattn_tdesc* od,
                                          float* lse, void* stream);

/*
 * Sparsity of each query head from a selection's counts: Eq. 5's sp_h
 * (Sec. 3.1.2), the table vecattn_plan_filter_ratios takes.
 *   sparsity[h] = 1 - (sum over b, i of counts[b, h, i]) / (B * sum_i L_i)
 * with L_i the eligible keys of block i (N, or min(N, (i + 1) * block) with
 * VECATTN_CAUSAL).  Integer sums, one fp64 division.
 *   counts   : int32 [B, Hq, N_p] (device, e.g. from vecattn_select)
 *   sparsity : fp64 [Hq] device output
 *   causal   : the selection's bits (VECATTN_KEEP_DIAG is accepted, no effect)
 * Errors: INVALID_ARG (NULL pointer, B, Hq or N < 1, N > 2^30, block < 1, bad
 * bits).
 */
vecattn_status vecattn_head_sparsity(const int32_t* counts, int64_t B, int64_t Hq, int64_t N,
                                     int32_t block, int32_t causal, double* sparsity,
                                     void* stream);

/*
 * Recall of a selected pattern, the statistic of the sparse-pattern study
 * (Sec. 2.2): for query row r of block i, the share of the row's exact
 * attention map that the block's list keeps,
 *   kept[b, h, r] = sum_{j in I[b,h,i,0:C) visible} exp(x_j) / sum_{j visible} exp(x_j),
 *   x_j = scale * <q_r, k_j>, visible = (j < N) and (causal == 0 or j <= r).
 * The mean of kept over rows is the recall of the pattern; 1 - keep ratio is
 * its sparsity.  One dense pass over the visible keys (2 * N * visible * D
 * MFMA FLOP per head), the list held as a bitmask in LDS.
 *   q : bf16 [B, Hq, N, D]   k : bf16 [B, Hkv, N, D]
 *   idx, counts, cap : as for vecattn_sparse_attn (entries outside [0, N) are
 *            ignored; a key listed twice counts once)
 *   scale : 0 means 1 / sqrt(D)
 *   kept  : fp32 [B, Hq, N] contiguous output
 * Errors: INVALID_ARG (null pointer, shape mismatch, block < 1, cap < 1, bad
 * scale or bits, misalignment); UNSUPPORTED (D not in {64, 128}, N > 2^18).
 */
vecattn_status vecattn_recall(const void* q, const vecattn_tdesc* qd, const void* k,
                              const vecattn_tdesc* kd, const int32_t* idx, int64_t cap,
                              const int32_t* counts, int32_t block, int32_t causal, float scale,
                              float* kept, void* stream);

/*
 * Attention with a sliding window and a few first keys that stay visible
 * (sinks), for the layers that look at a neighbourhood instead of a selection.
 * Row r of q is at position p = r + Nk - Nq (the queries are the last Nq rows of
 * the keys), and sees the keys
 *   V(p) = { j < L : (p - window < j and (causal ? j <= p : j < p + window))
 *                    or (j < sinks and (!causal or j <= p)) },
 * L = lens[b] or Nk:  o = sum over V(p) of softmax_j(scale * <q, k_j>) v_j, and
 * lse as for vecattn_sparse_attn.  A window of 1 is the row's own key; a window
 * (or sinks) of Nk or more is all of them.
 *   q, o : bf16 [B, Hq, Nq, D]     k, v : bf16 [B, Hkv, Nk, D], Nq <= Nk
 *   lens : optional int32 [B] device memory (clamped to [0, Nk]): the keys of
 *          sequence b that exist.  Rows at or past it are padding: they are not
 *          read, and their o and lse are left as they were.  NULL: all Nk.
 *   causal : the VECATTN_CAUSAL bit (other bits are invalid)
 *   scale  : 0 means 1 / sqrt(D)
 *   lse    : optional fp32 [B, Hq, Nq] contiguous output, may be NULL
 * A key outside a row's V(p) never reaches that row, whatever it holds.  The sums
 * are fp32: finite |V| up to 2^100 leaves finite rows finite.
 * Errors: INVALID_ARG (null pointer, shape mismatch, Nq > Nk, window < 1, sinks
 * < 0, bad scale or bits, misalignment); UNSUPPORTED (D not in {64, 128}, more
 * than 65535 sequences or query heads or 2^23 tiles of 128 rows in all, a K or V
 * row stride of 2^24 elements or more).
 */
vecattn_status vecattn_window_attn(const void* q, const vecattn_tdesc* qd, const void* k,
                                   const vecattn_tdesc* kd, const void* v, const vecattn_tdesc* vd,
                                   const int32_t* lens, int64_t window, int64_t sinks,
                                   int32_t causal, float scale, void* o, const vecattn_tdesc* od,
                                   float* lse, void* stream);

/*
 * A key/value cache in pages, held in 4 or 8 bits a value.  The tokens of a
 * sequence lie in pages of `page` tokens: table[b][c] is the page of tokens
 * [c * page, (c + 1) * page) of sequence b.  Every 64 values x of one token and
 * head (a group) are held as codes u and one pair (m, s) in bf16,
 *   m = min x,  s = bf16((max x - min x) / M),  u = min(M, rint((x - m) / s)),
 * M = 2^bits - 1, in fp32 steps, ties to even; they stand for m + s u.  A step
 * below 2^-100 is held as 0 (u = 0); a group with a NaN or an infinity, or whose
 * range is past fp32, stands for NaN.  4.5 or 8.5 bits a value.
 */
typedef struct vecattn_cache {
  void* data;    /* device memory, 16-byte aligned, vecattn_cache_size bytes; the
                    layout inside is the library's.  Contents need not be
                    initialised: only tokens below lens[b] are looked at */
  int64_t pages; /* pages held */
  int32_t H, D;  /* key/value heads; 64 or 128 */
  int32_t page;  /* tokens per page: a power of two, 32 to 1024 */
  int32_t bits;  /* 4 or 8 */
} vecattn_cache;

/*
 * Bytes of a cache (its data pointer is not looked at).
 * Errors: INVALID_ARG (null pointer, pages < 1, H < 1, a page size or bits other
 * than above, more than 2^62 bytes); UNSUPPORTED (D not in {64, 128}, H > 65535).
 */
vecattn_status vecattn_cache_size(const vecattn_cache* cache, size_t* bytes);

/*
 * Quantises the rows of k and v into the cache: the last rows of each sequence.
 *   k, v  : bf16 [B, H, n, D]
 *   table : int32 [B, cols] device memory.  An entry outside [0, pages) holds no
 *           page: its tokens are not written here, not read back by
 *           vecattn_cache_read, and not visible to vecattn_cache_attn (so pages
 *           that a window has left behind can be given away).  Tokens past
 *           cols * page are held nowhere either.
 *   lens  : int32 [B] device memory: tokens of each sequence, the new ones
 *           included (below 0: none; at most 2^30)
 *   n_new : optional int32 [B] device memory (clamped to [0, n]): the rows of
 *           sequence b that exist (a padded batch), rows [0, n_new[b]); NULL: all n.
 * Row r is written at position lens[b] - n_new[b] + r; rows at a position below 0
 * are skipped.  Tokens at other positions stay as they are.
 * Sequences of one call, and calls that may overlap, must not write the same
 * page (reading pages that several sequences share is fine).
 * Errors: INVALID_ARG (null pointer, shape mismatch between k, v and the cache,
 * cols < 1 or cols * page > 2^30, a bad cache, misalignment); UNSUPPORTED (D not
 * in {64, 128}, n > 2^28, more than 65535 sequences or heads).
 */
vecattn_status vecattn_cache_write(const void* k, const vecattn_tdesc* kd, const void* v,
                                   const vecattn_tdesc* vd, const vecattn_cache* cache,
                                   const int32_t* table, int64_t cols, const int32_t* lens,
                                   const int32_t* n_new, void* stream);

/*
 * The cache's tokens [start, start + N) of each sequence as bf16, m + s u rounded
 * once (e.g. a whole cached prompt for vecattn_select and vecattn_sparse_attn, which
 * take as many rows of q as of k; a part of one for vecattn_window_attn, whose
 * queries may be fewer than the keys).
 *   k, v : bf16 [B, H, N, D] outputs; row r is token start + r.  Rows of tokens
 *          at or past lens[b], and of tokens that no page holds, are left as they
 *          were.
 * Errors: as vecattn_cache_write (N > 2^28: UNSUPPORTED); INVALID_ARG for start
 * < 0 or > 2^30.
 */
vecattn_status vecattn_cache_read(const vecattn_cache* cache, const int32_t* table, int64_t cols,
                                  const int32_t* lens, int64_t start, void* k,
                                  const vecattn_tdesc* kd, void* v, const vecattn_tdesc* vd,
                                  void* stream);
/* vecattn_cache_read with every row of k and v written: 0 for tokens at or past lens[b]
 * and for those that no page holds. */
vecattn_status vecattn_cache_read_whole(const vecattn_cache* cache, const int32_t* table,
                                        int64_t cols, const int32_t* lens, int64_t start, void* k,
                                        const vecattn_tdesc* kd, void* v, const vecattn_tdesc* vd,
                                        void* stream);

/*
 * Attention of the last n tokens of each sequence over its cached tokens: one
 * token (decoding), a few (drafts), or a chunk of a prompt.  Row r of q is at
 * position p = lens[b] - n_new[b] + r and sees
 *   V(p) = { j <= p : j > p - window or j < sinks }, less the tokens that no
 * page holds; the values are m + s u, and o, lse as for vecattn_sparse_attn (a
 * row that sees nothing: o = 0, lse = -inf).  Rounded are only the softmax weights
 * before they meet V (bf16's 8 bits times V's steps; with more than 32 rows, n * Hq
 * / H, fp16's 11 bits, down to 2^-32 of the row's largest weight, and V's values to
 * as many, down to 2^-39 of the largest; lse is from what was not rounded)
 * and the output.  The sums are fp32: |q|, |K| and |V| up to 2^100.  The new tokens'
 * own K and V are in the cache already (vecattn_cache_write with the same lens).
 *   q, o   : bf16 [B, Hq, n, D], Hq a multiple of the cache's H
 *   table, cols, lens, n_new : as for vecattn_cache_write; rows at or past
 *            n_new[b] are left as they were
 *   window : >= 1 (2^30: everything)      sinks : >= 0
 *   scale  : 0 means 1 / sqrt(D)
 *   lse    : optional fp32 [B, Hq, n] contiguous output, may be NULL
 *   workspace : device memory (16-byte aligned) of at least
 *            vecattn_cache_attn_workspace_size bytes for the same qd, cache, cols,
 *            window and sinks (0: may be NULL); contents need not be initialised.
 *            Calls that may overlap need one each.
 * The result does not depend on the order of execution (no atomics).  What a
 * call does follows lens, n_new and table on the device, so that a captured call
 * can be replayed as they change.
 * Errors: as vecattn_cache_write; INVALID_ARG for window < 1, sinks < 0, a bad
 * scale, a misaligned workspace; CAPACITY (workspace too small); UNSUPPORTED
 * (sizes past the launch limits: B * Hq * n >= 2^24, or about 2^23 workgroups).
 */
vecattn_status vecattn_cache_attn_workspace_size(const vecattn_tdesc* qd,
                                                 const vecattn_cache* cache, int64_t cols,
                                                 int64_t window, int64_t sinks, size_t* bytes);
vecattn_status vecattn_cache_attn(const void* q, const vecattn_tdesc* qd,
                                  const vecattn_cache* cache, const int32_t* table, int64_t cols,
                                  const int32_t* lens, const int32_t* n_new, int64_t window,
                                  int64_t sinks, float scale, void* o, const vecattn_tdesc* od,
                                  float* lse, void* workspace, size_t workspace_bytes,
                                  void* stream);

/*
 * What new tokens' attention puts on each cached token, added up: the measure by which
 * a cache can drop what is not looked at.  For token j of a key/value head h,
 *   w[b,h,j] = sum over the rows r of q, and the query heads that read h, that see j, of
 *              exp(scale * <q_r, k_j> - lse_r),
 * with lse from vecattn_cache_attn over the same cache and sequences, and
 *   out[b,h,j] = w + decay * mass[b,h,j]      for tokens before the new ones,
 *   out[b,h,j] = w                            for the new ones (mass is not read),
 * j < lens[b].  A row whose lse is -inf adds nothing; a token that no page holds gets
 * w = 0.  Entries at or past lens[b] are left as they were.
 *   flags : 0 or VECATTN_CLEAR_PADDING
 *   q, table, cols, lens, n_new, window, sinks, scale : as for vecattn_cache_attn
 *   lse  : fp32 [B, Hq, n] contiguous
 *   mass : optional fp32 [B, H, M] contiguous; NULL: 0.  May be out itself.
 *   out  : fp32 [B, H, M] contiguous; tokens at or past M have no entry, and what is put on
 *          them is not kept: M is best the tokens of the table
 *   workspace : device memory (16-byte aligned) of at least
 *          vecattn_cache_mass_workspace_size bytes for the same qd and cache (0, with up to
 *          48 rows n * Hq / H: may be NULL); contents need not be initialised.  Calls that
 *          may overlap need one each.
 * Sums are fp32, of one order (no atomics).  What a call does follows lens, n_new and table
 * on the device, so that a captured call can be replayed as they change.
 * Errors: as vecattn_cache_attn; INVALID_ARG for M < 1 or > 2^30, a decay that is negative
 * or not finite, or other flags.
 */
vecattn_status vecattn_cache_mass_workspace_size(const vecattn_tdesc* qd,
                                                 const vecattn_cache* cache, size_t* bytes);
vecattn_status vecattn_cache_mass(const void* q, const vecattn_tdesc* qd, const float* lse,
                                  const vecattn_cache* cache, const int32_t* table, int64_t cols,
                                  const int32_t* lens, const int32_t* n_new, int64_t window,
                                  int64_t sinks, float scale, float decay, const float* mass,
                                  float* out, int64_t M, int32_t flags, void* workspace,
                                  size_t workspace_bytes, void* stream);

/*
 * Which tokens of each sequence and head a budget keeps.  Candidates are the tokens
 * j < min(lens[b], M) that a page holds; kept are min(budget, candidates) of them: those
 * with j < sinks or j >= lens[b] - recent first, then by mass, the largest first, equal
 * ones the lower index first (-0 equals 0; a NaN comes after all others).
 *   mass : fp32 [B, H, M] contiguous        cache : its pages, H and page size
 *   table, cols, lens : as for vecattn_cache_write
 *   idx  : int32 [B, H, budget] output, ascending, -1 past the kept ones
 *   kept : int32 [B] output, how many (the same for every head): lens of the pages
 *          that vecattn_cache_gather fills
 *   workspace : device memory (16-byte aligned) of at least
 *          vecattn_cache_keep_workspace_size bytes for the same cache, cols, B and M (0 for
 *          up to 32768 tokens: may be NULL); contents need not be initialised.  Calls that
 *          may overlap need one each.
 * Asynchronous; one launch for up to 32768 tokens (M, or cols * page), six for more.
 * Errors: INVALID_ARG (null pointer, B < 1, M or budget < 1 or > 2^30, sinks or recent
 * < 0, sinks + recent > budget, a bad cache, cols < 1 or cols * page > 2^30, misalignment);
 * CAPACITY (workspace too small); UNSUPPORTED (more than 65535 sequences or heads).
 */
vecattn_status vecattn_cache_keep_workspace_size(const vecattn_cache* cache, int64_t cols,
                                                 int64_t B, int64_t M, size_t* bytes);
vecattn_status vecattn_cache_keep(const float* mass, int64_t M, int64_t B,
                                  const vecattn_cache* cache, const int32_t* table, int64_t cols,
                                  const int32_t* lens, int64_t budget, int64_t sinks,
                                  int64_t recent, int32_t* idx, int32_t* kept, void* workspace,
                                  size_t workspace_bytes, void* stream);

/*
 * Moves chosen tokens, per head, into other pages: slot i < kept[b] of sequence b and
 * head h takes token idx[b,h,i] of the same sequence and head, codes and (m, s) as they
 * are.  Keys keep the rotary positions they were written with; a window of
 * vecattn_cache_attn counts slots.
 *   idx, kept : as from vecattn_cache_keep (any indices are accepted, in any order; one
 *          that is negative or of a token that no page holds leaves a slot that stands for
 *          NaN; kept is clamped to [0, budget])
 *   to, to_table, to_cols : the cache (it may be the same one) and pages that take the
 *          tokens.  No page of to_table may be one that this call reads.  Slots whose
 *          entry names no page are not written; what the written pages' blocks of 32 slots
 *          held past kept[b] is lost.
 *   mass : optional fp32 [B, H, M] contiguous; with mass_out, fp32 [B, H, budget]
 *          contiguous: mass_out[b,h,i] = mass[b,h,idx[b,h,i]] for i < kept[b] (NaN for an
 *          index outside [0, M)), the rest left as it was.  Both or neither.
 *   flags : 0 or VECATTN_CLEAR_PADDING (of mass_out)
 * Asynchronous, one launch.
 * Errors: INVALID_ARG (null pointer, other flags, one of mass and mass_out alone, B < 1,
 * budget or M < 1 or > 2^30, caches of other heads, D or bits, a bad cache, cols or to_cols
 * < 1 or more than 2^30 tokens); UNSUPPORTED (more than 65535 sequences or heads, or a
 * budget past 2^29).
 */
vecattn_status vecattn_cache_gather(const vecattn_cache* cache, const int32_t* table, int64_t cols,
                                    int64_t B, const int32_t* idx, const int32_t* kept,
                                    int64_t budget, const vecattn_cache* to,
                                    const int32_t* to_table, int64_t to_cols, const float* mass,
                                    int64_t M, float* mass_out, int32_t flags, void* stream);
/* vecattn_cache_gather with mass_out fp32 [B, H, M_out], M_out from budget to 2^30, so that
 * tokens that are written behind the kept ones have an entry in it: what
 * vecattn_cache_mass and vecattn_cache_keep then take as [B, H, M]. */
vecattn_status vecattn_cache_gather_wide(const vecattn_cache* cache, const int32_t* table,
                                         int64_t cols, int64_t B, const int32_t* idx,
                                         const int32_t* kept, int64_t budget,
                                         const vecattn_cache* to, const int32_t* to_table,
                                         int64_t to_cols, const float* mass, int64_t M,
                                         float* mass_out, int64_t M_out, int32_t flags,
                                         void* stream);

/*
 * Attention of rows over another sequence's keys, such as an encoder's states (encoded
 * text under a video layer, encoded frames under a decoder): every row sees the keys
 *   V(b) = { j < lens[b] : mask[b][j] != 0 },
 * o and lse as for vecattn_sparse_attn (where V(b) is empty: o = 0, lse = -inf).
 *   q, o : bf16 [B, Hq, Nq, D]     k, v : bf16 [B, Hkv, Nk, D], any Nq and Nk
 *   lens : optional int32 [B] device memory (clamped to [0, Nk]); NULL: all Nk.  Keys at
 *          or past it are not read.
 *   mask : optional bytes [B, Nk] device memory, mask_sB from one sequence to the next
 *          (0: one for all); what a masked key holds, NaN and infinities too, reaches no row
 *   n_q  : optional int32 [B] device memory (clamped to [0, Nq]): the rows of sequence b
 *          that exist; those past it are left as they were.  NULL: all Nq.
 *   flags : 0 or VECATTN_CLEAR_PADDING
 *   scale : 0 means 1 / sqrt(D)
 *   lse  : optional fp32 [B, Hq, Nq] contiguous output, may be NULL
 *   workspace : device memory (16-byte aligned) of at least
 *          vecattn_cross_attn_workspace_size bytes for the same qd and kd (0: may be
 *          NULL); contents need not be initialised.  Calls that may overlap need one each.
 * Scores and sums are fp32, the weights bf16 before they meet V (off by 2^-8 of a weight at
 * most), or, of up to 16 rows Nq * Hq / Hkv, two bf16 that add up to them (2^-16).  Finite |V|
 * up to 2^90 leaves finite rows finite.  The result does not depend on the order of
 * execution (no atomics).  What a call does follows lens, mask and n_q on the device, so
 * that a captured call can be replayed as they change.
 * Errors: INVALID_ARG (null pointer, shape mismatch, Hq % Hkv != 0, mask_sB < 0, a bad
 * scale, other flags, an output whose sequences or heads share memory, misalignment);
 * CAPACITY (workspace too small); UNSUPPORTED (D not in {64, 128}, Nq * Hq / Hkv > 2^30, more
 * than 2^24 sequences times Hkv, about 2^23 workgroups, a K or V row stride of 2^24 elements
 * or more).
 */
vecattn_status vecattn_cross_attn_workspace_size(const vecattn_tdesc* qd, const vecattn_tdesc* kd,
                                                 size_t* bytes);
vecattn_status vecattn_cross_attn(const void* q, const vecattn_tdesc* qd, const void* k,
                                  const vecattn_tdesc* kd, const void* v, const vecattn_tdesc* vd,
                                  const int32_t* lens, const uint8_t* mask, int64_t mask_sB,
                                  const int32_t* n_q, int32_t flags, float scale, void* o,
                                  const vecattn_tdesc* od, float* lse, void* workspace,
                                  size_t workspace_bytes, void* stream);

/*
 * Rotary positions: pairs (a, b) of a row's first `rot` values are turned by the angle
 * t = position * frequency of the pair,
 *   a' = factor * (a cos t - b sin t),   b' = factor * (a sin t + b cos t);
 * transposed, t is -t (with the same factor: the gradient of the turn, and with factor 1
 * its inverse).  Values past rot stay as they are, bit for bit.
 */
#define VECATTN_ROPE_TRANSPOSED 1

typedef enum vecattn_rope_layout {
  VECATTN_ROPE_HALF = 0,       /* pair i is values i and i + rot / 2 */
  VECATTN_ROPE_INTERLEAVED = 1 /* pair i is values 2 i and 2 i + 1 */
} vecattn_rope_layout;

typedef enum vecattn_rope_scaling { /* for contexts longer than the trained one */
  VECATTN_ROPE_NONE = 0,   /* f_i = base^(-2 i / rot) */
  VECATTN_ROPE_LINEAR = 1, /* f_i / factor */
  VECATTN_ROPE_NTK = 2,    /* base * factor^(rot / (rot - 2)) in place of base: the lowest
                              frequency divided by factor, the highest as it was */
  VECATTN_ROPE_PARTS = 3,  /* pairs up to the one that makes `fast` turns over `context`
                              keep f_i, from the one that makes `slow` on f_i / factor, those
                              between (both rounded outwards, to no less than 0; the second,
                              which may lie past the last pair, to no more than rot - 1) a
                              share of each that is linear in i; the turned values times
                              0.1 ln(factor) + 1 */
  VECATTN_ROPE_BANDS = 4   /* the same, but the share is linear in the turns c f_i / 2 pi */
} vecattn_rope_scaling;

typedef struct vecattn_rope_spec {
  int32_t rot;         /* values turned: even, 2 to D */
  int32_t layout;      /* vecattn_rope_layout */
  int32_t axes;        /* positions per token, 1 to 4 (e.g. time, height, width) */
  int32_t flags;       /* VECATTN_ROPE_TRANSPOSED and VECATTN_CLEAR_PADDING bits */
  double factor;
  const double* freq;  /* host memory, rot / 2 frequencies in radians per position */
  const int32_t* axis; /* host memory, rot / 2: which position turns each pair; NULL: the
                          first */
} vecattn_rope_spec;

/*
 * A ladder of frequencies (host function, no GPU) for vecattn_rope_spec.
 *   fast, slow, context : of PARTS and BANDS (not read by the others); factor : of all but
 *          NONE
 *   freq : double [rot / 2] output       mfactor : output, factor for the spec
 * Errors: INVALID_ARG (null output, rot odd or outside [2, 128], base <= 1, an unknown
 * scaling, factor < 1, context <= 0, slow <= 0, fast <= slow, anything not finite).
 */
vecattn_status vecattn_rope_ladder(int32_t rot, double base, int32_t scaling, double factor,
                                   double context, double fast, double slow, double* freq,
                                   double* mfactor);

/*
 * Turns the rows of q, and of k if it is not NULL, by their positions.
 *   q, qo : bf16 [B, Hq, N, D]      k, ko : bf16 [B, Hkv, N, D], both NULL or neither
 *           (kd and kod too).  An output may be its input (the same pointer and strides); the
 *           tensors must not overlap otherwise.
 *   spec  : read during the call
 *   positions of row r of sequence b, one of:
 *     pos  : int32 device memory, pos[axis * pos_sA + b * pos_sB + r] (strides in
 *            elements, >= 0; 0 shares one row of positions)
 *     lens : int32 [B] device memory, lens[b] - n_new[b] + r on every axis, as
 *            vecattn_cache_write places rows
 *     neither: start + r on every axis
 *   n_new : optional int32 [B] device memory (clamped to [0, N]): the rows of sequence b
 *           that exist; those past it are left as they were.  NULL: all N.
 * Angles are taken in 64 bits (off by 2^-51 of the angle), sines and cosines of what is left
 * of a quarter turn in fp32, so that they are good to fp32 for angles up to 2^28 radians, and a
 * result is rounded to bf16 once.  Asynchronous, one launch.
 * Errors: INVALID_ARG (null pointer, shape mismatch, both pos and lens, |start| > 2^30,
 * a bad stride, a spec outside what its comments allow, a factor or frequency that is not
 * finite, |frequency| > 1024, an output that is its input with other strides or whose
 * sequences or heads share memory (a stride of 0), misalignment); UNSUPPORTED (D not in
 * {64, 128}, more than 65535 heads in all, B * N > 2^30).
 */
vecattn_status vecattn_rope(const void* q, const vecattn_tdesc* qd, const void* k,
                            const vecattn_tdesc* kd, const vecattn_rope_spec* spec,
                            const int32_t* pos, int64_t pos_sA, int64_t pos_sB,
                            const int32_t* lens, const int32_t* n_new, int64_t start, void* qo,
                            const vecattn_tdesc* qod, void* ko, const vecattn_tdesc* kod,
                            void* stream);

/*
 * Per-head filter ratios, Eq. 5 (Sec. 3.1.2).  Host function (host memory, no
 * GPU).
 * For each of `heads` heads, n_cand candidate filter ratios were sampled
 * offline with their sparsity sp[h][c] in [0, 1] and a performance score
 * perf[h][c] (any finite value, larger is better).  The call picks one
 * candidate per head so that the mean sparsity over the heads is >= target
 * and the summed performance is largest: Eq. 5's table over heads and
 * sparsity, kept as the summed sparsity with each sp[h][c] rounded to a
 * multiple of 1 / grid.  Ties go to the lower candidate index.
 *   sparsity, perf : double [heads][n_cand], row-major
 *   choice         : int32 [heads] output, the chosen candidate per head
 *   best_perf      : output, the summed performance of that choice
 * Errors: INVALID_ARG (null pointer, heads or n_cand < 1, target outside
 * [0, 1], sparsity outside [0, 1] or non-finite perf, grid < 1 or
 * heads * grid > 2^26); CAPACITY (no choice reaches the target).
 */
vecattn_status vecattn_plan_filter_ratios(int32_t heads, int32_t n_cand, const double* sparsity,
                                          const double* perf, double target, int32_t grid,
                                          int32_t* choice, double* best_perf);

#ifdef __cplusplus
}
#endif

#endif /* VECATTN_H */
