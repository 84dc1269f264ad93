// Internal launch interface between the C ABI (vecattn_api.cpp) and the HIP
// kernels.  Arguments are already validated by the caller.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace vecattn {

struct Tensor4 {
  const void* ptr;
  int64_t B, H, N, D;
  int64_t sB, sH, sN;
};

hipError_t launch_pool(const Tensor4& q, int32_t block, void* qp, int64_t qp_sB, int64_t qp_sH,
                       int64_t qp_sN, hipStream_t stream);

struct SparseAttnArgs {
  Tensor4 q, k, v;
  void* o;
  int64_t o_sB, o_sH, o_sN;
  float* lse;
  const int32_t* idx;
  const int32_t* counts;
  int64_t cap;
  int32_t block;
  int32_t causal;
  float scale;
  const int32_t* order;  // [B, Hq, N_p] block order per (b, h), or NULL (ascending)
};

hipError_t launch_sparse_attn(const SparseAttnArgs& a, hipStream_t stream);

// Packed sequences: a's tensors hold all rows, sequence s the rows
// [cu[s], cu[s + 1]) of them; lists, counts and LSE lie sequence after sequence
// (B = 1, no block order).
hipError_t launch_sparse_attn_varlen(const SparseAttnArgs& a, const int64_t* cu, int32_t nseq,
                                     hipStream_t stream);

// Block order per (b, h) for the attention: blocks sorted by count (largest
// first), then by a sampled mean key, then by index, within consecutive
// segments of kOrderMaxBlocks blocks.  rows = B * Hq (fits the grid).
constexpr int32_t kOrderMaxBlocks = 16384;
hipError_t launch_attn_order(const int32_t* idx, int64_t cap, const int32_t* counts, int64_t rows,
                             int32_t Np, int64_t N, int32_t* order, hipStream_t stream);

struct SelectArgs {
  Tensor4 q, k;
  int32_t block;
  int32_t causal;
  int32_t keep_diag;  // every block also keeps the keys of its own rows
  int32_t unpadded;   // entries past a row's count are left unwritten
  int32_t mode;
  double param;
  const double* head_params;  // NULL, or one parameter per query head (host memory, Hq <= 128)
  int32_t tile;         // cross-tile minS: keys per tile (16 or 32)
  int32_t group_tiles;  // cross-tile minS: tiles per group (a power of two)
  int32_t* idx;
  int64_t cap;
  int32_t* counts;
  int32_t* n_clamped;
  void* workspace;
  size_t workspace_bytes;
};

// The library's own selection workspace (one copy per GPU, for callers that
// cannot allocate): its size, and this GPU's copy (the current device's).
constexpr size_t kStaticWorkspaceBytes = size_t(64) << 20;
hipError_t static_workspace(void** ptr);

// Selection of short sequences (select_short.hip): whether a call may take it,
// the least workspace it needs (one row tile's scores), and the workspace it
// makes use of.  The row kernel holds a row in the registers of at most eight
// waves, 32 keys a lane (64 spilled: 288 us for 2700 rows of 12k tokens), which
// sets the longest row; below it launch_select takes the faster kind.
constexpr int64_t kShortMaxN = 16384;
bool short_select_ok(int64_t N, int32_t mode);
size_t short_select_min_bytes(int64_t B, int64_t Hq, int64_t N, int64_t D, int32_t block);
size_t short_select_bytes(int64_t B, int64_t Hq, int64_t N, int64_t D, int32_t block);
hipError_t launch_select_short(const SelectArgs& a, hipStream_t stream);

// Workspace the size query reports, and the least that a call accepts (a short
// sequence can be done by either kind of selection, so the smaller of the two;
// a call takes the kind that fits, or the faster one if both do).
size_t select_workspace_bytes(int64_t B, int64_t Hq, int64_t Hkv, int64_t N, int64_t D,
                              int32_t block, int32_t mode, int64_t cap);
size_t select_min_workspace_bytes(int64_t B, int64_t Hq, int64_t Hkv, int64_t N, int64_t D,
                                  int32_t block, int32_t mode);
hipError_t launch_select(const SelectArgs& a, hipStream_t stream);

// Rows whose list breaks the attention's input contract, counted into *n_bad
// (cleared first).  rows <= 2^31 - 1 fits the grid.
hipError_t launch_check_lists(const int32_t* idx, const int32_t* counts, int64_t rows, int64_t cap,
                              int64_t n_keys, int32_t* n_bad, hipStream_t stream);

// Sparsity per query head from the counts of a selection (Eq. 5's sp_h):
// sparsity[h] = 1 - sum_{b,i} C[b,h,i] / (B * sum_i L_i), as fp64.
hipError_t launch_head_sparsity(const int32_t* counts, int64_t B, int64_t Hq, int64_t N,
                                int32_t block, int32_t causal, double* sparsity,
                                hipStream_t stream);

// Attention mass each query row's block list keeps (the recall of Sec. 2.2):
// kept[b,h,r] = sum over the listed visible keys of the row's softmax over
// all its visible keys.  N <= kRecallMaxN.
constexpr int64_t kRecallMaxN = int64_t(1) << 18;
struct RecallArgs {
  Tensor4 q, k;
  const int32_t* idx;
  const int32_t* counts;
  int64_t cap;
  int32_t block;
  int32_t causal;
  float scale;
  float* kept;
};
hipError_t launch_recall(const RecallArgs& a, hipStream_t stream);

// Attention with a sliding window and sinks.  Row r of q is at position
// r + k.N - q.N; lens (int32 [B], or NULL) bounds each sequence's keys and rows.
constexpr int32_t kWindowRows = 128;  // query rows per workgroup
struct WindowArgs {
  Tensor4 q, k, v;
  void* o;
  int64_t o_sB, o_sH, o_sN;
  float* lse;
  const int32_t* lens;
  int64_t window, sinks;
  int32_t causal;
  float scale;
};
hipError_t launch_window_attn(const WindowArgs& a, hipStream_t stream);

// The quantised key/value cache and the pages of a batch of sequences.
struct CacheArgs {
  void* data;
  int64_t pages;
  int32_t H, D, page, bits;
  const int32_t* table;  // [B, cols] pages
  int64_t cols;
  const int32_t* lens;   // [B] tokens held
};
hipError_t launch_cache_write(const Tensor4& k, const Tensor4& v, const CacheArgs& c,
                              const int32_t* n_new, hipStream_t stream);
// clear: rows of tokens that are not held become 0.
hipError_t launch_cache_read(const CacheArgs& c, int64_t start, const Tensor4& k, const Tensor4& v,
                             bool clear, hipStream_t stream);

// Attention over the cache.  How the work is dealt out, and so the workspace,
// follows from the shape.
struct CacheAttnShape {
  int64_t B, Hq, H, n, D;
  int64_t cols, page, window, sinks;
};
struct CacheAttnArgs {
  CacheAttnShape shape;
  Tensor4 q;
  CacheArgs cache;
  const int32_t* n_new;
  void* o;
  int64_t o_sB, o_sH, o_sN;
  float* lse;
  float scale;
  void* workspace;
};
bool cache_attn_grid_ok(const CacheAttnShape& s);
size_t cache_attn_workspace_bytes(const CacheAttnShape& s);
hipError_t launch_cache_attn(const CacheAttnArgs& a, hipStream_t stream);

// The attention weight that rows of q put on cached tokens, added up per token, and
// eviction by it: which tokens a budget keeps, and these into other pages.
struct CacheMassArgs {
  Tensor4 q;
  const float* lse;
  CacheArgs cache;
  const int32_t* n_new;
  int64_t window, sinks;
  float scale, decay;
  const float* mass;   // [B, H, M], or NULL
  float* out;          // [B, H, M]
  int64_t M;
  bool clear;          // entries past a sequence's tokens become 0
  void* workspace;
};
size_t cache_mass_workspace_bytes(const CacheAttnShape& s);
hipError_t launch_cache_mass(const CacheMassArgs& a, hipStream_t stream);
size_t cache_keep_workspace_bytes(const CacheArgs& c, int64_t B, int64_t M);
hipError_t launch_cache_keep(const CacheArgs& c, int64_t B, const float* mass, int64_t M,
                             int64_t budget, int64_t sinks, int64_t recent, int32_t* idx,
                             int32_t* kept, void* workspace, hipStream_t stream);
hipError_t launch_cache_gather(const CacheArgs& c, const CacheArgs& to, int64_t B,
                               const int32_t* idx, const int32_t* kept, int64_t budget,
                               const float* mass, int64_t M, float* mass_out, int64_t M_out,
                               bool clear, hipStream_t stream);

// Attention over an encoder's states.  How the work is dealt out, and so the
// workspace, follows from the shape.
struct CrossArgs {
  Tensor4 q, k, v;
  void* o;
  int64_t o_sB, o_sH, o_sN;
  float* lse;
  const int32_t* lens;
  const uint8_t* mask;
  int64_t mask_sB;
  const int32_t* n_q;
  bool clear;      // rows past n_q become 0
  float scale;
  void* workspace;
};
constexpr int32_t kCrossRows = 128;   // rows per workgroup, where there are many
bool cross_attn_grid_ok(int64_t B, int64_t Hq, int64_t Hkv, int64_t Nq, int64_t Nk, int64_t D);
size_t cross_attn_workspace_bytes(int64_t B, int64_t Hq, int64_t Hkv, int64_t Nq, int64_t Nk,
                                  int64_t D);
hipError_t launch_cross_attn(const CrossArgs& a, hipStream_t stream);

// Rotary positions of q and, where k.ptr is not NULL, of k.
constexpr int32_t kRopeMaxPairs = 64;
struct RopeArgs {
  Tensor4 q, k, qo, ko;
  int32_t rot;
  bool half, transposed, clear;   // clear: rows past n_new become 0
  double factor;
  const double* freq;    // host, [rot / 2], radians per position
  const int32_t* axis;   // host, [rot / 2], or NULL: axis 0
  const int32_t* pos;    // positions, or NULL: from lens, or start + row
  int64_t pos_sA, pos_sB;
  const int32_t *lens, *n_new;
  int64_t start;
};
hipError_t launch_rope(const RopeArgs& a, hipStream_t stream);

// Host: a ladder of frequencies, also of the forms for long contexts.
void rope_ladder(int32_t rot, double base, int32_t scaling, double factor, double context,
                 double fast, double slow, double* freq, double* mfactor);

// Host: per-head filter ratios by dynamic programming (Eq. 5).  Returns 0, or
// 1 when no choice reaches the target.
int plan_filter_ratios(int32_t H, int32_t C, const double* sp, const double* perf, double target,
                       int32_t grid, int32_t* choice, double* best);

}  // namespace vecattn
