// C ABI of libvecattn: argument validation and dispatch to the HIP kernels.
// Every check happens on the host before any launch; see include/vecattn.h for
// the contract of each entry point.
#include "vecattn.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "launch.h"

namespace {

using vecattn::Tensor4;

constexpr int64_t kMaxN = int64_t(1) << 30;

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// Sizes positive, D contiguous, rows 16-byte aligned.
vecattn_status check_desc(const void* ptr, const vecattn_tdesc* d) {
  if (!ptr || !d) return VECATTN_ERR_INVALID_ARG;
  if (d->B < 1 || d->H < 1 || d->N < 1 || d->D < 1 || d->N > kMaxN) return VECATTN_ERR_INVALID_ARG;
  if (d->sB < 0 || d->sH < 0 || d->sN < d->D) return VECATTN_ERR_INVALID_ARG;
  if ((d->sB % 8) || (d->sH % 8) || (d->sN % 8) || !aligned16(ptr)) return VECATTN_ERR_INVALID_ARG;
  if (d->D != 64 && d->D != 128) return VECATTN_ERR_UNSUPPORTED;
  return VECATTN_OK;
}

Tensor4 to_tensor(const void* p, const vecattn_tdesc* d) {
  return Tensor4{p, d->B, d->H, d->N, d->D, d->sB, d->sH, d->sN};
}

int64_t num_blocks(int64_t N, int32_t P) { return (N + P - 1) / P; }

int64_t topk_count(double ratio, int64_t L) {
  int64_t k = static_cast<int64_t>(std::ceil(ratio * static_cast<double>(L) - 1e-9));
  if (k < 1) k = 1;
  if (k > L) k = L;
  return k;
}

bool mode_ok(int32_t mode) {
  return mode == VECATTN_SEL_TOPK || mode == VECATTN_SEL_TOPP || mode == VECATTN_SEL_MINS ||
         mode == VECATTN_SEL_MINS_TILED;
}

bool param_ok(int32_t mode, double param) {
  if (mode == VECATTN_SEL_TOPK || mode == VECATTN_SEL_TOPP) return param > 0.0 && param <= 1.0;
  if (mode == VECATTN_SEL_MINS || mode == VECATTN_SEL_MINS_TILED) return param >= 0.0;
  return false;
}

// Tile of 16 or 32 keys; a power-of-two number of tiles per group, at most
// 2^30 keys per group.
bool tiling_ok(int32_t tile, int32_t group_tiles) {
  if (tile != 16 && tile != 32) return false;
  if (group_tiles < 1 || (group_tiles & (group_tiles - 1)) != 0) return false;
  return static_cast<int64_t>(tile) * group_tiles <= (int64_t(1) << 30);
}

// Bits of the `causal` argument of the selection entry points.
constexpr int32_t kCausal = VECATTN_CAUSAL, kKeepDiag = VECATTN_KEEP_DIAG,
                  kUnpadded = VECATTN_UNPADDED;
// Bits the selection entry points accept.
constexpr int32_t kSelBits = kCausal | kKeepDiag | kUnpadded;

// Largest count any block can produce.  Without the diagonal, k_i is
// non-decreasing in L_i, so the largest L_i decides; with it (block i adds
// its own n_i rows' keys), the largest min(L_i, k_i + n_i).  Every block but
// the last has n_i = P and L_i, k_i non-decreasing in i, so that value is
// non-decreasing over them: the last two blocks decide.
int64_t max_count(int64_t N, int32_t P, int32_t flags, int32_t mode, double param) {
  const bool causal = (flags & kCausal) != 0;
  const int64_t Np = num_blocks(N, P);
  const int64_t Lmax = causal ? std::min<int64_t>(N, Np * static_cast<int64_t>(P)) : N;
  if (mode != VECATTN_SEL_TOPK) return Lmax;
  if (!(flags & kKeepDiag)) return topk_count(param, Lmax);
  int64_t best = 0;
  for (int64_t i = std::max<int64_t>(0, Np - 2); i < Np; ++i) {
    const int64_t n_i = std::min<int64_t>(N, (i + 1) * P) - i * P;
    const int64_t L = causal ? std::min<int64_t>(N, (i + 1) * P) : N;
    best = std::max(best, std::min(L, topk_count(param, L) + n_i));
  }
  return best;
}

constexpr int64_t kMaxHeadParams = 128;  // query heads a per-head parameter list may cover

// The attention gathers K and V rows with 32-bit byte offsets inside one
// head: key j of a head sits at j * row_bytes, computed with a 24-bit
// multiply, and the head's rows must span < 2^31 bytes.  Heads beyond that
// are rejected (UNSUPPORTED) instead of gathering wrong rows.
bool gather_offsets_ok(const vecattn_tdesc* d) {
  const int64_t rowb = d->sN * 2;
  if (d->N >= (int64_t(1) << 24)) return false;
  if (d->N > 1 && rowb >= (int64_t(1) << 24)) return false;
  return (d->N - 1) * rowb + 2 * d->D < (int64_t(1) << 31);
}

// Every check of vecattn_sparse_attn, without launching anything.
vecattn_status check_attn(const void* q, const vecattn_tdesc* qd, const void* k,
                          const vecattn_tdesc* kd, const void* v, const vecattn_tdesc* vd,
                          const int32_t* idx, int64_t cap, const int32_t* counts, int32_t block,
                          int32_t causal, float scale, const void* o, const vecattn_tdesc* od) {
  vecattn_status st;
  if ((st = check_desc(q, qd)) != VECATTN_OK) return st;
  if ((st = check_desc(k, kd)) != VECATTN_OK) return st;
  if ((st = check_desc(v, vd)) != VECATTN_OK) return st;
  if ((st = check_desc(o, od)) != VECATTN_OK) return st;
  if (kd->B != qd->B || kd->N != qd->N || kd->D != qd->D || qd->H % kd->H != 0)
    return VECATTN_ERR_INVALID_ARG;
  if (vd->B != kd->B || vd->H != kd->H || vd->N != kd->N || vd->D != kd->D)
    return VECATTN_ERR_INVALID_ARG;
  if (od->B != qd->B || od->H != qd->H || od->N != qd->N || od->D != qd->D)
    return VECATTN_ERR_INVALID_ARG;
  if (!idx || !counts || block < 1 || cap < 1 || cap > kMaxN) return VECATTN_ERR_INVALID_ARG;
  if (!std::isfinite(scale) || scale < 0.0f) return VECATTN_ERR_INVALID_ARG;
  if ((causal & ~kSelBits) != 0) return VECATTN_ERR_INVALID_ARG;
  if (!gather_offsets_ok(kd) || !gather_offsets_ok(vd)) return VECATTN_ERR_UNSUPPORTED;
  return VECATTN_OK;
}

// Every argument check of the selection entry points except the workspace's;
// *need receives the workspace bytes the call needs.
vecattn_status select_check(const void* q, const vecattn_tdesc* qd, const void* k,
                            const vecattn_tdesc* kd, int32_t block, int32_t causal, int32_t mode,
                            double param, const double* head_params, int32_t tile,
                            int32_t group_tiles, const int32_t* idx, int64_t cap,
                            const int32_t* counts, size_t* need) {
  vecattn_status st = check_desc(q, qd);
  if (st != VECATTN_OK) return st;
  st = check_desc(k, kd);
  if (st != VECATTN_OK) return st;
  if (kd->B != qd->B || kd->N != qd->N || kd->D != qd->D || qd->H % kd->H != 0)
    return VECATTN_ERR_INVALID_ARG;
  if (!idx || !counts || block < 1 || cap < 1 || cap > kMaxN) return VECATTN_ERR_INVALID_ARG;
  if (!mode_ok(mode) || (causal & ~kSelBits) != 0) return VECATTN_ERR_INVALID_ARG;
  if (head_params) {
    if (qd->H > kMaxHeadParams) return VECATTN_ERR_UNSUPPORTED;
    for (int64_t h = 0; h < qd->H; ++h) {
      if (!param_ok(mode, head_params[h])) return VECATTN_ERR_INVALID_ARG;
      if (mode == VECATTN_SEL_TOPK && cap < max_count(qd->N, block, causal, mode, head_params[h]))
        return VECATTN_ERR_CAPACITY;
    }
    param = head_params[0];
  } else if (!param_ok(mode, param)) {
    return VECATTN_ERR_INVALID_ARG;
  }
  if (mode == VECATTN_SEL_MINS_TILED && !tiling_ok(tile, group_tiles))
    return VECATTN_ERR_INVALID_ARG;
  if (!head_params && mode == VECATTN_SEL_TOPK &&
      cap < max_count(qd->N, block, causal, mode, param))
    return VECATTN_ERR_CAPACITY;
  // With the diagonal kept, no block may be clamped: cap covers every count.
  if ((causal & kKeepDiag) && mode != VECATTN_SEL_TOPK &&
      cap < max_count(qd->N, block, causal, mode, param))
    return VECATTN_ERR_CAPACITY;
  *need = vecattn::select_min_workspace_bytes(qd->B, qd->H, kd->H, qd->N, qd->D, block, mode);
  return VECATTN_OK;
}

vecattn_status select_impl(const void* q, const vecattn_tdesc* qd, const void* k,
                           const vecattn_tdesc* kd, int32_t block, int32_t causal, int32_t mode,
                           double param, const double* head_params, int32_t tile,
                           int32_t group_tiles, int32_t* idx, int64_t cap, int32_t* counts,
                           int32_t* n_clamped, void* workspace, size_t workspace_bytes,
                           void* stream) {
  size_t need = 0;
  const vecattn_status st = select_check(q, qd, k, kd, block, causal, mode, param, head_params,
                                         tile, group_tiles, idx, cap, counts, &need);
  if (st != VECATTN_OK) return st;
  if (need > 0 && (!workspace || workspace_bytes < need)) return VECATTN_ERR_CAPACITY;
  if (workspace && !aligned16(workspace)) return VECATTN_ERR_INVALID_ARG;
  if (head_params) param = head_params[0];
  vecattn::SelectArgs a{to_tensor(q, qd), to_tensor(k, kd), block, (causal & kCausal) ? 1 : 0,
                        (causal & kKeepDiag) ? 1 : 0, (causal & kUnpadded) ? 1 : 0, mode, param,
                        head_params, tile, group_tiles,
                        idx, cap, counts, n_clamped, workspace, workspace_bytes};
  hipError_t e = vecattn::launch_select(a, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? VECATTN_OK : VECATTN_ERR_DEVICE;
}

}  // namespace

extern "C" {

int32_t vecattn_version(void) { return 102; }

const char* vecattn_status_string(vecattn_status s) {
  switch (s) {
    case VECATTN_OK: return "ok";
    case VECATTN_ERR_INVALID_ARG: return "invalid argument";
    case VECATTN_ERR_UNSUPPORTED: return "unsupported";
    case VECATTN_ERR_CAPACITY: return "capacity too small";
    case VECATTN_ERR_DEVICE: return "device error";
  }
  return "unknown status";
}

vecattn_status vecattn_pool(const void* q, const vecattn_tdesc* qd, int32_t block, void* qp,
                            const vecattn_tdesc* qpd, void* stream) {
  vecattn_status st = check_desc(q, qd);
  if (st != VECATTN_OK) return st;
  if (block < 1) return VECATTN_ERR_INVALID_ARG;
  st = check_desc(qp, qpd);
  if (st != VECATTN_OK) return st;
  if (qpd->B != qd->B || qpd->H != qd->H || qpd->D != qd->D || qpd->N != num_blocks(qd->N, block))
    return VECATTN_ERR_INVALID_ARG;
  hipError_t e = vecattn::launch_pool(to_tensor(q, qd), block, qp, qpd->sB, qpd->sH, qpd->sN,
                                      static_cast<hipStream_t>(stream));
  return e == hipSuccess ? VECATTN_OK : VECATTN_ERR_DEVICE;
}

vecattn_status vecattn_select_max_count(int64_t N, int32_t block, int32_t causal, int32_t mode,
                                        double param, int64_t* out) {
  if (!out || N < 1 || N > kMaxN || block < 1 || !mode_ok(mode) || !param_ok(mode, param) ||
      (causal & ~kSelBits) != 0)
    return VECATTN_ERR_INVALID_ARG;
  *out = max_count(N, block, causal, mode, param);
  return VECATTN_OK;
}

vecattn_status vecattn_select_workspace_size(const vecattn_tdesc* qd, const vecattn_tdesc* kd,
                                             int32_t block, int32_t causal, int32_t mode,
                                             int64_t cap, size_t* bytes) {
  (void)causal;
  if (!qd || !kd || !bytes || block < 1 || cap < 1) return VECATTN_ERR_INVALID_ARG;
  if (!mode_ok(mode) || qd->B < 1 || qd->H < 1 || qd->N < 1 || qd->N > kMaxN || kd->H < 1 ||
      qd->H % kd->H != 0 || (qd->D != 64 && qd->D != 128))
    return VECATTN_ERR_INVALID_ARG;
  *bytes = vecattn::select_workspace_bytes(qd->B, qd->H, kd->H, qd->N, qd->D, block, mode, cap);
  return VECATTN_OK;
}

size_t vecattn_select_workspace_bytes(const vecattn_tdesc* qd, const vecattn_tdesc* kd,
                                      int32_t block, int32_t mode, int64_t cap) {
  size_t n = 0;
  return vecattn_select_workspace_size(qd, kd, block, 0, mode, cap, &n) == VECATTN_OK ? n : 0;
}

vecattn_status vecattn_head_sparsity(const int32_t* counts, int64_t B, int64_t Hq, int64_t N,
                                     int32_t block, int32_t causal, double* sparsity,
                                     void* stream) {
  if (!counts || !sparsity || B < 1 || Hq < 1 || Hq > INT32_MAX || N < 1 || N > kMaxN ||
      block < 1 || (causal & ~kSelBits) != 0)
    return VECATTN_ERR_INVALID_ARG;
  hipError_t e = vecattn::launch_head_sparsity(counts, B, Hq, N, block, (causal & kCausal) ? 1 : 0,
                                               sparsity, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? VECATTN_OK : VECATTN_ERR_DEVICE;
}

vecattn_status vecattn_recall(const void* q, const vecattn_tdesc* qd, const void* k,
                              const vecattn_tdesc* kd, const int32_t* idx, int64_t cap,
                              const int32_t* counts, int32_t block, int32_t causal, float scale,
                              float* kept, void* stream) {
  vecattn_status st = check_desc(q, qd);
  if (st != VECATTN_OK) return st;
  if ((st = check_desc(k, kd)) != VECATTN_OK) return st;
  if (kd->B != qd->B || kd->N != qd->N || kd->D != qd->D || qd->H % kd->H != 0)
    return VECATTN_ERR_INVALID_ARG;
  if (!idx || !counts || !kept || block < 1 || cap < 1 || cap > kMaxN)
    return VECATTN_ERR_INVALID_ARG;
  if (!std::isfinite(scale) || scale < 0.0f) return VECATTN_ERR_INVALID_ARG;
  if ((causal & ~kSelBits) != 0) return VECATTN_ERR_INVALID_ARG;
  if (qd->N > vecattn::kRecallMaxN) return VECATTN_ERR_UNSUPPORTED;
  vecattn::RecallArgs a{to_tensor(q, qd), to_tensor(k, kd), idx, counts, cap, block,
                        (causal & kCausal) ? 1 : 0, scale, kept};
  hipError_t e = vecattn::launch_recall(a, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? VECATTN_OK : VECATTN_ERR_DEVICE;
}

vecattn_status vecattn_select(const void* q, const vecattn_tdesc* qd, const void* k,
                              const vecattn_tdesc* kd, int32_t block, int32_t causal, int32_t mode,
                              double param, int32_t* idx, int64_t cap, int32_t* counts,
                              int32_t* n_clamped, void* workspace, size_t workspace_bytes,
                              void* stream) {
  // Cross-tile minS through this entry point uses the paper's B_K = G_K = 16.
  return select_impl(q, qd, k, kd, block, causal, mode, param, nullptr, 16, 16, idx, cap, counts,
                     n_clamped, workspace, workspace_bytes, stream);
}

vecattn_status vecattn_select_noalloc(const void* q, const vecattn_tdesc* qd, const void* k,
                                      const vecattn_tdesc* kd, int32_t block, int32_t causal,
                                      int32_t mode, double param, int32_t* idx, int64_t cap,
                                      int32_t* counts, int32_t* n_clamped, void* stream) {
  // All checks first (no device call on an error), then the size limit, then
  // this GPU's copy of the library's workspace.
  size_t need = 0;
  vecattn_status st = select_check(q, qd, k, kd, block, causal, mode, param, nullptr, 16, 16, idx,
                                   cap, counts, &need);
  if (st != VECATTN_OK) return st;
  if (need > vecattn::kStaticWorkspaceBytes) return VECATTN_ERR_CAPACITY;
  void* ws = nullptr;
  if (vecattn::static_workspace(&ws) != hipSuccess) return VECATTN_ERR_DEVICE;
  return select_impl(q, qd, k, kd, block, causal, mode, param, nullptr, 16, 16, idx, cap, counts,
                     n_clamped, ws, vecattn::kStaticWorkspaceBytes, stream);
}

vecattn_status vecattn_select_per_head(const void* q, const vecattn_tdesc* qd, const void* k,
                                       const vecattn_tdesc* kd, int32_t block, int32_t causal,
                                       int32_t mode, const double* params, int32_t tile,
                                       int32_t group_tiles, int32_t* idx, int64_t cap,
                                       int32_t* counts, int32_t* n_clamped, void* workspace,
                                       size_t workspace_bytes, void* stream) {
  if (!params) return VECATTN_ERR_INVALID_ARG;
  return select_impl(q, qd, k, kd, block, causal, mode, 0.0, params, tile, group_tiles, idx, cap,
                     counts, n_clamped, workspace, workspace_bytes, stream);
}

vecattn_status vecattn_select_mins_tiled(const void* q, const vecattn_tdesc* qd, const void* k,
                                         const vecattn_tdesc* kd, int32_t block, int32_t causal,
                                         double alpha, int32_t tile, int32_t group_tiles,
                                         int32_t* idx, int64_t cap, int32_t* counts,
                                         int32_t* n_clamped, void* workspace,
                                         size_t workspace_bytes, void* stream) {
  return select_impl(q, qd, k, kd, block, causal, VECATTN_SEL_MINS_TILED, alpha, nullptr, tile,
                     group_tiles, idx, cap, counts, n_clamped, workspace, workspace_bytes, stream);
}

vecattn_status vecattn_sparse_attn_ordered(const void* q, const vecattn_tdesc* qd, const void* k,
                                           const vecattn_tdesc* kd, const void* v,
                                           const vecattn_tdesc* vd, const int32_t* idx,
                                           int64_t cap, const int32_t* counts,
                                           const int32_t* order, int32_t block, int32_t causal,
                                           float scale, void* o, const vecattn_tdesc* od,
                                           float* lse, void* stream) {
  const vecattn_status st =
      check_attn(q, qd, k, kd, v, vd, idx, cap, counts, block, causal, scale, o, od);
  if (st != VECATTN_OK) return st;
  vecattn::SparseAttnArgs a{to_tensor(q, qd), to_tensor(k, kd), to_tensor(v, vd),
                            o, od->sB, od->sH, od->sN, lse, idx, counts, cap, block,
                            (causal & kCausal) ? 1 : 0, scale, order};
  hipError_t e = vecattn::launch_sparse_attn(a, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? VECATTN_OK : VECATTN_ERR_DEVICE;
}

vecattn_status vecattn_sparse_attn(const void* q, const vecattn_tdesc* qd, const void* k,
                                   const vecattn_tdesc* kd, const void* v, const vecattn_tdesc* vd,
                                   const int32_t* idx, int64_t cap, const int32_t* counts,
                                   int32_t block, int32_t causal, float scale, void* o,
                                   const vecattn_tdesc* od, float* lse, void* stream) {
  return vecattn_sparse_attn_ordered(q, qd, k, kd, v, vd, idx, cap, counts, nullptr, block, causal,
                                     scale, o, od, lse, stream);
}

vecattn_status vecattn_attn_order(const int32_t* idx, int64_t cap, const int32_t* counts,
                                  int64_t B, int32_t Hq, int64_t N, int32_t block, int32_t* order,
                                  void* stream) {
  if (!idx || !counts || !order || B < 1 || Hq < 1 || N < 1 || N > kMaxN || block < 1 ||
      cap < 1 || cap > kMaxN || B * Hq > INT32_MAX)
    return VECATTN_ERR_INVALID_ARG;
  const int64_t Np = (N + block - 1) / block;
  hipError_t e = vecattn::launch_attn_order(idx, cap, counts, B * Hq, static_cast<int32_t>(Np), N,
                                            order, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? VECATTN_OK : VECATTN_ERR_DEVICE;
}

vecattn_status vecattn_check_lists(const int32_t* idx, int64_t rows, int64_t cap,
                                   const int32_t* counts, int64_t n_keys, int32_t* n_bad,
                                   void* stream) {
  if (!n_bad || rows < 0 || rows > INT32_MAX || cap < 1 || cap > kMaxN || n_keys < 1 ||
      n_keys > kMaxN)
    return VECATTN_ERR_INVALID_ARG;
  if (rows > 0 && (!idx || !counts)) return VECATTN_ERR_INVALID_ARG;
  hipError_t e = vecattn::launch_check_lists(idx, counts, rows, cap, n_keys, n_bad,
                                             static_cast<hipStream_t>(stream));
  return e == hipSuccess ? VECATTN_OK : VECATTN_ERR_DEVICE;
}

}  // extern "C"

namespace {

// Packed variable-length batches: sequence s is rows [cu[s], cu[s+1]) of the
// B = 1 tensors; its blocks, lists and counts follow those of the sequences
// before it.
bool cu_ok(const int64_t* cu, int32_t nseq, int64_t total) {
  if (!cu || nseq < 1 || cu[0] != 0 || cu[nseq] != total) return false;
  for (int32_t s = 0; s < nseq; ++s)
    if (cu[s + 1] < cu[s]) return false;
  return true;
}

vecattn_tdesc seq_desc(const vecattn_tdesc* d, int64_t n) {
  vecattn_tdesc r = *d;
  r.N = n;
  return r;
}

constexpr int64_t kMaxGridYZ = 65535;   // heads and sequences (grid dimensions)
constexpr int64_t kMaxCacheRows = int64_t(1) << 28;

bool same_shape(const vecattn_tdesc* a, const vecattn_tdesc* b) {
  return a->B == b->B && a->H == b->H && a->N == b->N && a->D == b->D;
}

bool flags_ok(int32_t flags) { return flags == 0 || flags == VECATTN_CLEAR_PADDING; }

// Strides of dimensions of size 1 address nothing.
bool same_strides(const vecattn_tdesc* a, const vecattn_tdesc* b) {
  return (a->B == 1 || a->sB == b->sB) && (a->H == 1 || a->sH == b->sH) &&
         (a->N == 1 || a->sN == b->sN);
}

// An output whose sequences or heads share memory would be written several times.
bool shares_rows(const vecattn_tdesc* d) {
  return (d->B > 1 && d->sB == 0) || (d->H > 1 && d->sH == 0);
}

// What the workspace of the attention over an encoder's states, and the call, need of
// the shapes.
vecattn_status check_cross(const vecattn_tdesc* qd, const vecattn_tdesc* kd) {
  if (!qd || !kd || qd->B < 1 || qd->H < 1 || qd->N < 1 || kd->H < 1 || kd->N < 1 ||
      qd->N > kMaxN || kd->N > kMaxN)
    return VECATTN_ERR_INVALID_ARG;
  if (kd->B != qd->B || kd->D != qd->D || qd->H % kd->H != 0) return VECATTN_ERR_INVALID_ARG;
  if ((qd->D != 64 && qd->D != 128) ||
      !vecattn::cross_attn_grid_ok(qd->B, qd->H, kd->H, qd->N, kd->N, qd->D))
    return VECATTN_ERR_UNSUPPORTED;
  return VECATTN_OK;
}

size_t cache_page_bytes(const vecattn_cache* c) {
  const size_t token = static_cast<size_t>(c->D) * c->bits / 8 + static_cast<size_t>(c->D) / 64 * 4;
  return 2 * token * static_cast<size_t>(c->page) * static_cast<size_t>(c->H);
}

vecattn_status check_cache(const vecattn_cache* c, bool with_data) {
  if (!c || c->pages < 1 || c->H < 1 || c->D < 1) return VECATTN_ERR_INVALID_ARG;
  if (c->page < 32 || c->page > 1024 || (c->page & (c->page - 1)) != 0)
    return VECATTN_ERR_INVALID_ARG;
  if (c->bits != 4 && c->bits != 8) return VECATTN_ERR_INVALID_ARG;
  if (with_data && (!c->data || !aligned16(c->data))) return VECATTN_ERR_INVALID_ARG;
  if ((c->D != 64 && c->D != 128) || c->H > kMaxGridYZ) return VECATTN_ERR_UNSUPPORTED;
  if (static_cast<size_t>(c->pages) > (size_t(1) << 62) / cache_page_bytes(c))
    return VECATTN_ERR_INVALID_ARG;
  return VECATTN_OK;
}

bool cols_ok(int64_t cols, int32_t page) { return cols >= 1 && cols <= kMaxN / page; }

// The arguments that writing and reading back share.
vecattn_status check_cache_rows(const void* k, const vecattn_tdesc* kd, const void* v,
                                const vecattn_tdesc* vd, const vecattn_cache* c,
                                const int32_t* table, int64_t cols, const int32_t* lens) {
  vecattn_status st;
  if ((st = check_desc(k, kd)) != VECATTN_OK) return st;
  if ((st = check_desc(v, vd)) != VECATTN_OK) return st;
  if ((st = check_cache(c, true)) != VECATTN_OK) return st;
  if (!same_shape(kd, vd) || kd->H != c->H || kd->D != c->D) return VECATTN_ERR_INVALID_ARG;
  if (!table || !lens || !cols_ok(cols, c->page)) return VECATTN_ERR_INVALID_ARG;
  if (kd->B > kMaxGridYZ || kd->N > kMaxCacheRows) return VECATTN_ERR_UNSUPPORTED;
  return VECATTN_OK;
}

vecattn_status check_cache_attn(const vecattn_tdesc* qd, const vecattn_cache* c, bool with_data,
                                int64_t cols, int64_t window, int64_t sinks,
                                vecattn::CacheAttnShape* s) {
  const vecattn_status st = check_cache(c, with_data);
  if (st != VECATTN_OK) return st;
  if (!qd || qd->B < 1 || qd->H < 1 || qd->N < 1 || qd->D != c->D || qd->H % c->H != 0)
    return VECATTN_ERR_INVALID_ARG;
  if (!cols_ok(cols, c->page) || window < 1 || sinks < 0) return VECATTN_ERR_INVALID_ARG;
  if (qd->B > kMaxGridYZ || qd->H > kMaxGridYZ || qd->N > kMaxCacheRows)
    return VECATTN_ERR_UNSUPPORTED;
  // A window or sinks past every position is all of it (and keeps the sums of
  // positions in range).
  *s = vecattn::CacheAttnShape{qd->B, qd->H, c->H, qd->N, qd->D, cols, c->page,
                               std::min(window, kMaxN), std::min(sinks, kMaxN)};
  return vecattn::cache_attn_grid_ok(*s) ? VECATTN_OK : VECATTN_ERR_UNSUPPORTED;
}

vecattn_status check_keep(const vecattn_cache* c, bool with_data, int64_t cols, int64_t B,
                          int64_t M) {
  const vecattn_status st = check_cache(c, with_data);
  if (st != VECATTN_OK) return st;
  if (!cols_ok(cols, c->page) || B < 1 || M < 1 || M > kMaxN) return VECATTN_ERR_INVALID_ARG;
  return B > kMaxGridYZ ? VECATTN_ERR_UNSUPPORTED : VECATTN_OK;
}

vecattn::CacheArgs to_cache(const vecattn_cache* c, const int32_t* table, int64_t cols,
                            const int32_t* lens) {
  return vecattn::CacheArgs{c->data, c->pages, c->H, c->D, c->page, c->bits, table, cols, lens};
}

const void* seq_ptr(const void* p, const vecattn_tdesc* d, int64_t row) {
  return static_cast<const char*>(p) + row * d->sN * 2;  // bf16 elements
}

}  // namespace

extern "C" {

vecattn_status vecattn_select_varlen(const void* q, const vecattn_tdesc* qd, const void* k,
                                     const vecattn_tdesc* kd, const int64_t* cu_seqlens,
                                     int32_t nseq, int32_t block, int32_t causal, int32_t mode,
                                     double param, int32_t* idx, int64_t cap, int32_t* counts,
                                     int32_t* n_clamped, void* workspace, size_t workspace_bytes,
                                     void* stream) {
  vecattn_status st = check_desc(q, qd);
  if (st != VECATTN_OK) return st;
  if ((st = check_desc(k, kd)) != VECATTN_OK) return st;
  if (qd->B != 1 || kd->B != 1 || kd->N != qd->N || kd->D != qd->D || qd->H % kd->H != 0)
    return VECATTN_ERR_INVALID_ARG;
  if (!cu_ok(cu_seqlens, nseq, qd->N) || !idx || !counts || block < 1 || cap < 1 || cap > kMaxN)
    return VECATTN_ERR_INVALID_ARG;
  if (!mode_ok(mode) || !param_ok(mode, param) || (causal & ~kSelBits) != 0)
    return VECATTN_ERR_INVALID_ARG;
  // Every sequence's checks first, so that an error launches nothing.
  for (int32_t s = 0; s < nseq; ++s) {
    const int64_t n = cu_seqlens[s + 1] - cu_seqlens[s];
    if (n == 0) continue;
    if ((mode == VECATTN_SEL_TOPK || (causal & kKeepDiag)) &&
        cap < max_count(n, block, causal, mode, param))
      return VECATTN_ERR_CAPACITY;
    const size_t need = vecattn::select_min_workspace_bytes(1, qd->H, kd->H, n, qd->D, block, mode);
    if (need > 0 && (!workspace || workspace_bytes < need)) return VECATTN_ERR_CAPACITY;
  }
  int64_t blocks = 0;  // blocks of the sequences before s
  for (int32_t s = 0; s < nseq; ++s) {
    const int64_t n = cu_seqlens[s + 1] - cu_seqlens[s];
    if (n == 0) continue;
    const vecattn_tdesc qs = seq_desc(qd, n), ks = seq_desc(kd, n);
    st = select_impl(seq_ptr(q, qd, cu_seqlens[s]), &qs, seq_ptr(k, kd, cu_seqlens[s]), &ks, block,
                     causal, mode, param, nullptr, 16, 16, idx + blocks * qd->H * cap, cap,
                     counts + blocks * qd->H, n_clamped, workspace, workspace_bytes, stream);
    if (st != VECATTN_OK) return st;
    blocks += num_blocks(n, block);
  }
  return VECATTN_OK;
}

vecattn_status vecattn_sparse_attn_varlen(const void* q, const vecattn_tdesc* qd, const void* k,
                                          const vecattn_tdesc* kd, const void* v,
                                          const vecattn_tdesc* vd, const int64_t* cu_seqlens,
                                          int32_t nseq, const int32_t* idx, int64_t cap,
                                          const int32_t* counts, int32_t block, int32_t causal,
                                          float scale, void* o, const vecattn_tdesc* od,
                                          float* lse, void* stream) {
  // The whole packed tensors first (sizes, strides, the relations between
  // Q, K, V and O), then every sequence's view, so that an error launches
  // nothing.
  vecattn_status st = check_attn(q, qd, k, kd, v, vd, idx, cap, counts, block, causal, scale, o, od);
  if (st != VECATTN_OK) return st;
  if (qd->B != 1 || kd->B != 1 || vd->B != 1 || od->B != 1) return VECATTN_ERR_INVALID_ARG;
  if (!cu_ok(cu_seqlens, nseq, qd->N)) return VECATTN_ERR_INVALID_ARG;
  for (int32_t s = 0; s < nseq; ++s) {
    const int64_t n = cu_seqlens[s + 1] - cu_seqlens[s];
    if (n == 0) continue;
    const int64_t r0 = cu_seqlens[s];
    const vecattn_tdesc qs = seq_desc(qd, n), ks = seq_desc(kd, n), vs = seq_desc(vd, n),
                        os = seq_desc(od, n);
    st = check_attn(seq_ptr(q, qd, r0), &qs, seq_ptr(k, kd, r0), &ks, seq_ptr(v, vd, r0), &vs, idx,
                    cap, counts, block, causal, scale, seq_ptr(o, od, r0), &os);
    if (st != VECATTN_OK) return st;
  }
  vecattn::SparseAttnArgs a{to_tensor(q, qd), to_tensor(k, kd), to_tensor(v, vd),
                            o, od->sB, od->sH, od->sN, lse, idx, counts, cap, block,
                            (causal & kCausal) ? 1 : 0, scale, nullptr};
  hipError_t e = vecattn::launch_sparse_attn_varlen(a, cu_seqlens, nseq, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? VECATTN_OK : VECATTN_ERR_DEVICE;
}

vecattn_status vecattn_window_attn(const void* q, const vecattn_tdesc* qd, const void* k,
                                   const vecattn_tdesc* kd, const void* v, const vecattn_tdesc* vd,
                                   const int32_t* lens, int64_t window, int64_t sinks,
                                   int32_t causal, float scale, void* o, const vecattn_tdesc* od,
                                   float* lse, void* stream) {
  vecattn_status st;
  if ((st = check_desc(q, qd)) != VECATTN_OK) return st;
  if ((st = check_desc(k, kd)) != VECATTN_OK) return st;
  if ((st = check_desc(v, vd)) != VECATTN_OK) return st;
  if ((st = check_desc(o, od)) != VECATTN_OK) return st;
  if (kd->B != qd->B || kd->D != qd->D || qd->N > kd->N || qd->H % kd->H != 0)
    return VECATTN_ERR_INVALID_ARG;
  if (vd->B != kd->B || vd->H != kd->H || vd->N != kd->N || vd->D != kd->D || !same_shape(od, qd))
    return VECATTN_ERR_INVALID_ARG;
  if (window < 1 || sinks < 0 || !std::isfinite(scale) || scale < 0.0f || (causal & ~kCausal) != 0)
    return VECATTN_ERR_INVALID_ARG;
  if (qd->B > kMaxGridYZ || qd->H > kMaxGridYZ ||
      qd->B * qd->H * num_blocks(qd->N, vecattn::kWindowRows) > (int64_t(1) << 23))
    return VECATTN_ERR_UNSUPPORTED;
  // A tile's rows are addressed with 32-bit byte offsets.
  if (kd->N > 1 && (kd->sN >= (int64_t(1) << 24) || vd->sN >= (int64_t(1) << 24)))
    return VECATTN_ERR_UNSUPPORTED;
  vecattn::WindowArgs a{to_tensor(q, qd), to_tensor(k, kd), to_tensor(v, vd), o, od->sB, od->sH,
                        od->sN, lse, lens, window, sinks, causal, scale};
  hipError_t e = vecattn::launch_window_attn(a, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? VECATTN_OK : VECATTN_ERR_DEVICE;
}

vecattn_status vecattn_cache_size(const vecattn_cache* cache, size_t* bytes) {
  if (!bytes) return VECATTN_ERR_INVALID_ARG;
  const vecattn_status st = check_cache(cache, false);
  if (st != VECATTN_OK) return st;
  *bytes = static_cast<size_t>(cache->pages) * cache_page_bytes(cache);
  return VECATTN_OK;
}

vecattn_status vecattn_cache_write(const void* k, const vecattn_tdesc* kd, const void* v,
                                   const vecattn_tdesc* vd, const vecattn_cache* cache,
                                   const int32_t* table, int64_t cols, const int32_t* lens,
                                   const int32_t* n_new, void* stream) {
  vecattn_status st = check_cache_rows(k, kd, v, vd, cache, table, cols, lens);
  if (st != VECATTN_OK) return st;
  hipError_t e = vecattn::launch_cache_write(to_tensor(k, kd), to_tensor(v, vd),
                                             to_cache(cache, table, cols, lens), n_new,
                                             static_cast<hipStream_t>(stream));
  return e == hipSuccess ? VECATTN_OK : VECATTN_ERR_DEVICE;
}

static vecattn_status read_cache(const vecattn_cache* cache, const int32_t* table, int64_t cols,
                                 const int32_t* lens, int64_t start, void* k,
                                 const vecattn_tdesc* kd, void* v, const vecattn_tdesc* vd,
                                 bool clear, void* stream) {
  vecattn_status st = check_cache_rows(k, kd, v, vd, cache, table, cols, lens);
  if (st != VECATTN_OK) return st;
  if (start < 0 || start > kMaxN) return VECATTN_ERR_INVALID_ARG;
  hipError_t e = vecattn::launch_cache_read(to_cache(cache, table, cols, lens), start,
                                            to_tensor(k, kd), to_tensor(v, vd), clear,
                                            static_cast<hipStream_t>(stream));
  return e == hipSuccess ? VECATTN_OK : VECATTN_ERR_DEVICE;
}

vecattn_status vecattn_cache_read(const vecattn_cache* cache, const int32_t* table, int64_t cols,
                                  const int32_t* lens, int64_t start, void* k,
                                  const vecattn_tdesc* kd, void* v, const vecattn_tdesc* vd,
                                  void* stream) {
  return read_cache(cache, table, cols, lens, start, k, kd, v, vd, false, stream);
}

vecattn_status vecattn_cache_read_whole(const vecattn_cache* cache, const int32_t* table,
                                        int64_t cols, const int32_t* lens, int64_t start, void* k,
                                        const vecattn_tdesc* kd, void* v, const vecattn_tdesc* vd,
                                        void* stream) {
  return read_cache(cache, table, cols, lens, start, k, kd, v, vd, true, stream);
}

vecattn_status vecattn_cache_attn_workspace_size(const vecattn_tdesc* qd,
                                                 const vecattn_cache* cache, int64_t cols,
                                                 int64_t window, int64_t sinks, size_t* bytes) {
  if (!bytes) return VECATTN_ERR_INVALID_ARG;
  vecattn::CacheAttnShape s;
  const vecattn_status st = check_cache_attn(qd, cache, false, cols, window, sinks, &s);
  if (st != VECATTN_OK) return st;
  *bytes = vecattn::cache_attn_workspace_bytes(s);
  return VECATTN_OK;
}

vecattn_status vecattn_cache_attn(const void* q, const vecattn_tdesc* qd,
                                  const vecattn_cache* cache, const int32_t* table, int64_t cols,
                                  const int32_t* lens, const int32_t* n_new, int64_t window,
                                  int64_t sinks, float scale, void* o, const vecattn_tdesc* od,
                                  float* lse, void* workspace, size_t workspace_bytes,
                                  void* stream) {
  vecattn_status st;
  if ((st = check_desc(q, qd)) != VECATTN_OK) return st;
  if ((st = check_desc(o, od)) != VECATTN_OK) return st;
  vecattn::CacheAttnShape s;
  if ((st = check_cache_attn(qd, cache, true, cols, window, sinks, &s)) != VECATTN_OK) return st;
  if (!table || !lens || !same_shape(od, qd) || !std::isfinite(scale) || scale < 0.0f)
    return VECATTN_ERR_INVALID_ARG;
  const size_t need = vecattn::cache_attn_workspace_bytes(s);
  if (need > 0 && (!workspace || workspace_bytes < need)) return VECATTN_ERR_CAPACITY;
  if (workspace && !aligned16(workspace)) return VECATTN_ERR_INVALID_ARG;
  vecattn::CacheAttnArgs a{s, to_tensor(q, qd), to_cache(cache, table, cols, lens), n_new, o,
                           od->sB, od->sH, od->sN, lse, scale, workspace};
  hipError_t e = vecattn::launch_cache_attn(a, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? VECATTN_OK : VECATTN_ERR_DEVICE;
}

vecattn_status vecattn_cache_mass_workspace_size(const vecattn_tdesc* qd,
                                                 const vecattn_cache* cache, size_t* bytes) {
  if (!bytes) return VECATTN_ERR_INVALID_ARG;
  vecattn::CacheAttnShape s;
  const vecattn_status st = check_cache_attn(qd, cache, false, 1, 1, 0, &s);
  if (st != VECATTN_OK) return st;
  *bytes = vecattn::cache_mass_workspace_bytes(s);
  return VECATTN_OK;
}

vecattn_status vecattn_cache_mass(const void* q, const vecattn_tdesc* qd, const float* lse,
                                  const vecattn_cache* cache, const int32_t* table, int64_t cols,
                                  const int32_t* lens, const int32_t* n_new, int64_t window,
                                  int64_t sinks, float scale, float decay, const float* mass,
                                  float* out, int64_t M, int32_t flags, void* workspace,
                                  size_t workspace_bytes, void* stream) {
  vecattn_status st;
  if ((st = check_desc(q, qd)) != VECATTN_OK) return st;
  vecattn::CacheAttnShape s;
  if ((st = check_cache_attn(qd, cache, true, cols, window, sinks, &s)) != VECATTN_OK) return st;
  if (!lse || !table || !lens || !out || M < 1 || M > kMaxN) return VECATTN_ERR_INVALID_ARG;
  if (!std::isfinite(scale) || scale < 0.0f || !std::isfinite(decay) || decay < 0.0f ||
      !flags_ok(flags))
    return VECATTN_ERR_INVALID_ARG;
  const size_t need = vecattn::cache_mass_workspace_bytes(s);
  if (need > 0 && (!workspace || workspace_bytes < need)) return VECATTN_ERR_CAPACITY;
  if (workspace && !aligned16(workspace)) return VECATTN_ERR_INVALID_ARG;
  vecattn::CacheMassArgs a{to_tensor(q, qd), lse, to_cache(cache, table, cols, lens), n_new,
                           s.window, s.sinks, scale, decay, mass, out, M, flags != 0, workspace};
  hipError_t e = vecattn::launch_cache_mass(a, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? VECATTN_OK : VECATTN_ERR_DEVICE;
}

vecattn_status vecattn_cache_keep_workspace_size(const vecattn_cache* cache, int64_t cols,
                                                 int64_t B, int64_t M, size_t* bytes) {
  if (!bytes) return VECATTN_ERR_INVALID_ARG;
  const vecattn_status st = check_keep(cache, false, cols, B, M);
  if (st != VECATTN_OK) return st;
  *bytes = vecattn::cache_keep_workspace_bytes(to_cache(cache, nullptr, cols, nullptr), B, M);
  return VECATTN_OK;
}

vecattn_status vecattn_cache_keep(const float* mass, int64_t M, int64_t B,
                                  const vecattn_cache* cache, const int32_t* table, int64_t cols,
                                  const int32_t* lens, int64_t budget, int64_t sinks,
                                  int64_t recent, int32_t* idx, int32_t* kept, void* workspace,
                                  size_t workspace_bytes, void* stream) {
  const vecattn_status st = check_keep(cache, true, cols, B, M);
  if (st != VECATTN_OK) return st;
  if (!mass || !table || !lens || !idx || !kept) return VECATTN_ERR_INVALID_ARG;
  if (budget < 1 || budget > kMaxN || sinks < 0 || recent < 0 || sinks > budget ||
      recent > budget - sinks)
    return VECATTN_ERR_INVALID_ARG;
  const vecattn::CacheArgs c = to_cache(cache, table, cols, lens);
  const size_t need = vecattn::cache_keep_workspace_bytes(c, B, M);
  if (need > 0 && (!workspace || workspace_bytes < need)) return VECATTN_ERR_CAPACITY;
  if (workspace && !aligned16(workspace)) return VECATTN_ERR_INVALID_ARG;
  hipError_t e = vecattn::launch_cache_keep(c, B, mass, M, budget, sinks, recent, idx, kept,
                                            workspace, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? VECATTN_OK : VECATTN_ERR_DEVICE;
}

vecattn_status vecattn_cache_gather_wide(const vecattn_cache* cache, const int32_t* table,
                                         int64_t cols, int64_t B, const int32_t* idx,
                                         const int32_t* kept, int64_t budget,
                                         const vecattn_cache* to, const int32_t* to_table,
                                         int64_t to_cols, const float* mass, int64_t M,
                                         float* mass_out, int64_t M_out, int32_t flags,
                                         void* stream) {
  vecattn_status st;
  if ((st = check_cache(cache, true)) != VECATTN_OK) return st;
  if ((st = check_cache(to, true)) != VECATTN_OK) return st;
  if (to->H != cache->H || to->D != cache->D || to->bits != cache->bits)
    return VECATTN_ERR_INVALID_ARG;
  if (!table || !idx || !kept || !to_table || B < 1 || budget < 1 || budget > kMaxN)
    return VECATTN_ERR_INVALID_ARG;
  if (!cols_ok(cols, cache->page) || !cols_ok(to_cols, to->page)) return VECATTN_ERR_INVALID_ARG;
  if ((mass == nullptr) != (mass_out == nullptr) || !flags_ok(flags) ||
      (mass && (M < 1 || M > kMaxN || M_out < budget || M_out > kMaxN)))
    return VECATTN_ERR_INVALID_ARG;
  // 256 threads per 64 slots, fewer than 2^32 of them.
  if (B > kMaxGridYZ || budget > kMaxN / 2) return VECATTN_ERR_UNSUPPORTED;
  hipError_t e = vecattn::launch_cache_gather(
      to_cache(cache, table, cols, nullptr), to_cache(to, to_table, to_cols, nullptr), B, idx, kept,
      budget, mass, M, mass_out, M_out, flags != 0, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? VECATTN_OK : VECATTN_ERR_DEVICE;
}

vecattn_status vecattn_cache_gather(const vecattn_cache* cache, const int32_t* table, int64_t cols,
                                    int64_t B, const int32_t* idx, const int32_t* kept,
                                    int64_t budget, const vecattn_cache* to,
                                    const int32_t* to_table, int64_t to_cols, const float* mass,
                                    int64_t M, float* mass_out, int32_t flags, void* stream) {
  return vecattn_cache_gather_wide(cache, table, cols, B, idx, kept, budget, to, to_table, to_cols,
                                   mass, M, mass_out, budget, flags, stream);
}

vecattn_status vecattn_cross_attn_workspace_size(const vecattn_tdesc* qd, const vecattn_tdesc* kd,
                                                 size_t* bytes) {
  if (!bytes) return VECATTN_ERR_INVALID_ARG;
  const vecattn_status st = check_cross(qd, kd);
  if (st != VECATTN_OK) return st;
  *bytes = vecattn::cross_attn_workspace_bytes(qd->B, qd->H, kd->H, qd->N, kd->N, qd->D);
  return VECATTN_OK;
}

vecattn_status vecattn_cross_attn(const void* q, const vecattn_tdesc* qd, const void* k,
                                  const vecattn_tdesc* kd, const void* v, const vecattn_tdesc* vd,
                                  const int32_t* lens, const uint8_t* mask, int64_t mask_sB,
                                  const int32_t* n_q, int32_t flags, float scale, void* o,
                                  const vecattn_tdesc* od, float* lse, void* workspace,
                                  size_t workspace_bytes, void* stream) {
  vecattn_status st;
  if ((st = check_desc(q, qd)) != VECATTN_OK) return st;
  if ((st = check_desc(k, kd)) != VECATTN_OK) return st;
  if ((st = check_desc(v, vd)) != VECATTN_OK) return st;
  if ((st = check_desc(o, od)) != VECATTN_OK) return st;
  if ((st = check_cross(qd, kd)) != VECATTN_OK) return st;
  if (!same_shape(vd, kd) || !same_shape(od, qd) || shares_rows(od)) return VECATTN_ERR_INVALID_ARG;
  if (mask_sB < 0 || !std::isfinite(scale) || scale < 0.0f || !flags_ok(flags))
    return VECATTN_ERR_INVALID_ARG;
  // A tile's rows are addressed with 32-bit byte offsets.
  if (kd->N > 1 && (kd->sN >= (int64_t(1) << 24) || vd->sN >= (int64_t(1) << 24)))
    return VECATTN_ERR_UNSUPPORTED;
  const size_t need = vecattn::cross_attn_workspace_bytes(qd->B, qd->H, kd->H, qd->N, kd->N, qd->D);
  if (need > 0 && (!workspace || workspace_bytes < need)) return VECATTN_ERR_CAPACITY;
  if (workspace && !aligned16(workspace)) return VECATTN_ERR_INVALID_ARG;
  vecattn::CrossArgs a{to_tensor(q, qd), to_tensor(k, kd), to_tensor(v, vd), o, od->sB, od->sH,
                       od->sN, lse, lens, mask, mask_sB, n_q, flags != 0, scale, workspace};
  hipError_t e = vecattn::launch_cross_attn(a, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? VECATTN_OK : VECATTN_ERR_DEVICE;
}

vecattn_status vecattn_rope_ladder(int32_t rot, double base, int32_t scaling, double factor,
                                   double context, double fast, double slow, double* freq,
                                   double* mfactor) {
  if (!freq || !mfactor || rot < 2 || rot > 2 * vecattn::kRopeMaxPairs || rot % 2 != 0)
    return VECATTN_ERR_INVALID_ARG;
  if (scaling < VECATTN_ROPE_NONE || scaling > VECATTN_ROPE_BANDS || !std::isfinite(base) ||
      base <= 1.0)
    return VECATTN_ERR_INVALID_ARG;
  if (scaling != VECATTN_ROPE_NONE && (!std::isfinite(factor) || factor < 1.0))
    return VECATTN_ERR_INVALID_ARG;
  if ((scaling == VECATTN_ROPE_PARTS || scaling == VECATTN_ROPE_BANDS) &&
      (!std::isfinite(context) || context <= 0.0 || !std::isfinite(slow) || slow <= 0.0 ||
       !std::isfinite(fast) || fast <= slow))
    return VECATTN_ERR_INVALID_ARG;
  vecattn::rope_ladder(rot, base, scaling, factor, context, fast, slow, freq, mfactor);
  return VECATTN_OK;
}

vecattn_status vecattn_rope(const void* q, const vecattn_tdesc* qd, const void* k,
                            const vecattn_tdesc* kd, const vecattn_rope_spec* spec,
                            const int32_t* pos, int64_t pos_sA, int64_t pos_sB,
                            const int32_t* lens, const int32_t* n_new, int64_t start, void* qo,
                            const vecattn_tdesc* qod, void* ko, const vecattn_tdesc* kod,
                            void* stream) {
  vecattn_status st;
  if ((st = check_desc(q, qd)) != VECATTN_OK) return st;
  if ((st = check_desc(qo, qod)) != VECATTN_OK) return st;
  if (!same_shape(qod, qd) || shares_rows(qod) || (q == qo && !same_strides(qod, qd)))
    return VECATTN_ERR_INVALID_ARG;
  const bool with_k = k || kd || ko || kod;
  if (with_k) {
    if ((st = check_desc(k, kd)) != VECATTN_OK) return st;
    if ((st = check_desc(ko, kod)) != VECATTN_OK) return st;
    if (!same_shape(kod, kd) || shares_rows(kod) || (k == ko && !same_strides(kod, kd)))
      return VECATTN_ERR_INVALID_ARG;
    if (kd->B != qd->B || kd->N != qd->N || kd->D != qd->D) return VECATTN_ERR_INVALID_ARG;
  }
  if (!spec || spec->rot < 2 || spec->rot > qd->D || spec->rot % 2 != 0 || !spec->freq ||
      (spec->layout != VECATTN_ROPE_HALF && spec->layout != VECATTN_ROPE_INTERLEAVED) ||
      spec->axes < 1 || spec->axes > 4 || (spec->flags & ~(VECATTN_ROPE_TRANSPOSED | VECATTN_CLEAR_PADDING)) != 0 ||
      !std::isfinite(spec->factor))
    return VECATTN_ERR_INVALID_ARG;
  for (int32_t i = 0; i < spec->rot / 2; ++i) {
    if (!(std::fabs(spec->freq[i]) <= 1024.0)) return VECATTN_ERR_INVALID_ARG;
    if (spec->axis && (spec->axis[i] < 0 || spec->axis[i] >= spec->axes))
      return VECATTN_ERR_INVALID_ARG;
  }
  if ((pos && lens) || pos_sA < 0 || pos_sB < 0 || start > kMaxN || start < -kMaxN)
    return VECATTN_ERR_INVALID_ARG;
  if (qd->H + (with_k ? kd->H : 0) > kMaxGridYZ || qd->B > kMaxN / qd->N)
    return VECATTN_ERR_UNSUPPORTED;
  vecattn::RopeArgs a{to_tensor(q, qd),
                      with_k ? to_tensor(k, kd) : Tensor4{},
                      to_tensor(qo, qod),
                      with_k ? to_tensor(ko, kod) : Tensor4{},
                      spec->rot,
                      spec->layout == VECATTN_ROPE_HALF,
                      (spec->flags & VECATTN_ROPE_TRANSPOSED) != 0,
                      (spec->flags & VECATTN_CLEAR_PADDING) != 0,
                      spec->factor,
                      spec->freq,
                      spec->axis,
                      pos,
                      pos_sA,
                      pos_sB,
                      lens,
                      n_new,
                      start};
  hipError_t e = vecattn::launch_rope(a, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? VECATTN_OK : VECATTN_ERR_DEVICE;
}

vecattn_status vecattn_plan_filter_ratios(int32_t heads, int32_t n_cand, const double* sparsity,
                                          const double* perf, double target, int32_t grid,
                                          int32_t* choice, double* best_perf) {
  if (heads < 1 || n_cand < 1 || !sparsity || !perf || !choice || !best_perf)
    return VECATTN_ERR_INVALID_ARG;
  if (grid < 1 || grid > (1 << 20) || !(target >= 0.0 && target <= 1.0))
    return VECATTN_ERR_INVALID_ARG;
  if (static_cast<int64_t>(heads) * grid > (int64_t(1) << 26)) return VECATTN_ERR_INVALID_ARG;
  for (int64_t t = 0; t < static_cast<int64_t>(heads) * n_cand; ++t)
    if (!(sparsity[t] >= 0.0 && sparsity[t] <= 1.0) || !std::isfinite(perf[t]))
      return VECATTN_ERR_INVALID_ARG;
  return vecattn::plan_filter_ratios(heads, n_cand, sparsity, perf, target, grid, choice,
                                     best_perf) == 0
             ? VECATTN_OK
             : VECATTN_ERR_CAPACITY;
}

}  // extern "C"
