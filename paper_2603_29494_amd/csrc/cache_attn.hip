// Attention of new tokens over the quantised, paged key/value cache: one token
// per sequence (decoding), a few (drafts), or a chunk of a prompt; causal, with
// an optional sliding window and sinks.
//
// A key's value is m + s u per group of 64 head-dim values (cache_common.h), so
//   q . k = sum_G s_G (q_G . u_G) + m_G sum(q_G),
//   sum_j p_j v_j = sum_j (p_j s_jG) u_j + sum_j p_j m_jG,
// and the codes go into the matrix instructions as they are: exact in bf16.
// Codes of 4 bits become 16 + u there (one shift and one and-or per pair); the
// 16 is taken out by starting the score accumulators at -16 sum(q_G) and by
// summing -16 times the rounded weights p_j s_jG with a matrix instruction of
// its own, so that no rounding but that of p_j s_jG to bf16 (half a step, 2^-9)
// remains.  The normaliser and the m_jG terms take the fp32 weights.
//
// The query heads that share a key/value head and the new tokens of a sequence
// are the rows (row = token * group + head), R tiles of 16 of them per
// workgroup; four waves take every fourth block of 32 tokens each.  A long
// sequence is split over workgroups of `chunk` blocks, joined by k_cache_merge.
//
// MFMA 16x16x32 lane layout (lane l = 16 g + n): A: row n, K-slots 8 g .. 8 g + 7;
// B: column n, the same slots; C: column n, rows 4 g .. 4 g + 3.
#include <algorithm>

#include "cache_common.h"

namespace vecattn {
namespace {

constexpr float kUnseen = -3.4028234663852886e38f;  // reference of a row that has met no key
constexpr float kLn2 = 0.69314718055994531f;

struct AttnParams {
  const uint16_t* q;
  int64_t q_sB, q_sH, q_sN;
  uint16_t* o;
  int64_t o_sB, o_sH, o_sN;
  float* lse;
  const uint8_t* data;
  const int32_t* table;
  const int32_t* lens;
  const int32_t* n_new;
  float* part;       // [work item][16 R] (m, l), then [work item][16 R][D] sums
  int64_t cols, pages;
  int64_t window, sinks;
  int32_t H, n, group, page_shift;
  int32_t tiles;     // row tiles per head
  int32_t splits;    // workgroups a row tile's keys are split over
  int32_t chunk;     // blocks of 32 keys per split
  float scale_log2;
};

// What one row tile sees, in blocks of 32 tokens: the first `ns` blocks (sinks),
// then blocks nb0 ..; `total` of both.
struct Span {
  int64_t p_first;   // position of the sequence's row 0
  int64_t p_lo, p_hi;   // positions of the tile's rows
  int64_t ns, nb0, total;
  int32_t rows;      // rows of the sequence (all tiles)
};

__device__ __forceinline__ Span span_of(const AttnParams& a, int64_t b, int row0, int nrows) {
  Span s;
  const int64_t len = a.lens[b];
  const int64_t nb = a.n_new ? min(max(a.n_new[b], 0), a.n) : a.n;
  s.p_first = len - nb;
  s.rows = static_cast<int32_t>(nb) * a.group;
  s.p_lo = s.p_first + row0 / a.group;
  s.p_hi = s.p_first + (min(row0 + nrows, s.rows) - 1) / a.group;
  s.ns = s.nb0 = s.total = 0;
  if (row0 >= s.rows || s.p_hi < 0) return s;
  const int64_t near = max(int64_t(0), s.p_lo - a.window + 1);
  s.nb0 = near >> 5;
  s.ns = min(s.nb0, (min(a.sinks, near) + 31) >> 5);
  // Tokens past the table are held nowhere.
  const int64_t held = a.cols << (a.page_shift - 5);
  const int64_t end = min((s.p_hi >> 5) + 1, held);
  s.ns = min(s.ns, held);
  s.total = s.ns + max(int64_t(0), end - s.nb0);
  return s;
}

template <int BITS>
struct Unpack;
template <>
struct Unpack<4> {
  static constexpr float kOff = 16.0f;
  static __device__ __forceinline__ bf16x8 get(const uint32_t* w) {
    const uint32_t x = w[0];
    u32x4 r;
    r[0] = ((x << 3) & 0x00780078u) | 0x41804180u;
    r[1] = ((x >> 1) & 0x00780078u) | 0x41804180u;
    r[2] = ((x >> 5) & 0x00780078u) | 0x41804180u;
    r[3] = ((x >> 9) & 0x00780078u) | 0x41804180u;
    return __builtin_bit_cast(bf16x8, r);
  }
};
template <>
struct Unpack<8> {
  static constexpr float kOff = 0.0f;
  static __device__ __forceinline__ bf16x8 get(const uint32_t* w) {
    u32x4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t x = w[i >> 1];
      const uint32_t lo = __float_as_uint(static_cast<float>((x >> (16 * (i & 1))) & 0xFFu));
      const uint32_t hi = __float_as_uint(static_cast<float>((x >> (16 * (i & 1) + 8)) & 0xFFu));
      r[i] = __builtin_amdgcn_perm(hi, lo, 0x07060302u);  // exact: an integer below 256
    }
    return __builtin_bit_cast(bf16x8, r);
  }
};

// Over the four lanes that hold a column (n = lane % 16).
__device__ __forceinline__ float col_max(float x) {
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}
__device__ __forceinline__ float col_sum(float x) {
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
}

template <int D, int BITS, int R>
__global__ __launch_bounds__(256) void k_cache_attn(const AttnParams a) {
  using L = CacheLayout<D, BITS>;
  constexpr int G = L::kG, DW = L::kDw, ST = D / 32, DB = D / 16;
  const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);

  const int64_t item = blockIdx.x;   // ((b * H + h) * tiles + tile) * splits + split
  const int split = static_cast<int>(item % a.splits);
  int64_t rest = item / a.splits;
  const int tile = static_cast<int>(rest % a.tiles);
  rest /= a.tiles;
  const int h = static_cast<int>(rest % a.H);
  const int64_t b = rest / a.H;
  const int row0 = tile * 16 * R;
  const Span s = span_of(a, b, row0, 16 * R);
  if (row0 >= s.rows) return;
  const int64_t t0 = static_cast<int64_t>(split) * a.chunk;
  const int64_t t1 = min(s.total, t0 + a.chunk);
  if (split > 0 && t0 >= t1) return;

  // Rows of this lane's columns.
  bf16x8 qf[R][ST];
  float qs[R][G];
  int64_t pos[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int row = row0 + 16 * r + n;
    const int tok = row / a.group, hq = h * a.group + row % a.group;
    const bool have = row < s.rows;
    pos[r] = have ? s.p_first + tok : -1;
    const uint16_t* src = a.q + b * a.q_sB + hq * a.q_sH + tok * a.q_sN;
#pragma unroll
    for (int gi = 0; gi < G; ++gi) qs[r][gi] = 0.0f;
#pragma unroll
    for (int st = 0; st < ST; ++st) {
      u32x4 w = {0, 0, 0, 0};
      if (have) w = *reinterpret_cast<const u32x4*>(src + 32 * st + 8 * g);
      qf[r][st] = __builtin_bit_cast(bf16x8, w);
#pragma unroll
      for (int e = 0; e < 4; ++e)
        qs[r][st / 2] += __uint_as_float(w[e] << 16) + __uint_as_float(w[e] & 0xFFFF0000u);
    }
#pragma unroll
    for (int gi = 0; gi < G; ++gi) qs[r][gi] = col_sum(qs[r][gi]);
  }

  f32x4 oacc[R][DB], off[R][G];
  float pm[R][G], m_run[R], l_run[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    m_run[r] = kUnseen;
    l_run[r] = 0.0f;
#pragma unroll
    for (int db = 0; db < DB; ++db) oacc[r][db] = f32x4{};
#pragma unroll
    for (int gi = 0; gi < G; ++gi) {
      off[r][gi] = f32x4{};
      pm[r][gi] = 0.0f;
    }
  }
  const bf16x8 minus_off = {-16.0f, -16.0f, -16.0f, -16.0f, -16.0f, -16.0f, -16.0f, -16.0f};

  const int sh = a.page_shift - 5;
  for (int64_t t = t0 + wave; t < t1; t += 4) {
    const int64_t jb = t < s.ns ? t : s.nb0 + (t - s.ns);
    const int64_t page = a.table[b * a.cols + (jb >> sh)];
    if (page < 0 || page >= a.pages) continue;
    const uint8_t* blk =
        a.data + (((page * a.H + h) << sh) + (jb & ((int64_t(1) << sh) - 1))) * L::kBytes;
    uint32_t kc[L::kRun], vc[L::kRun], kp[2][4 * G], vp[2][4 * G];
#pragma unroll
    for (int c = 0; c < L::kRun / 4; ++c) {
      *reinterpret_cast<u32x4*>(kc + 4 * c) =
          *reinterpret_cast<const u32x4*>(blk + (c * 64 + lane) * 16);
      *reinterpret_cast<u32x4*>(vc + 4 * c) =
          *reinterpret_cast<const u32x4*>(blk + L::kHalf + (c * 64 + lane) * 16);
    }
#pragma unroll
    for (int tl = 0; tl < 2; ++tl)
#pragma unroll
      for (int c = 0; c < G; ++c) {
        const int at = L::kCodes + (16 * tl + 4 * g) * G * 4 + 16 * c;
        *reinterpret_cast<u32x4*>(kp[tl] + 4 * c) = *reinterpret_cast<const u32x4*>(blk + at);
        *reinterpret_cast<u32x4*>(vp[tl] + 4 * c) =
            *reinterpret_cast<const u32x4*>(blk + L::kHalf + at);
      }
    const int64_t j0 = jb * kCacheBlock;
    // Every row of the tile sees the whole block, or masks are needed.
    const bool masked = j0 + 31 > s.p_lo || (j0 <= s.p_hi - a.window && j0 + 31 >= a.sinks);

    bf16x8 vf[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db) vf[db] = Unpack<BITS>::get(vc + db * DW);
#pragma unroll
    for (int r = 0; r < R; ++r) {
      float sc[2][4];
#pragma unroll
      for (int tl = 0; tl < 2; ++tl) {
        f32x4 acc[G];
#pragma unroll
        for (int gi = 0; gi < G; ++gi) {
          const float z = -Unpack<BITS>::kOff * qs[r][gi];
          acc[gi] = f32x4{z, z, z, z};
        }
#pragma unroll
        for (int st = 0; st < ST; ++st)
          acc[st / 2] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
              Unpack<BITS>::get(kc + (tl * ST + st) * DW), qf[r][st], acc[st / 2], 0, 0, 0);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float x = 0.0f;
#pragma unroll
          for (int gi = 0; gi < G; ++gi) {
            const uint32_t w = kp[tl][e * G + gi];
            x = __builtin_fmaf(__uint_as_float(w & 0xFFFF0000u), acc[gi][e], x);
            x = __builtin_fmaf(__uint_as_float(w << 16), qs[r][gi], x);
          }
          sc[tl][e] = x;
        }
      }
      uint32_t ok = 0xFFu;
      if (masked) {
        ok = 0;
#pragma unroll
        for (int tl = 0; tl < 2; ++tl)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int64_t j = j0 + 16 * tl + 4 * g + e;
            const bool see = j <= pos[r] && (j > pos[r] - a.window || j < a.sinks);
            ok |= see ? 1u << (4 * tl + e) : 0u;
            sc[tl][e] = see ? sc[tl][e] : kNegInf;
          }
      }
      float top = kNegInf;
#pragma unroll
      for (int e = 0; e < 4; ++e) top = fmaxf(top, fmaxf(sc[0][e], sc[1][e]));
      top = col_max(top) * a.scale_log2;
      if (__any(top > m_run[r] + 8.0f)) {  // references move rarely, by steps of 8 (log2 units)
        const float m_new = top > m_run[r] + 8.0f ? top : m_run[r];
        const float alpha = __builtin_amdgcn_exp2f(m_run[r] - m_new);
        m_run[r] = m_new;
        l_run[r] *= alpha;
#pragma unroll
        for (int db = 0; db < DB; ++db) oacc[r][db] *= alpha;
#pragma unroll
        for (int gi = 0; gi < G; ++gi) {
          off[r][gi] *= alpha;
          pm[r][gi] *= alpha;
        }
      }
      float p[2][4];
#pragma unroll
      for (int tl = 0; tl < 2; ++tl)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          p[tl][e] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[tl][e], a.scale_log2, -m_run[r]));
          l_run[r] += p[tl][e];
        }
#pragma unroll
      for (int gi = 0; gi < G; ++gi) {
        f32x8 y;
#pragma unroll
        for (int tl = 0; tl < 2; ++tl)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            uint32_t w = vp[tl][e * G + gi];
            if (masked && !(ok >> (4 * tl + e) & 1u)) w = 0;  // whatever a hidden token holds
            y[4 * tl + e] = p[tl][e] * __uint_as_float(w & 0xFFFF0000u);
            pm[r][gi] = __builtin_fmaf(p[tl][e], __uint_as_float(w << 16), pm[r][gi]);
          }
        const bf16x8 pb = __builtin_convertvector(y, bf16x8);
        if constexpr (BITS == 4)
          off[r][gi] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(minus_off, pb, off[r][gi], 0, 0, 0);
#pragma unroll
        for (int db = 4 * gi; db < 4 * gi + 4; ++db)
          oacc[r][db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[db], pb, oacc[r][db], 0, 0, 0);
      }
    }
  }

  // Join the four waves: each scales its sums to the largest reference and adds
  // what the codes' sums leave out.
  __shared__ float s_m[4][16 * R], s_l[4][16 * R];
  __shared__ float s_o[4][16][D + 4];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    l_run[r] = col_sum(l_run[r]);
    if (g == 0) s_m[wave][16 * r + n] = m_run[r];
  }
  __syncthreads();
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int c = 16 * r + n;
    const float m = fmaxf(fmaxf(s_m[0][c], s_m[1][c]), fmaxf(s_m[2][c], s_m[3][c]));
    const float alpha = __builtin_amdgcn_exp2f(m_run[r] - m);
    if (g == 0) s_l[wave][c] = l_run[r] * alpha;
#pragma unroll
    for (int gi = 0; gi < G; ++gi) pm[r][gi] = col_sum(pm[r][gi]);
#pragma unroll
    for (int db = 0; db < DB; ++db) {
      f32x4 y;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        y[e] = (oacc[r][db][e] + off[r][db / 4][e] + pm[r][db / 4]) * alpha;
      *reinterpret_cast<f32x4*>(&s_o[wave][n][16 * db + 4 * g]) = y;
    }
    __syncthreads();
    // 256 threads: row threadIdx / 16, every sixteenth group of four values.
    const int rr = threadIdx.x >> 4, cc = threadIdx.x & 15;
    const int row = row0 + 16 * r + rr;
    const float l = (s_l[0][16 * r + rr] + s_l[1][16 * r + rr]) +
                    (s_l[2][16 * r + rr] + s_l[3][16 * r + rr]);
    const float mr = fmaxf(fmaxf(s_m[0][16 * r + rr], s_m[1][16 * r + rr]),
                           fmaxf(s_m[2][16 * r + rr], s_m[3][16 * r + rr]));
    const int tok = row / a.group, hq = h * a.group + row % a.group;
    const bool have = row < s.rows;
#pragma unroll
    for (int d = 4 * cc; d < D; d += 64) {
      f32x4 y = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int w = 0; w < 4; ++w) y += *reinterpret_cast<const f32x4*>(&s_o[w][rr][d]);
      if (!have) continue;
      if (a.splits > 1) {
        *reinterpret_cast<f32x4*>(a.part + (static_cast<int64_t>(gridDim.x) * 2 +
                                            item * D) * (16 * R) + (16 * r + rr) * D + d) = y;
        if (d == 0) {
          float* ml = a.part + (item * 16 * R + 16 * r + rr) * 2;
          ml[0] = mr;
          ml[1] = l;
        }
      } else {
        const float inv = l > 0.0f ? 1.0f / l : l;   // no key: 0; NaN stays
        y *= inv;
        *reinterpret_cast<bf16x4*>(a.o + b * a.o_sB + hq * a.o_sH + tok * a.o_sN + d) =
            __builtin_convertvector(y, bf16x4);
        if (a.lse && d == 0)
          a.lse[(b * a.H * a.group + hq) * a.n + tok] =
              l == 0.0f ? kNegInf : (mr + __builtin_log2f(l)) * kLn2;
      }
    }
    __syncthreads();
  }
}

// Joins the splits of a row: one wave per row.
template <int D>
__global__ __launch_bounds__(256) void k_cache_merge(const AttnParams a, int32_t tile_rows,
                                                     int64_t items, int64_t total_rows) {
  const int64_t id = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  if (id >= total_rows) return;
  const int rows_all = a.n * a.group;
  const int row = static_cast<int>(id % rows_all);
  const int64_t bh = id / rows_all;
  const int h = static_cast<int>(bh % a.H);
  const int64_t b = bh / a.H;
  const int tile = row / tile_rows;
  const Span s = span_of(a, b, tile * tile_rows, tile_rows);
  const int tok = row / a.group, hq = h * a.group + row % a.group;
  if (row >= s.rows) return;
  const int used = static_cast<int>(max(int64_t(1), (s.total + a.chunk - 1) / a.chunk));
  const int64_t item0 = (bh * a.tiles + tile) * a.splits;
  const int in_tile = row - tile * tile_rows;
  float m = kUnseen;
  for (int i = 0; i < used; ++i)
    m = fmaxf(m, a.part[((item0 + i) * tile_rows + in_tile) * 2]);
  float l = 0.0f, y[D / 64] = {};
  for (int i = 0; i < used; ++i) {
    const float* ml = a.part + ((item0 + i) * tile_rows + in_tile) * 2;
    const float alpha = __builtin_amdgcn_exp2f(ml[0] - m);
    l += ml[1] * alpha;
    const float* src = a.part + (items * 2 + (item0 + i) * D) * tile_rows + in_tile * D;
#pragma unroll
    for (int x = 0; x < D / 64; ++x) y[x] = __builtin_fmaf(src[64 * x + lane], alpha, y[x]);
  }
  const float inv = l > 0.0f ? 1.0f / l : l;
#pragma unroll
  for (int x = 0; x < D / 64; ++x)
    reinterpret_cast<__bf16*>(a.o)[b * a.o_sB + hq * a.o_sH + tok * a.o_sN + 64 * x + lane] =
        static_cast<__bf16>(y[x] * inv);
  if (a.lse && lane == 0)
    a.lse[(b * a.H * a.group + hq) * a.n + tok] =
        l == 0.0f ? kNegInf : (m + __builtin_log2f(l)) * kLn2;
}

// How a call is dealt out; depends on its shapes alone, so that the workspace
// query and the launch agree.
struct Deal {
  int32_t R, tiles, splits, chunk;
  int64_t items;
};

Deal deal(const CacheAttnShape& s) {
  Deal d;
  const int64_t rows = s.n * (s.Hq / s.H);
  d.R = rows <= 16 ? 1 : rows <= 32 ? 2 : 4;
  d.tiles = static_cast<int32_t>((rows + 16 * d.R - 1) / (16 * d.R));
  const int64_t base = s.B * s.H * d.tiles;
  // Blocks a row tile can see: the table's, or the window's and the sinks'.
  const int64_t held = s.cols * (s.page / kCacheBlock);
  const int64_t seen = std::min(held, (std::min<int64_t>(s.window, held * 32) +
                                       std::min<int64_t>(s.n, 16 * d.R) + 31) / 32 + 1 +
                                          (std::min<int64_t>(s.sinks, held * 32) + 31) / 32);
  constexpr int64_t kTarget = 1024, kLeast = 16;
  const int64_t want = std::max<int64_t>(1, kTarget / base);
  const int64_t chunk = std::max<int64_t>(kLeast, (seen + want - 1) / want);
  d.chunk = static_cast<int32_t>(chunk);
  d.splits = static_cast<int32_t>((seen + chunk - 1) / chunk);
  d.items = base * d.splits;
  return d;
}

}  // namespace

size_t cache_attn_workspace_bytes(const CacheAttnShape& s) {
  const Deal d = deal(s);
  if (d.splits == 1) return 0;
  return static_cast<size_t>(d.items) * 16 * d.R * (s.D + 2) * sizeof(float);
}

bool cache_attn_grid_ok(const CacheAttnShape& s) {
  if (s.Hq * s.n > (int64_t(1) << 30) || s.B * s.Hq * s.n > (int64_t(1) << 31)) return false;
  const Deal d = deal(s);
  return d.items < (int64_t(1) << 24);
}

hipError_t launch_cache_attn(const CacheAttnArgs& x, hipStream_t stream) {
  const Deal d = deal(x.shape);
  const CacheArgs& c = x.cache;
  AttnParams a;
  a.q = static_cast<const uint16_t*>(x.q.ptr);
  a.q_sB = x.q.sB, a.q_sH = x.q.sH, a.q_sN = x.q.sN;
  a.o = static_cast<uint16_t*>(x.o);
  a.o_sB = x.o_sB, a.o_sH = x.o_sH, a.o_sN = x.o_sN;
  a.lse = x.lse;
  a.data = static_cast<const uint8_t*>(c.data);
  a.table = c.table;
  a.lens = c.lens;
  a.n_new = x.n_new;
  a.part = static_cast<float*>(x.workspace);
  a.cols = c.cols, a.pages = c.pages;
  a.window = x.shape.window, a.sinks = x.shape.sinks;
  a.H = c.H;
  a.n = static_cast<int32_t>(x.shape.n);
  a.group = static_cast<int32_t>(x.shape.Hq / x.shape.H);
  a.page_shift = __builtin_ctz(static_cast<unsigned>(c.page));
  a.tiles = d.tiles, a.splits = d.splits, a.chunk = d.chunk;
  const float scale = x.scale != 0.0f ? x.scale : 1.0f / sqrtf(static_cast<float>(c.D));
  a.scale_log2 = scale * 1.4426950408889634f;
  auto run = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(d.items)), dim3(256), 0, stream, a);
  };
  auto pick = [&](auto bits) {
    constexpr int BITS = decltype(bits)::value;
    if (c.D == 128)
      d.R == 1 ? run(k_cache_attn<128, BITS, 1>)
               : d.R == 2 ? run(k_cache_attn<128, BITS, 2>) : run(k_cache_attn<128, BITS, 4>);
    else
      d.R == 1 ? run(k_cache_attn<64, BITS, 1>)
               : d.R == 2 ? run(k_cache_attn<64, BITS, 2>) : run(k_cache_attn<64, BITS, 4>);
  };
  if (c.bits == 4) pick(std::integral_constant<int, 4>{});
  else pick(std::integral_constant<int, 8>{});
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || d.splits == 1) return e;
  const int64_t rows = x.shape.B * x.shape.Hq * x.shape.n;
  const dim3 grid(static_cast<unsigned>((rows + 3) / 4));
  if (c.D == 128)
    hipLaunchKernelGGL(k_cache_merge<128>, grid, dim3(256), 0, stream, a, 16 * d.R, d.items, rows);
  else
    hipLaunchKernelGGL(k_cache_merge<64>, grid, dim3(256), 0, stream, a, 16 * d.R, d.items, rows);
  return hipGetLastError();
}

}  // namespace vecattn
