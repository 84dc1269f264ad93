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
// workgroup; its waves take blocks of 32 tokens in turn.  A long
// sequence is split over workgroups of `chunk` blocks, joined by k_cache_merge.
//
// MFMA 16x16x32 lane layout (lane l = 16 g + n): A: row n, K-slots 8 g .. 8 g + 7;
// B: column n, the same slots; C: column n, rows 4 g .. 4 g + 3.
#include <algorithm>
#include <type_traits>

#include "cache_common.h"

namespace vecattn {
namespace {

constexpr float kUnseen = -3.4028234663852886e38f;  // reference of a row that has met no key
constexpr int32_t kMaxLen = 1 << 30;                 // positions stay in 32 bits
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
  int32_t cols, pages;   // pages past the first 2^31 - 1 cannot be named
  int32_t window, sinks;
  int32_t H, n, group, page_shift;
  int32_t tiles;     // row tiles per head
  int32_t splits;    // workgroups a row tile's keys are split over
  int32_t chunk;     // blocks of 32 keys per split
  float scale_log2;
};

// What one row tile sees, in blocks of 32 tokens: the first `ns` blocks (sinks),
// then blocks nb0 ..; `total` of both.
struct Span {
  int32_t p_first;      // position of the sequence's row 0
  int32_t p_lo, p_hi;   // positions of the tile's rows
  int32_t ns, nb0, total;
  int32_t rows;         // rows of the sequence (all tiles)
};

__device__ __forceinline__ Span span_of(const AttnParams& a, int64_t b, int row0, int nrows) {
  Span s;
  const int len = min(max(a.lens[b], 0), kMaxLen);
  const int nb = a.n_new ? min(max(a.n_new[b], 0), a.n) : a.n;
  s.p_first = len - nb;
  s.rows = nb * a.group;
  s.p_lo = s.p_first + row0 / a.group;
  s.p_hi = s.p_first + (min(row0 + nrows, s.rows) - 1) / a.group;
  s.ns = s.nb0 = s.total = 0;
  if (row0 >= s.rows || s.p_hi < 0) return s;
  const int near = max(0, s.p_lo - a.window + 1);
  s.nb0 = near >> 5;
  s.ns = min(s.nb0, (min(a.sinks, near) + 31) >> 5);
  // Tokens past the table are held nowhere.
  const int held = a.cols << (a.page_shift - 5);
  const int end = min((s.p_hi >> 5) + 1, held);
  s.ns = min(s.ns, held);
  s.total = s.ns + max(0, end - s.nb0);
  return s;
}

// Eight codes as bf16.  `ones` is kOnes in a vector register that the compiler does
// not see through: with both constants in scalar registers it takes two instructions
// for (x & mask) | ones instead of one.
template <int BITS>
struct Unpack;
template <>
struct Unpack<4> {
  static constexpr float kOff = 16.0f;
  static constexpr uint32_t kOnes = 0x41804180u;   // a pair of 16.0
  static __device__ __forceinline__ bf16x8 get(const uint32_t* w, uint32_t ones) {
    constexpr uint32_t mask = 0x00780078u;
    const uint32_t x = w[0];
    const u32x4 r = {((x << 3) & mask) | ones, ((x >> 1) & mask) | ones, ((x >> 5) & mask) | ones,
                     ((x >> 9) & mask) | ones};
    return __builtin_bit_cast(bf16x8, r);
  }
};
template <>
struct Unpack<8> {
  static constexpr float kOff = 0.0f;
  static constexpr uint32_t kOnes = 0;
  static __device__ __forceinline__ bf16x8 get(const uint32_t* w, uint32_t) {
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

// What a wave holds of a block: its lanes' codes and the (m, s) of the tokens of
// their C-layout rows.
template <int D, int BITS>
struct Block {
  using L = CacheLayout<D, BITS>;
  uint32_t kc[L::kRun], vc[L::kRun], kp[2][4 * L::kG], vp[2][4 * L::kG];
  __device__ __forceinline__ void load(const uint8_t* blk, int lane) {
#pragma unroll
    for (int c = 0; c < L::kRun / 4; ++c)
      *reinterpret_cast<u32x4*>(kc + 4 * c) =
          *reinterpret_cast<const u32x4*>(blk + (c * 64 + lane) * 16);
#pragma unroll
    for (int tl = 0; tl < 2; ++tl)
#pragma unroll
      for (int c = 0; c < L::kG; ++c)
        *reinterpret_cast<u32x4*>(kp[tl] + 4 * c) = *reinterpret_cast<const u32x4*>(
            blk + L::kCodes + (16 * tl + 4 * (lane >> 4)) * L::kG * 4 + 16 * c);
    blk += L::kHalf;
#pragma unroll
    for (int c = 0; c < L::kRun / 4; ++c)
      *reinterpret_cast<u32x4*>(vc + 4 * c) =
          *reinterpret_cast<const u32x4*>(blk + (c * 64 + lane) * 16);
#pragma unroll
    for (int tl = 0; tl < 2; ++tl)
#pragma unroll
      for (int c = 0; c < L::kG; ++c)
        *reinterpret_cast<u32x4*>(vp[tl] + 4 * c) = *reinterpret_cast<const u32x4*>(
            blk + L::kCodes + (16 * tl + 4 * (lane >> 4)) * L::kG * 4 + 16 * c);
  }
};

typedef const __attribute__((address_space(4))) int32_t* ScalarInts;

template <int D, int BITS, int R, int W>
__global__ __launch_bounds__(64 * W) void k_cache_attn(const AttnParams a) {
  using L = CacheLayout<D, BITS>;
  constexpr int G = L::kG, DW = L::kDw, ST = D / 32, DB = D / 16;
  constexpr bool kAhead = R == 1;   // registers for a second block
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
  const int t0 = split * a.chunk;
  const int t1 = min(s.total, t0 + a.chunk);
  if (split > 0 && t0 >= t1) return;

  // The t-th block this row tile sees, and its page; where no page is held, or past
  // the last block, a block that can be read and is not used.
  const int sh = a.page_shift - 5;
  const ScalarInts pages = (ScalarInts)(a.table + b * a.cols);
  auto block_of = [&](int t) __attribute__((always_inline)) {
    t = min(t, t1 - 1);
    return t < s.ns ? t : s.nb0 + (t - s.ns);
  };
  auto page_of = [&](int t) __attribute__((always_inline)) { return pages[block_of(t) >> sh]; };
  auto held = [&](int page) __attribute__((always_inline)) { return page >= 0 && page < a.pages; };
  auto address = [&](int t, int page) __attribute__((always_inline)) {
    const int64_t pg = held(page) ? page : 0;
    return a.data + (((pg * a.H + h) << sh) + (block_of(t) & ((1 << sh) - 1))) * L::kBytes;
  };
  int t = t0 + wave;
  Block<D, BITS> cur, nxt;
  int page = -1, page1 = -1;
  if (kAhead && t0 < t1) {
    page = page_of(t);
    page1 = page_of(t + W);
    cur.load(address(t, page), lane);
  }

  // Rows of this lane's columns.
  bf16x8 qf[R][ST];
  float qs[R][G];
  int pos[R];
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
  uint32_t ones = Unpack<BITS>::kOnes;
  asm volatile("" : "+v"(ones));
  const bf16x8 minus_off = {-16.0f, -16.0f, -16.0f, -16.0f, -16.0f, -16.0f, -16.0f, -16.0f};

  auto work = [&](const Block<D, BITS>& x, int t) __attribute__((always_inline)) {
    const int j0 = block_of(t) * kCacheBlock;
    // Every row of the tile sees the whole block, or masks are needed.
    const bool masked = j0 + 31 > s.p_lo || (j0 <= s.p_hi - a.window && j0 + 31 >= a.sinks);
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
              Unpack<BITS>::get(x.kc + (tl * ST + st) * DW, ones), qf[r][st], acc[st / 2], 0, 0, 0);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float y = 0.0f;
#pragma unroll
          for (int gi = 0; gi < G; ++gi) {
            const uint32_t w = x.kp[tl][e * G + gi];
            y = __builtin_fmaf(__uint_as_float(w & 0xFFFF0000u), acc[gi][e], y);
            y = __builtin_fmaf(__uint_as_float(w << 16), qs[r][gi], y);
          }
          sc[tl][e] = y;
        }
      }
      uint32_t vp[2][4 * G];
#pragma unroll
      for (int tl = 0; tl < 2; ++tl)
#pragma unroll
        for (int e = 0; e < 4 * G; ++e) vp[tl][e] = x.vp[tl][e];
      if (masked) {
        // What a hidden token holds must not reach the row: its weight is 0, and so
        // are its m and s.
#pragma unroll
        for (int tl = 0; tl < 2; ++tl)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int j = j0 + 16 * tl + 4 * g + e;
            const bool see = j <= pos[r] && (j > pos[r] - a.window || j < a.sinks);
            sc[tl][e] = see ? sc[tl][e] : kNegInf;
#pragma unroll
            for (int gi = 0; gi < G; ++gi) vp[tl][e * G + gi] = see ? vp[tl][e * G + gi] : 0u;
          }
      }
      // Weights against the reference as it is; where a lane's sum is past 256 (a row
      // that had none among them) the row's reference moves to its maximum first.
      float p[2][4], sum;
      auto weigh = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int tl = 0; tl < 2; ++tl)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            p[tl][e] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[tl][e], a.scale_log2, -m_run[r]));
        sum = ((p[0][0] + p[0][1]) + (p[0][2] + p[0][3])) +
              ((p[1][0] + p[1][1]) + (p[1][2] + p[1][3]));
      };
      weigh();
      if (__any(sum > 256.0f)) {
        float top = kNegInf;
#pragma unroll
        for (int e = 0; e < 4; ++e) top = fmaxf(top, fmaxf(sc[0][e], sc[1][e]));
        top = col_max(top) * a.scale_log2;
        const float m_new = fmaxf(m_run[r], top);
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
        weigh();
      }
      l_run[r] += sum;
#pragma unroll
      for (int gi = 0; gi < G; ++gi) {
        f32x8 y;
#pragma unroll
        for (int tl = 0; tl < 2; ++tl)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint32_t w = vp[tl][e * G + gi];
            y[4 * tl + e] = p[tl][e] * __uint_as_float(w & 0xFFFF0000u);
            pm[r][gi] = __builtin_fmaf(p[tl][e], __uint_as_float(w << 16), pm[r][gi]);
          }
        const bf16x8 pb = __builtin_convertvector(y, bf16x8);
        if constexpr (BITS == 4)
          off[r][gi] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(minus_off, pb, off[r][gi], 0, 0, 0);
#pragma unroll
        for (int db = 4 * gi; db < 4 * gi + 4; ++db)
          oacc[r][db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
              Unpack<BITS>::get(x.vc + db * DW, ones), pb, oacc[r][db], 0, 0, 0);
      }
    }
  };
  // Each block is fetched while the one before is worked on, its page's entry one
  // block earlier still.
  if constexpr (!kAhead) {
    for (; t < t1; t += W) {
      page = page_of(t);
      if (!held(page)) continue;
      cur.load(address(t, page), lane);
      work(cur, t);
    }
  }
  while (kAhead && t < t1) {
    nxt.load(address(t + W, page1), lane);
    int page2 = page_of(t + 2 * W);
    if (held(page)) work(cur, t);
    t += W;
    if (t >= t1) break;
    cur.load(address(t + W, page2), lane);
    page = page_of(t + 2 * W);
    if (held(page1)) work(nxt, t);
    t += W;
    page1 = page;
    page = page2;
  }

  // Join the waves: each scales its sums to the largest reference and adds what the
  // codes' sums leave out.
  constexpr int kPad = D + 4;
  __shared__ float s_m[W][16 * R], s_l[W][16 * R];
  __shared__ __align__(16) float s_o[W][16][kPad];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    l_run[r] = col_sum(l_run[r]);
    if (g == 0) s_m[wave][16 * r + n] = m_run[r];
  }
  __syncthreads();
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int c = 16 * r + n;
    float m = s_m[0][c];
#pragma unroll
    for (int w = 1; w < W; ++w) m = fmaxf(m, s_m[w][c]);
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
    // Four values of a row per thread.
    for (int i = threadIdx.x; i < 4 * D; i += 64 * W) {
      const int rr = i / (D / 4), d = i % (D / 4) * 4;
      const int row = row0 + 16 * r + rr;
      if (row >= s.rows) break;
      float l = 0.0f, mr = s_m[0][16 * r + rr];
      f32x4 y = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int w = 0; w < W; ++w) {
        l += s_l[w][16 * r + rr];
        mr = fmaxf(mr, s_m[w][16 * r + rr]);
        y += *reinterpret_cast<const f32x4*>(&s_o[w][rr][d]);
      }
      const int tok = row / a.group, hq = h * a.group + row % a.group;
      if (a.splits > 1) {
        *reinterpret_cast<f32x4*>(a.part + (static_cast<int64_t>(gridDim.x) * 2 + item * D) *
                                               (16 * R) + (16 * r + rr) * D + d) = y;
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
    if (r + 1 < R) __syncthreads();
  }
}

// Joins the splits of a row: a workgroup per row, its four waves taking every
// fourth split, a lane D / 64 values.
template <int D>
__global__ __launch_bounds__(256) void k_cache_merge(const AttnParams a, int32_t tile_rows,
                                                     int64_t items) {
  constexpr int V = D / 64;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int rows_all = a.n * a.group;
  const int row = static_cast<int>(blockIdx.x % rows_all);
  const int64_t bh = blockIdx.x / rows_all;
  const int h = static_cast<int>(bh % a.H);
  const int64_t b = bh / a.H;
  const int tile = row / tile_rows;
  const Span s = span_of(a, b, tile * tile_rows, tile_rows);
  const int tok = row / a.group, hq = h * a.group + row % a.group;
  if (row >= s.rows) return;
  const int used = max(1, (s.total + a.chunk - 1) / a.chunk);
  const int64_t item0 = (bh * a.tiles + tile) * a.splits;
  const int in_tile = row - tile * tile_rows;
  const float* ml = a.part + (item0 * tile_rows + in_tile) * 2;
  const float* src = a.part + (items * 2 + item0 * D) * tile_rows + in_tile * D + V * lane;
  float m = kUnseen;
  for (int i = lane; i < used; i += 64) m = fmaxf(m, ml[static_cast<int64_t>(i) * tile_rows * 2]);
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) m = fmaxf(m, __shfl_xor(m, o));
  float l = 0.0f, y[V] = {};
#pragma unroll 4
  for (int i = wave; i < used; i += 4) {
    const int64_t at = static_cast<int64_t>(i) * tile_rows;
    const float alpha = __builtin_amdgcn_exp2f(ml[at * 2] - m);
    l = __builtin_fmaf(ml[at * 2 + 1], alpha, l);
#pragma unroll
    for (int x = 0; x < V; ++x) y[x] = __builtin_fmaf(src[at * D + x], alpha, y[x]);
  }
  __shared__ float s_y[4][D + 1];
#pragma unroll
  for (int x = 0; x < V; ++x) s_y[wave][V * lane + x] = y[x];
  if (lane == 0) s_y[wave][D] = l;
  __syncthreads();
  if (threadIdx.x >= D) return;
  const int d = threadIdx.x;
  l = (s_y[0][D] + s_y[1][D]) + (s_y[2][D] + s_y[3][D]);
  const float v = (s_y[0][d] + s_y[1][d]) + (s_y[2][d] + s_y[3][d]);
  const float inv = l > 0.0f ? 1.0f / l : l;
  reinterpret_cast<__bf16*>(a.o)[b * a.o_sB + hq * a.o_sH + tok * a.o_sN + d] =
      static_cast<__bf16>(v * inv);
  if (a.lse && d == 0)
    a.lse[(b * a.H * a.group + hq) * a.n + tok] =
        l == 0.0f ? kNegInf : (m + __builtin_log2f(l)) * kLn2;
}

// How a call is dealt out; depends on its shapes alone, so that the workspace
// query and the launch agree.
struct Deal {
  int32_t R, W, tiles, splits, chunk;
  int64_t items;
};

Deal deal(const CacheAttnShape& s) {
  Deal d;
  const int64_t rows = s.n * (s.Hq / s.H);
  d.R = rows <= 16 ? 1 : 2;
  d.tiles = static_cast<int32_t>((rows + 16 * d.R - 1) / (16 * d.R));
  const int64_t base = s.B * s.H * d.tiles;
  // Blocks a row tile can see: the table's, or the window's and the sinks'.
  const int64_t held = s.cols * (s.page / kCacheBlock);
  const int64_t seen = std::min(held, (std::min<int64_t>(s.window, held * 32) +
                                       std::min<int64_t>(s.n, 16 * d.R) + 31) / 32 + 1 +
                                          (std::min<int64_t>(s.sinks, held * 32) + 31) / 32);
  d.W = d.R == 1 ? 8 : 4;
  constexpr int64_t kTarget = 512, kLeast = 32;
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
  if (s.Hq * s.n > (int64_t(1) << 30) || s.B * s.Hq * s.n >= (int64_t(1) << 24)) return false;
  const Deal d = deal(s);
  return d.items < (int64_t(1) << 23);
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
  a.cols = static_cast<int32_t>(c.cols);
  a.pages = static_cast<int32_t>(std::min<int64_t>(c.pages, INT32_MAX));
  a.window = static_cast<int32_t>(x.shape.window), a.sinks = static_cast<int32_t>(x.shape.sinks);
  a.H = c.H;
  a.n = static_cast<int32_t>(x.shape.n);
  a.group = static_cast<int32_t>(x.shape.Hq / x.shape.H);
  a.page_shift = __builtin_ctz(static_cast<unsigned>(c.page));
  a.tiles = d.tiles, a.splits = d.splits, a.chunk = d.chunk;
  const float scale = x.scale != 0.0f ? x.scale : 1.0f / sqrtf(static_cast<float>(c.D));
  a.scale_log2 = scale * 1.4426950408889634f;
  auto launch = [&](auto kernel, int waves) {
    hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(d.items)), dim3(64 * waves), 0, stream,
                       a);
  };
  auto pick = [&](auto dim, auto bits) {
    constexpr int D = decltype(dim)::value, BITS = decltype(bits)::value;
    if (d.R == 1 && d.W == 8) launch(k_cache_attn<D, BITS, 1, 8>, 8);
    else if (d.R == 1) launch(k_cache_attn<D, BITS, 1, 4>, 4);
    else launch(k_cache_attn<D, BITS, 2, 4>, 4);
  };
  using std::integral_constant;
  if (c.D == 128)
    c.bits == 4 ? pick(integral_constant<int, 128>{}, integral_constant<int, 4>{})
                : pick(integral_constant<int, 128>{}, integral_constant<int, 8>{});
  else
    c.bits == 4 ? pick(integral_constant<int, 64>{}, integral_constant<int, 4>{})
                : pick(integral_constant<int, 64>{}, integral_constant<int, 8>{});
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || d.splits == 1) return e;
  const dim3 grid(static_cast<unsigned>(x.shape.B * x.shape.Hq * x.shape.n));
  if (c.D == 128)
    hipLaunchKernelGGL(k_cache_merge<128>, grid, dim3(256), 0, stream, a, 16 * d.R, d.items);
  else
    hipLaunchKernelGGL(k_cache_merge<64>, grid, dim3(256), 0, stream, a, 16 * d.R, d.items);
  return hipGetLastError();
}

}  // namespace vecattn
