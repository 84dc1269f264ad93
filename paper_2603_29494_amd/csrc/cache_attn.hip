// Attention of new tokens over the quantised, paged key/value cache: one token
// per sequence (decoding), a few (drafts), or a chunk of a prompt; causal, with
// an optional sliding window and sinks.
//
// A key's value is m + s u per group of 64 head-dim values (cache_common.h), so
//   q . k = sum_G s_G (q_G . u_G) + m_G sum(q_G),
//   sum_j p_j v_j = sum_j (p_j s_jG) u_j + sum_j p_j m_jG,
// and the codes go into the matrix instructions as they are, exactly.
//   K: the code is the bits of a small fp16 number, so shifts and masks are all the
//     unpacking; a row of q is scaled by a power of two, which fits bf16's eight bits
//     into fp16 down to 2^-30 of its largest value.
//   V, 4 bits: 16 + u in bf16 (a shift and an and-or per pair); the 16 is taken out by
//     summing -16 times the rounded weights with a matrix instruction of its own.
//   V, 8 bits: bf16 holds integers to 256.
// No rounding remains but that of p_j s_jG to bf16 (half a step, 2^-9 at most of
// it); the normaliser and the m_jG terms take the fp32 weights.
//
// The query heads that share a key/value head and the new tokens of a sequence
// are the rows (row = token * group + head), up to 32 of them per workgroup; its
// waves take blocks of 32 tokens in turn.  Where eight rows are all, the 16 columns
// of the matrix instructions hold them twice, once for either 16 tokens of a block,
// which halves the work per score.
//
// How the keys are dealt out follows the lengths on the device: every workgroup
// sums what the sequences see, takes chunks of such a size that the workgroups fill
// the chip, and finds its own chunk; k_cache_merge joins the chunks of a row.
//
// Bound by memory in long sequences: 28 query and 4 key/value heads of 128 over 4 x
// 131072 tokens of 4 bits take 54 us (302 MB, 5.6 TB/s) and the join 5.  In short ones
// by the chain of loads before the first codes (lengths, table, codes) and the join
// after the last: 9 us for 700 tokens; 64 sequences of 37 to 8192 tokens, 8 heads, take
// 32 us (105 MB, 3.3 TB/s).
//
// MFMA 16x16x32 lane layout (lane l = 16 g + n): A: row n, K-slots 8 g .. 8 g + 7;
// B: column n, the same slots; C: column n, rows 4 g .. 4 g + 3.
#include <algorithm>
#include <type_traits>

#include "cache_plan.h"

namespace vecattn {
namespace {

// Eight codes of V as bf16.  `ones` is kOnes in a vector register that the compiler does
// not see through: with both constants in scalar registers it takes two instructions
// for (x & mask) | ones instead of one.
template <int BITS>
struct Unpack;
template <>
struct Unpack<4> {
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

// What a wave holds of a block: its lanes' codes and the (m, s) of its tokens in
// the scores' C layout (with HALF of the 16 tokens that the lane's column is for).
template <int D, int BITS, bool HALF>
struct Block {
  using L = CacheLayout<D, BITS>;
  static constexpr int NT = HALF ? 1 : 2;
  uint32_t kc[L::kRun], vc[L::kRun], kp[NT][4 * L::kG], vp[NT][4 * L::kG];
  static __device__ __forceinline__ void codes(uint32_t* to, const uint8_t* from, int lane) {
#pragma unroll
    for (int c = 0; c < L::kRun / 4; ++c)
      *reinterpret_cast<u32x4*>(to + 4 * c) =
          *reinterpret_cast<const u32x4*>(from + (c * 64 + lane) * 16);
  }
  static __device__ __forceinline__ void params(uint32_t (&to)[NT][4 * L::kG], const uint8_t* from,
                                                int lane) {
#pragma unroll
    for (int tl = 0; tl < NT; ++tl) {
      const int tile = HALF ? (lane >> 3) & 1 : tl;
#pragma unroll
      for (int c = 0; c < L::kG; ++c)
        *reinterpret_cast<u32x4*>(to[tl] + 4 * c) = *reinterpret_cast<const u32x4*>(
            from + (16 * tile + 4 * (lane >> 4)) * L::kG * 4 + 16 * c);
    }
  }
  __device__ __forceinline__ void load(const uint8_t* blk, int lane) {
    codes(kc, blk, lane);
    params(kp, blk + L::kCodes, lane);
    codes(vc, blk + L::kHalf, lane);
    params(vp, blk + L::kHalf + L::kCodes, lane);
  }
};

// Rows of q as the score products take them, scaled by 2^k.  sum: of a group's values,
// in the products' scale; unscale: from that scale to scores.
template <int D, int BITS>
struct Rows {
  static constexpr int G = D / kCacheGroup, ST = D / 32;
  f16x8 q[ST];
  float sum[G], unscale;

  __device__ __forceinline__ void load(const uint16_t* src, bool have, int g) {
    u32x4 w[ST];
    float top = 0x1p-100f;
#pragma unroll
    for (int st = 0; st < ST; ++st) {
      w[st] = u32x4{0, 0, 0, 0};
      if (have) w[st] = *reinterpret_cast<const u32x4*>(src + 32 * st + 8 * g);
#pragma unroll
      for (int e = 0; e < 4; ++e)
        top = fmaxf(top, fmaxf(fabsf(low_of(w[st][e])), fabsf(high_of(w[st][e]))));
    }
    // The largest value between 2^14 and 2^15.
    const int k = 15 - __builtin_amdgcn_frexp_expf(col_max(top));
#pragma unroll
    for (int gi = 0; gi < G; ++gi) sum[gi] = 0.0f;
#pragma unroll
    for (int st = 0; st < ST; ++st) {
      u32x4 x;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float lo = low_of(w[st][e]), hi = high_of(w[st][e]);
        sum[st / 2] += lo + hi;
        x[e] = to_f16(__builtin_amdgcn_ldexpf(lo, k), __builtin_amdgcn_ldexpf(hi, k));
      }
      q[st] = __builtin_bit_cast(f16x8, x);
    }
#pragma unroll
    for (int gi = 0; gi < G; ++gi) sum[gi] = __builtin_amdgcn_ldexpf(col_sum(sum[gi]), k - kCodeExp<BITS>);
    unscale = __builtin_amdgcn_ldexpf(1.0f, kCodeExp<BITS> - k);
  }

  // acc + q . u over 32 head-dim values of 16 tokens.
  __device__ __forceinline__ f32x4 dot(const uint32_t* codes, int st, f32x4 acc) const {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, codes_f16<BITS>(codes)),
                                                  q[st], acc, 0, 0, 0);
  }
};

typedef const __attribute__((address_space(4))) int32_t* ScalarInts;

// R tiles of 16 rows, or (HALF, R = 1) 8 rows; W waves.
template <int D, int BITS, int R, bool HALF, int W>
__global__ __launch_bounds__(64 * W) __attribute__((amdgpu_waves_per_eu(HALF ? 2 : 1))) void k_cache_attn(const AttnParams a) {
  using L = CacheLayout<D, BITS>;
  constexpr int G = L::kG, DW = L::kDw, ST = D / 32, DB = D / 16;
  constexpr int NT = HALF ? 1 : 2;             // groups of four tokens whose scores a lane holds
  constexpr int RW = HALF ? 8 : 16;            // rows per tile of columns
  constexpr int kRows = R * RW;
  const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);

  const int h = blockIdx.x % a.H;
  const int index = blockIdx.x / a.H;
  const Share share = find_share(a, kRows, index);
  if (share.unit < 0) return;
  if (a.target && h == 0 && index == share.first && threadIdx.x == 0)
    shares_of(a, kRows, D)[share.unit] = int2{share.first, share.count};
  const int64_t b = share.unit / a.tiles;
  const int row0 = share.unit % a.tiles * kRows;
  const Span s = span_of(a, b, row0, kRows);
  if (row0 >= s.rows) return;
  const int t0 = (index - share.first) * (share.count > 1 ? share.chunk : 0);
  const int t1 = share.count > 1 ? min(s.total, t0 + share.chunk) : s.total;

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

  // Rows of this lane's columns.
  Rows<D, BITS> rows[R];
  int pos[R];
  float to_log2[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int row = row0 + RW * r + n % RW;
    const int tok = row / a.group, hq = h * a.group + row % a.group;
    const bool have = row < s.rows;
    pos[r] = have ? s.p_first + tok : -1;
    rows[r].load(a.q + b * a.q_sB + hq * a.q_sH + tok * a.q_sN, have, g);
    to_log2[r] = fmaxf(a.scale_log2 * rows[r].unscale, 0x1p-126f);   // -inf * 0 is no mask
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
  const bool second = HALF && (n & 8);   // the lane's columns are for the block's last 16 tokens

  auto work = [&](const Block<D, BITS, HALF>& x, int t) __attribute__((always_inline)) {
    const int j0 = block_of(t) * kCacheBlock;
    // Every row of the tile sees the whole block, or masks are needed.
    const bool masked = j0 + 31 > s.p_lo || (j0 <= s.p_hi - a.window && j0 + 31 >= a.sinks);
#pragma unroll
    for (int r = 0; r < R; ++r) {
      float sc[NT][4];
      {
        f32x4 acc[2][G];
#pragma unroll
        for (int tl = 0; tl < 2; ++tl) {
#pragma unroll
          for (int gi = 0; gi < G; ++gi) acc[tl][gi] = f32x4{};
#pragma unroll
          for (int st = 0; st < ST; ++st)
            acc[tl][st / 2] = rows[r].dot(x.kc + (tl * ST + st) * DW, st, acc[tl][st / 2]);
        }
#pragma unroll
        for (int tl = 0; tl < NT; ++tl)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            float y = 0.0f;
#pragma unroll
            for (int gi = 0; gi < G; ++gi) {
              const uint32_t w = x.kp[tl][e * G + gi];
              const float c = HALF ? (second ? acc[1][gi][e] : acc[0][gi][e]) : acc[tl][gi][e];
              y = __builtin_fmaf(high_of(w), c, y);
              y = __builtin_fmaf(low_of(w), rows[r].sum[gi], y);
            }
            sc[tl][e] = y;
          }
      }
      uint32_t vp[NT][4 * G];
#pragma unroll
      for (int tl = 0; tl < NT; ++tl)
#pragma unroll
        for (int e = 0; e < 4 * G; ++e) vp[tl][e] = x.vp[tl][e];
      if (masked) {
        // What a hidden token holds must not reach the row: its weight is 0, and so
        // are its m and s.
#pragma unroll
        for (int tl = 0; tl < NT; ++tl)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int j = j0 + (HALF ? 2 * (n & 8) : 16 * tl) + 4 * g + e;
            const bool see = j <= pos[r] && (j > pos[r] - a.window || j < a.sinks);
            sc[tl][e] = see ? sc[tl][e] : kNegInf;
#pragma unroll
            for (int gi = 0; gi < G; ++gi) vp[tl][e * G + gi] = see ? vp[tl][e * G + gi] : 0u;
          }
      }
      // Weights against the reference as it is; where a lane's sum is past 256 (a row
      // that had none among them) the row's reference moves to its maximum first.
      float p[NT][4], sum;
      auto weigh = [&]() __attribute__((always_inline)) {
        sum = 0.0f;
#pragma unroll
        for (int tl = 0; tl < NT; ++tl) {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            p[tl][e] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[tl][e], to_log2[r], -m_run[r]));
          sum += (p[tl][0] + p[tl][1]) + (p[tl][2] + p[tl][3]);
        }
      };
      weigh();
      if (__any(sum > 256.0f)) {
        float top = kNegInf;
#pragma unroll
        for (int tl = 0; tl < NT; ++tl)
#pragma unroll
          for (int e = 0; e < 4; ++e) top = fmaxf(top, sc[tl][e]);
        top = col_max(top) * to_log2[r];
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
        u32x2 y2[NT];
#pragma unroll
        for (int tl = 0; tl < NT; ++tl) {
          f32x4 y;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint32_t w = vp[tl][e * G + gi];
            y[e] = p[tl][e] * high_of(w);
            pm[r][gi] = __builtin_fmaf(p[tl][e], low_of(w), pm[r][gi]);
          }
          y2[tl] = __builtin_bit_cast(u32x2, __builtin_convertvector(y, bf16x4));
        }
        u32x4 yb;
        if constexpr (HALF)
          yb = u32x4{second ? 0u : y2[0][0], second ? 0u : y2[0][1], second ? y2[0][0] : 0u,
                     second ? y2[0][1] : 0u};
        else yb = u32x4{y2[0][0], y2[0][1], y2[NT - 1][0], y2[NT - 1][1]};
        const bf16x8 pb = __builtin_bit_cast(bf16x8, yb);
        if constexpr (BITS == 4)
          off[r][gi] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(minus_off, pb, off[r][gi], 0, 0, 0);
#pragma unroll
        for (int db = 4 * gi; db < 4 * gi + 4; ++db)
          oacc[r][db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
              Unpack<BITS>::get(x.vc + db * DW, ones), pb, oacc[r][db], 0, 0, 0);
      }
    }
  };
  Block<D, BITS, HALF> cur;
  int t = t0 + wave;
  if constexpr (HALF) {
    // Each block is fetched while the one before is worked on, its page's entry one
    // block earlier still.
    Block<D, BITS, HALF> nxt;
    int page = -1, page1 = -1;
    if (t < t1) {
      page = page_of(t);
      page1 = page_of(t + W);
      cur.load(address(t, page), lane);
    }
    while (t < t1) {
      nxt.load(address(t + W, page1), lane);
      const int page2 = page_of(t + 2 * W);
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
  } else {
    for (; t < t1; t += W) {
      const int page = page_of(t);
      if (!held(page)) continue;
      cur.load(address(t, page), lane);
      work(cur, t);
    }
  }

  // Join the waves (and the two halves of the columns): each scales its sums to the
  // largest reference and adds what the codes' sums leave out.
  __shared__ float s_m[W][16 * R], s_l[W][16 * R];
  __shared__ __align__(16) float s_o[W][16][D + 4];
  auto top_ref = [&](int row) __attribute__((always_inline)) {   // row of the tile, 0 .. kRows - 1
    const int c = row / RW * 16 + row % RW;
    float m = kUnseen;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      m = fmaxf(m, s_m[w][c]);
      if (HALF) m = fmaxf(m, s_m[w][c + 8]);
    }
    return m;
  };
#pragma unroll
  for (int r = 0; r < R; ++r) {
    l_run[r] = col_sum(l_run[r]);
    if (g == 0) s_m[wave][16 * r + n] = m_run[r];
  }
  __syncthreads();
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const float alpha = __builtin_amdgcn_exp2f(m_run[r] - top_ref(RW * r + n % RW));
    if (g == 0) s_l[wave][16 * r + n] = l_run[r] * alpha;
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
    for (int i = threadIdx.x; i < RW * (D / 4); i += 64 * W) {
      const int rr = i / (D / 4), d = i % (D / 4) * 4;
      const int row = row0 + RW * r + rr;
      if (row >= s.rows) break;
      float l = 0.0f;
      f32x4 y = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int w = 0; w < W; ++w)
#pragma unroll
        for (int hf = 0; hf < (HALF ? 2 : 1); ++hf) {
          l += s_l[w][16 * r + rr + 8 * hf];
          y += *reinterpret_cast<const f32x4*>(&s_o[w][rr + 8 * hf][d]);
        }
      const float m = top_ref(RW * r + rr);
      const int tok = row / a.group, hq = h * a.group + row % a.group;
      if (share.count > 1) {
        const int64_t at = static_cast<int64_t>(blockIdx.x) * kRows + RW * r + rr;
        *reinterpret_cast<f32x4*>(a.part + at * D + d) = y;
        if (d == 0) {
          float* ml = a.part + static_cast<int64_t>(a.items) * kRows * D + at * 2;
          ml[0] = m;
          ml[1] = l;
        }
      } else {
        const float inv = l > 0.0f ? 1.0f / l : l;   // no key: 0; NaN stays
        y *= inv;
        *reinterpret_cast<bf16x4*>(a.o + b * a.o_sB + hq * a.o_sH + tok * a.o_sN + d) =
            __builtin_convertvector(y, bf16x4);
        if (a.lse && d == 0)
          a.lse[(b * a.H * a.group + hq) * a.n + tok] =
              l == 0.0f ? kNegInf : (m + __builtin_log2f(l)) * kLn2;
      }
    }
    if (r + 1 < R) __syncthreads();
  }
}

// Joins the chunks of a row: WAVES waves per row take every WAVES-th chunk, a lane
// D / 64 values.  Rows of one chunk are done already.
template <int D, int WAVES>
__global__ __launch_bounds__(256) void k_cache_merge(const AttnParams a, int32_t tile_rows,
                                                     int64_t total_rows) {
  constexpr int V = D / 64, kRowsPer = 4 / WAVES;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int rows_all = a.n * a.group;
  const int64_t id = static_cast<int64_t>(blockIdx.x) * kRowsPer + wave / WAVES;
  if (id >= total_rows) return;   // whole workgroups with four waves per row
  const int row = static_cast<int>(id % rows_all);
  const int bh = static_cast<int>(id / rows_all);
  const int h = bh % a.H;
  const int64_t b = bh / a.H;
  const int tile = row / tile_rows;
  const int2 share = shares_of(a, tile_rows, D)[b * a.tiles + tile];   // first, count
  const int count = share.y;
  if (count <= 1) return;
  const int nb = a.n_new ? min(max(a.n_new[b], 0), a.n) : a.n;
  const int tok = row / a.group, hq = h * a.group + row % a.group;
  if (tok >= nb) return;
  const int64_t at0 = (static_cast<int64_t>(share.x) * a.H + h) * tile_rows + row % tile_rows;
  const int64_t step = static_cast<int64_t>(a.H) * tile_rows;
  const float* src = a.part + at0 * D + V * lane;
  const float* ml = a.part + static_cast<int64_t>(a.items) * tile_rows * D + at0 * 2;
  float m = kUnseen;
  for (int i = lane; i < count; i += 64) m = fmaxf(m, ml[i * step * 2]);
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) m = fmaxf(m, __shfl_xor(m, o));
  float l = 0.0f, y[V] = {};
#pragma unroll 4
  for (int i = wave % WAVES; i < count; i += WAVES) {
    const float alpha = __builtin_amdgcn_exp2f(ml[i * step * 2] - m);
    l = __builtin_fmaf(ml[i * step * 2 + 1], alpha, l);
#pragma unroll
    for (int x = 0; x < V; ++x) y[x] = __builtin_fmaf(src[i * step * D + x], alpha, y[x]);
  }
  if constexpr (WAVES > 1) {
    __shared__ float s_y[WAVES][D + 1];
#pragma unroll
    for (int x = 0; x < V; ++x) s_y[wave][V * lane + x] = y[x];
    if (lane == 0) s_y[wave][D] = l;
    __syncthreads();
    if (wave > 0) return;
    l = 0.0f;
#pragma unroll
    for (int x = 0; x < V; ++x) y[x] = 0.0f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      l += s_y[w][D];
#pragma unroll
      for (int x = 0; x < V; ++x) y[x] += s_y[w][V * lane + x];
    }
  }
  const float inv = l > 0.0f ? 1.0f / l : l;
  __bf16* orow = reinterpret_cast<__bf16*>(a.o) + b * a.o_sB + hq * a.o_sH + tok * a.o_sN;
#pragma unroll
  for (int x = 0; x < V; ++x) orow[V * lane + x] = static_cast<__bf16>(y[x] * inv);
  if (a.lse && lane == 0)
    a.lse[(b * a.H * a.group + hq) * a.n + tok] =
        l == 0.0f ? kNegInf : (m + __builtin_log2f(l)) * kLn2;
}

Deal deal(const CacheAttnShape& s) {
  Deal d;
  const int64_t rows = s.n * (s.Hq / s.H);
  d.half = rows <= 8;
  d.many = rows > 32;
  d.R = rows <= 16 ? 1 : 2;
  // Eight rows at most: few row tiles take more waves on each, and have half the chunks
  // to join (16 sequences x 4 heads, a window of 4096: 14.1 us, 16.8 with four waves);
  // many fill the chip with four (64 x 8 heads: 117 us, 129 with eight).  Many rows:
  // eight waves share what rebuilding a tile costs (136 rows: 66 us, 69 with four; 3584
  // rows: 364 and 441), but not where half of them had no row (40 rows: 65, 111 with
  // eight).
  // Up to 32 rows the codes go in as they are (8 sequences of 16k tokens, 4 heads, 4 bits,
  // 24 rows: 37 us, 60 rebuilt; 32 rows 38 and 60).  From 33 on rows take rebuilt tiles,
  // which keep 11 bits of the weights and of V where the other way keeps 8 of the
  // weights.  That is also the faster way for 65 rows and more over long sequences (96
  // rows 68 us, 124 in tiles of 32 rows; 128 rows 73 and 105), but not for fewer (35 rows
  // 62 and 59; of 64 values over 32k tokens 86 and 53) unless they are very many tokens (4
  // x 131k: 201 and 215), nor over short ones (700 tokens: 27 and 15.5).
  d.W = d.many ? (rows > 128 ? 8 : 4) : d.half && s.B * s.H <= 128 ? 8 : 4;
  d.rows = d.many ? 32 * d.W : d.half ? 8 : 16 * d.R;
  d.tiles = static_cast<int32_t>((rows + d.rows - 1) / d.rows);
  d.units = s.B * d.tiles;
  // Blocks a row tile can see: the table's, or the window's and the sinks'.
  const int64_t held = s.cols * (s.page / kCacheBlock);
  const int64_t seen = std::min(held, (std::min<int64_t>(s.window, held * 32) +
                                       std::min<int64_t>(s.n, d.rows) + 31) / 32 + 1 +
                                          (std::min<int64_t>(s.sinks, held * 32) + 31) / 32);
  // Blocks that pay for a chunk's start and end (128 rows of 4 x 16k tokens rebuilt: 50
  // us with 16, 60 with 24; 16 rows of 8 x 32k: 24 us with 32, 27 with 64).
  d.least = d.many ? 16 : 32;
  d.merge = seen > d.least && d.units <= kMaxUnits;
  d.items = d.units * s.H;
  d.target = 0;
  if (d.merge) {
    // The workgroups that run at a time: two of four waves per CU, or one of eight, or
    // one of 32 rows x 128 values, whose registers leave one wave per SIMD (32 rows of 8
    // x 16k tokens: 38 us with 256, 46 with 512; of 64 values 44 and 35 with 32k).  Never
    // fewer than two chunks per row tile, and two workgroups after each other where
    // their work is long, so that those of hidden tokens even out (512 tokens over 33k:
    // 364 us, 420 with one).
    const int64_t slots = d.W == 8 || (!d.many && d.R == 2 && s.D == 128) ? 256 : 512;
    int64_t rounds = std::max<int64_t>(1, (2 * d.items + slots - 1) / slots);
    if (d.many && d.items * seen >= 64 * 2 * slots) rounds = std::max<int64_t>(2, rounds);
    d.target = static_cast<int32_t>(slots * rounds);
    d.items = std::min<int64_t>(d.target, d.items * ((seen + d.least - 1) / d.least));
  }
  return d;
}

}  // namespace

size_t cache_attn_workspace_bytes(const CacheAttnShape& s) {
  const Deal d = deal(s);
  if (!d.merge) return 0;
  return static_cast<size_t>(d.items) * d.rows * (s.D + 2) * sizeof(float) +
         static_cast<size_t>(d.units) * 2 * sizeof(int32_t);
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
  a.tiles = d.tiles, a.units = static_cast<int32_t>(d.units);
  a.items = static_cast<int32_t>(d.items), a.target = d.target, a.least = d.least;
  const float scale = x.scale != 0.0f ? x.scale : 1.0f / sqrtf(static_cast<float>(c.D));
  a.scale_log2 = scale * 1.4426950408889634f;
  auto pick = [&](auto dim, auto bits) {
    constexpr int D = decltype(dim)::value, BITS = decltype(bits)::value;
    auto launch = [&](auto kernel) {
      hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(d.items)), dim3(64 * d.W), 0, stream, a);
    };
    if (d.many) {
      const hipError_t e = launch_cache_chunk(a, D, BITS, d.W, d.items, stream);
      if (e != hipSuccess) return e;
    } else if (d.half && d.W == 8) launch(k_cache_attn<D, BITS, 1, true, 8>);
    else if (d.half) launch(k_cache_attn<D, BITS, 1, true, 4>);
    else if (d.R == 1) launch(k_cache_attn<D, BITS, 1, false, 4>);
    else launch(k_cache_attn<D, BITS, 2, false, 4>);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || !d.merge) return e;
    // A wave per row where rows fill the chip, four where they do not (14336 rows: 10 us
    // less than with four; 256 rows of 64 chunks: 2 us less than with one).
    const int64_t n = x.shape.B * x.shape.Hq * x.shape.n;
    if (n > 2048)
      hipLaunchKernelGGL((k_cache_merge<D, 1>), dim3(static_cast<unsigned>((n + 3) / 4)), dim3(256),
                         0, stream, a, d.rows, n);
    else
      hipLaunchKernelGGL((k_cache_merge<D, 4>), dim3(static_cast<unsigned>(n)), dim3(256), 0, stream,
                         a, d.rows, n);
    return hipGetLastError();
  };
  using std::integral_constant;
  if (c.D == 128)
    return c.bits == 4 ? pick(integral_constant<int, 128>{}, integral_constant<int, 4>{})
                       : pick(integral_constant<int, 128>{}, integral_constant<int, 8>{});
  return c.bits == 4 ? pick(integral_constant<int, 64>{}, integral_constant<int, 4>{})
                     : pick(integral_constant<int, 64>{}, integral_constant<int, 8>{});
}

}  // namespace vecattn
