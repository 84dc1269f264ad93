// What new tokens' attention puts on each cached token: for token j of a key/value
// head, the sum over the rows (new tokens and query heads that share the head) of
// exp(scale q . k_j - lse), added to the sum that the token has collected before.
//
// A key is m + s u per group of 64 values (cache_common.h), q . k = sum_G s_G (q_G . u_G)
// + m_G sum(q_G): the codes go into the matrix instructions as small fp16 numbers,
// exactly, and rows of q as fp16 times a power of two (many rows: both as bf16), so that
// only fp32 sums round.  A token belongs to one wave, which adds its rows in one order: no
// atomics.
//
// Few rows are bound by reading K's half of the cache: four sequences of 131072 tokens in 4
// bits, 4 heads of 128, 7 rows each: 34 us, 4.9 TB/s.  Many rows by the matrix products and
// the exponentials, whose times add: 512 tokens of 28 heads over 33280 in 8 bits, 4 heads:
// 175 to 187 us over the cards it ran on, 650 to 693 TFLOP/s, 7 of them k_mass_rows (13 more with rows of q in fp16 and their powers of two applied
// to every score; 5 more with the codes fetched by dwords and each sum's lanes added on
// their own, which also takes 207 us instead of 128 for 126 rows over 4 x 131072 tokens).
// Three workgroups fit a CU at a time, and 1040 come out uneven there; splitting their rows
// gains 3%.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "cache_rows.h"

namespace vecattn {
namespace {

struct MassParams {
  const uint16_t* q;
  int64_t q_sB, q_sH, q_sN;
  const float* lse;
  const uint8_t* data;
  const int32_t* table;
  const int32_t* lens;
  const int32_t* n_new;
  const float* mass;   // NULL: nothing collected before
  float* out;
  int64_t M;           // entries per sequence and head
  int32_t cols, pages, page_shift;
  int32_t H, n, group, window, sinks;
  int32_t in_place;    // what no row sees stays as it is
  int32_t clear;       // entries past a sequence's tokens become 0
  float* part;         // [split][B * H][slots], where the rows are split
  int64_t slots;
  int32_t splits;
  float scale_log2, decay;
};

constexpr float kLog2e = 1.4426950408889634f;

// Where a sequence's tokens and rows are.
struct Place {
  int32_t p_first, rows, end;   // position of row 0, rows of all heads, tokens with an entry
};
__device__ __forceinline__ Place place_of(const MassParams& a, int64_t b) {
  const int len = min(max(a.lens[b], 0), 1 << 30);
  const int nb = a.n_new ? min(max(a.n_new[b], 0), a.n) : a.n;
  return Place{len - nb, nb * a.group, static_cast<int>(min<int64_t>(len, a.M))};
}

// The page that holds a block (past the table: some page), and the base of a head's keys of
// the block, or NULL where no page is held.
__device__ __forceinline__ int page_of(const MassParams& a, int64_t b, int jb) {
  return ((ScalarInts)(a.table + b * a.cols))[min(jb >> (a.page_shift - 5), a.cols - 1)];
}
template <int BYTES>
__device__ __forceinline__ const uint8_t* keys_of(const MassParams& a, int64_t page, int h, int jb) {
  const int sh = a.page_shift - 5;
  if (jb >> sh >= a.cols || page < 0 || page >= a.pages) return nullptr;
  return a.data + (((page * a.H + h) << sh) + (jb & ((1 << sh) - 1))) * BYTES;
}

// x of the lane that DPP control CTL names (0 past a row's end).
template <int CTL>
__device__ __forceinline__ float from_lane(float x) {
  return __builtin_bit_cast(
      float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTL, 0xf, 0xf, true));
}
constexpr int kRor8 = 0x128, kHalfMirror = 0x141, kXor2 = 0x4E, kXor1 = 0xB1, kShl4 = 0x104;

// Sums over lanes of several values: every step leaves half of the values, each with the lane
// (of the two that CTL pairs) that has its bit in n, the lane's number.
template <int CTL, int BIT>
__device__ __forceinline__ float halve(float clear, float set, int n) {
  return (n & BIT ? set : clear) + from_lane<CTL>(n & BIT ? clear : set);
}
// v[n % COUNT] over the COUNT lanes that differ in these bits of n.
template <int COUNT>
__device__ __forceinline__ float lanes_sum(const float* v, int n) {
  if constexpr (COUNT == 1) {
    return v[0];
  } else {
    constexpr int CTL = COUNT == 16 ? kRor8 : COUNT == 8 ? kHalfMirror : COUNT == 4 ? kXor2 : kXor1;
    float x[COUNT / 2];
#pragma unroll
    for (int e = 0; e < COUNT / 2; ++e) x[e] = halve<CTL, COUNT / 2>(v[e], v[e + COUNT / 2], n);
    return lanes_sum<COUNT / 2>(x, n);
  }
}

// Blocks that a (sequence, head) has entries to write in.
__device__ __forceinline__ int blocks_of(const MassParams& a, const Place& s) {
  return static_cast<int>(((a.clear ? a.M : s.end) + kCacheBlock - 1) / kCacheBlock);
}

// What token j has collected before (a new token: nothing).
__device__ __forceinline__ float before(const MassParams& a, const Place& s, int64_t bh, int j) {
  return a.mass && j < s.p_first && j < s.end ? a.mass[bh * a.M + j] : 0.0f;
}

// Token j's sum.
__device__ __forceinline__ void collect(const MassParams& a, const Place& s, int64_t bh, int j,
                                        float old, float w) {
  const int64_t at = bh * a.M + j;
  if (j >= s.end) {
    if (a.clear && j < a.M) a.out[at] = 0.0f;
    return;
  }
  a.out[at] = __builtin_fmaf(a.decay, old, w);
}

// Few rows, T times 16 at most: waves take blocks of 32 tokens in turn.  HALF, up to eight
// rows: the 16 columns of the matrix instructions hold them twice, once for either 16 tokens
// of a block, which halves the work per score.
template <int D, int BITS, bool HALF, int T>
__global__ __launch_bounds__(256) void k_mass_few(const MassParams a) {
  using L = CacheLayout<D, BITS>;
  constexpr int G = L::kG, DW = L::kDw, ST = D / 32;
  constexpr int NT = HALF ? 1 : 2;   // groups of four tokens whose scores a lane holds
  const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int h = blockIdx.y;
  const int64_t b = blockIdx.z, bh = b * a.H + h;
  const Place s = place_of(a, b);
  const int blocks = blocks_of(a, s);
  const int step = gridDim.x * 4;
  int jb = blockIdx.x * 4 + wave;
  if (jb >= blocks) return;

  static_assert(!HALF || T == 1);
  const bool second = HALF && (n & 8);   // the lane's columns are for the block's last 16 tokens
  Rows<D, BITS> rows[T];
  float to_log2[T], off[T];
  int pos[T];
#pragma unroll
  for (int t = 0; t < T; ++t) {
    const int row = 16 * t + (HALF ? n & 7 : n);
    const int tok = row / a.group, hq = h * a.group + row % a.group;
    bool have = row < s.rows;
    const float lse = have ? a.lse[(b * a.H * a.group + hq) * a.n + tok] : kNegInf;
    have = have && lse != kNegInf;
    rows[t].load(a.q + b * a.q_sB + hq * a.q_sH + tok * a.q_sN, have, g);
    to_log2[t] = a.scale_log2 * rows[t].unscale;
    off[t] = have ? lse * kLog2e : INFINITY;   // a row that is not there weighs 0
    pos[t] = have ? s.p_first + tok : -1;
  }
  const int p_lo = s.p_first, p_hi = s.p_first + (s.rows - 1) / a.group;

  auto seen = [&](int i) __attribute__((always_inline)) {   // by some row
    const int j0 = i * kCacheBlock;
    return s.rows > 0 && j0 <= p_hi && (j0 + 31 > p_lo - a.window || j0 < a.sinks);
  };
  struct Keys {
    uint32_t c[L::kRun], p[NT][4 * G];
    float old;
  };
  // The lane's token in what is written of a block, element n % 4 of one of its tiles; half
  // of the lanes write one.
  const bool writes = HALF ? (n & 4) == 0 : n < 8;
  auto token = [&](int i) __attribute__((always_inline)) {
    return i * kCacheBlock + 2 * (HALF ? n & 8 : 2 * (n & 4)) + 4 * g + (n & 3);
  };
  auto load = [&](Keys& x, int i, int page) __attribute__((always_inline)) {
    x.old = i < blocks && writes ? before(a, s, bh, token(i)) : 0.0f;
    const uint8_t* blk = i < blocks && seen(i) ? keys_of<L::kBytes>(a, page, h, i) : nullptr;
    if (!blk) return false;
#pragma unroll
    for (int c = 0; c < L::kRun / 4; ++c)
      *reinterpret_cast<u32x4*>(x.c + 4 * c) =
          *reinterpret_cast<const u32x4*>(blk + (c * 64 + lane) * 16);
#pragma unroll
    for (int tl = 0; tl < NT; ++tl)
#pragma unroll
      for (int c = 0; c < G; ++c)
        *reinterpret_cast<u32x4*>(x.p[tl] + 4 * c) = *reinterpret_cast<const u32x4*>(
            blk + L::kCodes + (16 * (HALF ? n >> 3 : tl) + 4 * g) * G * 4 + 16 * c);
    return true;
  };
  auto work = [&](const Keys& x, bool held, int i) __attribute__((always_inline)) {
    const int j0 = i * kCacheBlock, j = token(i);
    float w = 0.0f;
    if (held) {
      const bool masked = j0 + 31 > p_lo || (j0 <= p_hi - a.window && j0 + 31 >= a.sinks);
      f32x4 acc[2][T][G];
      float sums[4 * NT];
      auto multiply = [&](int tl) __attribute__((always_inline)) {
#pragma unroll
        for (int t = 0; t < T; ++t)
#pragma unroll
          for (int gi = 0; gi < G; ++gi) acc[tl][t][gi] = f32x4{};
#pragma unroll
        for (int st = 0; st < ST; ++st)
#pragma unroll
          for (int t = 0; t < T; ++t)
            acc[tl][t][st / 2] = rows[t].dot(x.c + (tl * ST + st) * DW, st, acc[tl][t][st / 2]);
      };
      multiply(0);
      if constexpr (HALF) multiply(1);
#pragma unroll
      for (int tl = 0; tl < NT; ++tl) {
        if (tl > 0) multiply(tl);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float all = 0.0f;
#pragma unroll
          for (int t = 0; t < T; ++t) {
            float y = 0.0f;
#pragma unroll
            for (int gi = 0; gi < G; ++gi) {
              const float c = HALF && second ? acc[1][t][gi][e] : acc[tl][t][gi][e];
              y = __builtin_fmaf(high_of(x.p[tl][e * G + gi]), c, y);
              y = __builtin_fmaf(low_of(x.p[tl][e * G + gi]), rows[t].sum[gi], y);
            }
            y = __builtin_amdgcn_exp2f(__builtin_fmaf(y, to_log2[t], -off[t]));
            if (masked) {
              const int jt = j0 + (HALF ? 2 * (n & 8) : 16 * tl) + 4 * g + e;
              y = jt <= pos[t] && (jt > pos[t] - a.window || jt < a.sinks) ? y : 0.0f;
            }
            all = t == 0 ? y : all + y;
          }
          sums[4 * tl + e] = all;
        }
      }
      // To the lanes that write: of 16 columns, or of each half of them.
      w = lanes_sum<4 * NT>(sums, n);
      w += HALF ? from_lane<kShl4>(w) : from_lane<kRor8>(w);
    }
    if (writes && (held || !a.in_place || j >= s.p_first)) collect(a, s, bh, j, x.old, w);
  };
  // Each block is fetched while the one before is worked on, its page's entry one block
  // earlier still.
  Keys cur, nxt;
  int page = page_of(a, b, jb + step);
  bool held = load(cur, jb, page_of(a, b, jb));
  while (jb < blocks) {
    const bool more = load(nxt, jb + step, page);
    page = page_of(a, b, jb + 2 * step);
    work(cur, held, jb);
    jb += step;
    if (jb >= blocks) break;
    held = load(cur, jb + step, page);
    page = page_of(a, b, jb + 2 * step);
    work(nxt, more, jb);
    jb += step;
  }
}

// More rows, in tiles of 32, brought once into the form in which the products take them: as
// they are, and with what starts their scores (in log2 units), the sums over each group's
// values and less the lse.  bf16 is their own type and holds codes of 8 bits exactly.
template <int D>
struct RowTile {
  static constexpr int kRowBytes = 2 * D + 16;   // rows 16 bytes apart in the banks
  uint8_t q[32 * kRowBytes];
  u32x4 start[2][32];   // as three bf16 that add up to them: each group's sum; less the lse
  float off[32];        // the lse; inf where the row weighs nothing
};

// One tile per workgroup, eight threads a row.
template <int D, int BITS>
__global__ __launch_bounds__(256) void k_mass_rows(const MassParams a, RowTile<D>* out) {
  constexpr int C = D / 64;   // 16-byte chunks per thread
  const int h = blockIdx.y;
  const int64_t b = blockIdx.z;
  const Place s = place_of(a, b);
  const int t = blockIdx.x;
  if (32 * t >= s.rows) return;
  RowTile<D>& to = out[(b * a.H + h) * gridDim.x + t];
  const int sr = threadIdx.x >> 3, sc = threadIdx.x & 7;
  const int row = 32 * t + sr;
  const int tok = row / a.group, hq = h * a.group + row % a.group;
  const float lse = row < s.rows ? a.lse[(b * a.H * a.group + hq) * a.n + tok] : kNegInf;
  const bool have = lse != kNegInf;
  float sum[C];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    u32x4 x = {0, 0, 0, 0};
    if (have)
      x = *reinterpret_cast<const u32x4*>(a.q + b * a.q_sB + hq * a.q_sH + tok * a.q_sN +
                                          8 * (c * 8 + sc));
    *reinterpret_cast<u32x4*>(to.q + sr * RowTile<D>::kRowBytes + 16 * (c * 8 + sc)) = x;
    sum[c] = 0.0f;
#pragma unroll
    for (int e = 0; e < 4; ++e) sum[c] += low_of(x[e]) + high_of(x[e]);
  }
#pragma unroll
  for (int o = 1; o < 8; o <<= 1)
#pragma unroll
    for (int c = 0; c < C; ++c) sum[c] += __shfl_xor(sum[c], o);   // chunks c hold group c
  if (sc > 0) return;
  const float off = have ? lse * kLog2e : INFINITY;
  uint32_t part[9] = {};
  auto cut = [&](float x, int at) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      const uint32_t bits = __float_as_uint(x) & 0xFFFF0000u;   // eight leading bits
      part[at + i] = bits >> 16;
      x = (bits & 0x7F800000u) == 0x7F800000u ? 0.0f : x - __uint_as_float(bits);
    }
  };
#pragma unroll
  for (int c = 0; c < C; ++c) cut(sum[c] * a.scale_log2, 3 * c);
  cut(-off, 6);
  to.start[0][sr] = u32x4{part[0] | part[1] << 16, part[2] | part[3] << 16, part[4] | part[5] << 16, 0u};
  to.start[1][sr] = u32x4{part[6] | part[7] << 16, part[8], 0u, 0u};
  to.off[sr] = off;
}

// A block of 32 tokens per wave stays in registers as bf16 codes, and the row tiles pass by
// in LDS, fetched two ahead by the workgroup's four waves.  v_mfma_f32_32x32x16 (lane l =
// 32 g + n): A: token n, head-dim values 16 st + 8 g + 0..7; B: row n, the same; C: row n,
// tokens 8 (e / 4) + 4 g + e % 4.  The m_G sum(q_G) terms and the lse start the sums, m_G
// being bf16 as it is; what is left per score is a product and sum for each group, an exp2
// and its sum.  Row tiles that see all of the workgroup's tokens, most of them, pass without
// masks, in a loop of their own.
template <int D, int BITS>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(3))) void k_mass_many(
    const MassParams a, const RowTile<D>* row_tiles, int32_t tiles_held) {
  using L = CacheLayout<D, BITS>;
  using Tile = RowTile<D>;
  constexpr int G = L::kG, DW = L::kDw, ST = D / 16, SW = D / 32;
  constexpr int U = (sizeof(Tile) + 4095) / 4096;   // direct loads per wave and tile
  __shared__ __align__(16) uint8_t ring[3][U * 4096];
  const int lane = threadIdx.x & 63, n = lane & 31, g = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int h = blockIdx.y;
  const int64_t b = blockIdx.z, bh = b * a.H + h;
  const int page = page_of(a, b, blockIdx.x / a.splits * 4 + wave);   // beside what follows
  const Place s = place_of(a, b);
  const int blocks = blocks_of(a, s);
  const int split = blockIdx.x % a.splits;
  const int first = blockIdx.x / a.splits * 4;   // the workgroup's blocks
  if (first >= blocks) return;
  const int jb = first + wave, j0 = jb * kCacheBlock;

  // Row tiles: [t0, c0) and [c1, ntiles) with masks, [c0, c1) whole; those before t0 see
  // none of the workgroup's tokens [j_lo, j_hi].
  int ntiles = first * kCacheBlock < s.end ? (s.rows + 31) / 32 : 0;
  const int j_lo = first * kCacheBlock, j_hi = min(j_lo + 4 * kCacheBlock, s.end) - 1;
  auto tile_at = [&](int64_t row) __attribute__((always_inline)) {
    const int64_t t = row < 0 ? 0 : row >> 5;
    return t < ntiles ? static_cast<int>(t) : ntiles;
  };
  const int64_t off_lo = int64_t(j_lo) - s.p_first, off_hi = int64_t(j_hi) - s.p_first;
  int t0 = tile_at(off_lo * a.group), c0 = tile_at(off_hi * a.group + 31);
  int c1 = j_hi < a.sinks ? ntiles : tile_at((off_lo + a.window) * a.group);
  // Of these the workgroup's share.
  const int share = (ntiles - t0 + a.splits - 1) / a.splits;
  t0 = min(t0 + split * share, ntiles);
  ntiles = min(t0 + share, ntiles);
  c0 = min(max(c0, t0), ntiles);
  c1 = min(max(c1, c0), ntiles);

  const Tile* tiles = row_tiles + bh * tiles_held;
  auto fetch = [&](int t, int st) __attribute__((always_inline)) {
    const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<Tile*>(tiles + t), 0, sizeof(Tile), 0x00020000);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int at = (wave * U + u) * 1024;
      gather16_to_lds(rs, at + 16 * lane, ring[st] + at);
    }
  };
  if (t0 < ntiles) {
    fetch(t0, 0);
    fetch(min(t0 + 1, ntiles - 1), 1);
  }

  // A block that no page holds passes as some other, and its sums are left out at the end.
  const uint8_t* blk = j0 < s.end ? keys_of<L::kBytes>(a, page, h, jb) : nullptr;
  const uint8_t* src = blk ? blk : a.data;
  bf16x8 codes[ST];
  float step_of[G][16], w[16];
#pragma unroll
  for (int e = 0; e < 16; ++e) w[e] = 0.0f;
  // Token n = 16 t + n % 16, values 16 st + 8 g on: run dword (t D / 32 + st / 2) kDw
  // of lane 16 (2 (st % 2) + g) + n % 16.
  constexpr int RUN = SW * DW, LOAD = RUN < 4 ? RUN : 4;
  typedef uint32_t Words __attribute__((ext_vector_type(LOAD)));
  Words u[2][RUN / LOAD];
#pragma unroll
  for (int odd = 0; odd < 2; ++odd)
#pragma unroll
    for (int c = 0; c < RUN / LOAD; ++c)
      u[odd][c] = *reinterpret_cast<const Words*>(
          src + code_byte((n >> 4) * RUN + c * LOAD, (2 * odd + g) * 16 + (n & 15)));
  const uint32_t* par = reinterpret_cast<const uint32_t*>(src + L::kCodes);
  u32x4 steps[4][G];
#pragma unroll
  for (int q = 0; q < 4; ++q)
#pragma unroll
    for (int c = 0; c < G; ++c)
      steps[q][c] = reinterpret_cast<const u32x4*>(par + (8 * q + 4 * g) * G)[c];
  const uint32_t m0 = par[n * G] & 0xFFFFu, m1 = G > 1 ? par[n * G + G - 1] & 0xFFFFu : 0u;
  const bf16x8 low = __builtin_bit_cast(
      bf16x8, g == 0 ? u32x4{m0 | m0 << 16, m0 | m1 << 16, m1 | m1 << 16, 0u}
                     : u32x4{0x3F803F80u, 0x3F80u, 0u, 0u});   // 1, 1, 1
#pragma unroll
  for (int st = 0; st < ST; ++st) {
    uint32_t run[DW];
#pragma unroll
    for (int y = 0; y < DW; ++y) {
      const int at = st / 2 * DW + y;
      run[y] = u[st & 1][at / LOAD][at % LOAD];
    }
    u32x4 x = codes_16<BITS>(run);
#pragma unroll
    for (int y = 0; y < 4; ++y)
      x[y] = __float_as_uint(static_cast<float>(x[y] & 0xFFu)) >> 16 |
             (__float_as_uint(static_cast<float>(x[y] >> 16)) & 0xFFFF0000u);
    codes[st] = __builtin_bit_cast(bf16x8, x);
  }
#pragma unroll
  for (int e = 0; e < 16; ++e)
#pragma unroll
    for (int gi = 0; gi < G; ++gi) {
      const int at = e % 4 * G + gi;
      step_of[gi][e] = a.scale_log2 * high_of(steps[e / 4][at / 4][at % 4]);
    }

  int st = 0;
  auto turn = [&](int t, auto masked_tag) __attribute__((always_inline)) {
    wait_vmcnt<U>();   // of the tile after it
    __builtin_amdgcn_s_barrier();
    // Past the last tile that one is fetched again (into a stage that nothing reads).
    fetch(min(t + 2, ntiles - 1), st == 0 ? 2 : st - 1);
    const Tile& tile = *reinterpret_cast<const Tile*>(ring[st]);
    st = st == 2 ? 0 : st + 1;
    const u32x4 first_terms = tile.start[g][n];
    const uint8_t* qrow = tile.q + n * Tile::kRowBytes + 16 * g;
    const f32x16 start = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
        low, __builtin_bit_cast(bf16x8, first_terms), f32x16{}, 0, 0, 0);
    f32x16 acc[G];
#pragma unroll
    for (int gi = 0; gi < G; ++gi) acc[gi] = f32x16{};
#pragma unroll
    for (int st = 0; st < ST; ++st)
      acc[st / 4] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
          codes[st], __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(qrow + 32 * st)),
          acc[st / 4], 0, 0, 0);
    const int pos = tile.off[n] == INFINITY ? -1 : s.p_first + (32 * t + n) / a.group;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      float y = start[e];
#pragma unroll
      for (int gi = 0; gi < G; ++gi) y = __builtin_fmaf(step_of[gi][e], acc[gi][e], y);
      y = __builtin_amdgcn_exp2f(y);
      if constexpr (decltype(masked_tag)::value) {
        const int j = j0 + 8 * (e / 4) + 4 * g + e % 4;
        y = j <= pos && (j > pos - a.window || j < a.sinks) ? y : 0.0f;
      }
      w[e] += y;
    }
  };
#pragma unroll 1
  for (int t = t0; t < c0; ++t) turn(t, std::true_type{});
#pragma unroll 1
  for (int t = c0; t < c1; ++t) turn(t, std::false_type{});
#pragma unroll 1
  for (int t = c1; t < ntiles; ++t) turn(t, std::true_type{});
  wait_all();

  const int j = j0 + 8 * ((n & 15) / 4) + 4 * g + (n & 3);
  const bool writes = n < 16 && jb < blocks;
  const float old = writes && a.splits == 1 ? before(a, s, bh, j) : 0.0f;
  float mine = lanes_sum<16>(w, n);
  mine += __shfl_xor(mine, 16);
  if (!writes) return;
  if (!blk) mine = 0.0f;
  if (a.splits == 1) collect(a, s, bh, j, old, mine);
  else a.part[(static_cast<int64_t>(split) * gridDim.z * a.H + bh) * a.slots + j] = mine;
}

// The sums of a token's rows, split by split.
__global__ __launch_bounds__(256) void k_mass_join(const MassParams a) {
  const int h = blockIdx.y;
  const int64_t b = blockIdx.z, bh = b * a.H + h, heads = static_cast<int64_t>(gridDim.z) * a.H;
  const Place s = place_of(a, b);
  const int j = blockIdx.x * 256 + threadIdx.x;
  if (j >= min(a.slots, kCacheBlock * static_cast<int64_t>(blocks_of(a, s)))) return;
  float w = 0.0f;
  for (int i = 0; i < a.splits; ++i) w += a.part[(i * heads + bh) * a.slots + j];
  collect(a, s, bh, j, before(a, s, bh, j), w);
}

template <int D>
size_t row_tiles_bytes(int64_t heads, int64_t rows) {
  return static_cast<size_t>(heads) * ((rows + 31) / 32) * sizeof(RowTile<D>);
}

// Rows whose columns the waves of k_mass_few hold: sixteen to a register tile, three of those
// (4 x 131072 tokens, 4 heads of 128 in 4 bits: 34 us for 7 rows, 38 for 14, 57 for 28, 68 for
// 42, where k_mass_many takes 104; both about 100 for 63).
constexpr int kFewRows = 48;

// Where blocks alone leave CUs without a workgroup (a CU holds three), their rows are split
// among as many as fill them, with eight tiles each at least (512 tokens of 28 heads over 512
// tokens: 23 us, 77 in one; over 8192: 61 and 81).
constexpr int64_t kFill = 3 * 256, kLeastTiles = 8;
int64_t splits_of(int64_t groups, int64_t rows) {
  return std::max<int64_t>(1, std::min(kFill / groups, rows / (32 * kLeastTiles)));
}
size_t parts_bytes(int64_t rows) {
  return rows < 64 * kLeastTiles ? 0 : kFill * 4 * kCacheBlock * sizeof(float);
}

}  // namespace

size_t cache_mass_workspace_bytes(const CacheAttnShape& s) {
  const int64_t rows = s.n * (s.Hq / s.H);
  if (rows <= kFewRows) return 0;
  return parts_bytes(rows) + (s.D == 128 ? row_tiles_bytes<128>(s.B * s.H, rows)
                                         : row_tiles_bytes<64>(s.B * s.H, rows));
}

hipError_t launch_cache_mass(const CacheMassArgs& x, hipStream_t stream) {
  const CacheArgs& c = x.cache;
  MassParams a;
  a.q = static_cast<const uint16_t*>(x.q.ptr);
  a.q_sB = x.q.sB, a.q_sH = x.q.sH, a.q_sN = x.q.sN;
  a.lse = x.lse;
  a.data = static_cast<const uint8_t*>(c.data);
  a.table = c.table;
  a.lens = c.lens;
  a.n_new = x.n_new;
  a.mass = x.mass;
  a.out = x.out;
  a.M = x.M;
  a.cols = static_cast<int32_t>(c.cols);
  a.pages = static_cast<int32_t>(std::min<int64_t>(c.pages, INT32_MAX));
  a.page_shift = __builtin_ctz(static_cast<unsigned>(c.page));
  a.H = c.H;
  a.n = static_cast<int32_t>(x.q.N);
  a.group = static_cast<int32_t>(x.q.H / c.H);
  a.window = static_cast<int32_t>(x.window);
  a.sinks = static_cast<int32_t>(x.sinks);
  a.in_place = x.mass == x.out && x.decay == 1.0f;
  a.clear = x.clear;
  const float scale = x.scale != 0.0f ? x.scale : 1.0f / sqrtf(static_cast<float>(c.D));
  a.scale_log2 = scale * kLog2e;
  a.decay = x.decay;
  const int64_t rows = static_cast<int64_t>(a.n) * a.group;
  const int64_t blocks = (x.M + kCacheBlock - 1) / kCacheBlock;
  const int64_t heads = x.q.B * c.H;
  auto launch = [&](auto kernel, int64_t groups, auto... more) {
    hipLaunchKernelGGL(kernel,
                       dim3(static_cast<unsigned>(groups), static_cast<unsigned>(c.H),
                            static_cast<unsigned>(x.q.B)),
                       dim3(256), 0, stream, a, more...);
  };
  auto pick = [&](auto dim, auto bits) {
    constexpr int D = decltype(dim)::value, BITS = decltype(bits)::value;
    if (rows <= kFewRows) {
      // Two workgroups per place on the CUs, so that unequal lengths even out (4 x 131072
      // tokens, 4 heads: 34 us, also with half of them; 37 with twice as many).
      const int64_t fill = std::max<int64_t>(1, 2048 / heads);
      const int64_t groups = std::min((blocks + 3) / 4, fill);
      if (rows <= 8) launch(k_mass_few<D, BITS, true, 1>, groups);
      else if (rows <= 16) launch(k_mass_few<D, BITS, false, 1>, groups);
      else if (rows <= 32) launch(k_mass_few<D, BITS, false, 2>, groups);
      else launch(k_mass_few<D, BITS, false, 3>, groups);
    } else {
      RowTile<D>* prepared = static_cast<RowTile<D>*>(x.workspace);
      const int64_t tiles = (rows + 31) / 32;
      launch(k_mass_rows<D, BITS>, tiles, prepared);
      const int64_t groups = (blocks + 3) / 4;
      a.splits = static_cast<int32_t>(splits_of(groups * heads, rows));
      a.slots = groups * 4 * kCacheBlock;
      a.part = reinterpret_cast<float*>(static_cast<uint8_t*>(x.workspace) +
                                        row_tiles_bytes<D>(heads, rows));
      launch(k_mass_many<D, BITS>, groups * a.splits, prepared, static_cast<int32_t>(tiles));
      if (a.splits > 1) launch(k_mass_join, (a.slots + 255) / 256);
    }
  };
  using std::integral_constant;
  if (c.D == 128)
    c.bits == 4 ? pick(integral_constant<int, 128>{}, integral_constant<int, 4>{})
                : pick(integral_constant<int, 128>{}, integral_constant<int, 8>{});
  else
    c.bits == 4 ? pick(integral_constant<int, 64>{}, integral_constant<int, 4>{})
                : pick(integral_constant<int, 64>{}, integral_constant<int, 8>{});
  return hipGetLastError();
}

}  // namespace vecattn
