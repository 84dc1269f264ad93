// Attention of many rows over the quantised cache (a chunk of a prompt, or drafts of
// many heads): the cache's values are rebuilt once per 128 rows.
//
// A workgroup owns 128 or 256 rows (row = token * group + head; waves of 32) and walks
// its chunk of the tokens in tiles of 64 (two blocks of the cache).  The codes of a
// tile are fetched two tiles ahead and put into LDS one tile ahead, in the order in
// which the matrix instructions take them: K as [eight head-dim values][token], V as
// [eight tokens][head-dim value], 16 bytes each, which is how the cache holds them, so
// that neither needs a transpose.
//   K goes in as it is, fp16 numbers whose bits are the code; its steps s are applied
//   to the scores, and sum_G m_G sum(q_G) comes from a product of the m, bf16 as they
//   are, with the sums in three bf16 parts: nothing is rounded but fp32 sums.
//   V goes in as fp16 values m + s u (rounded once, 2^-11, by one packed fma per pair),
//   in units of a power of two above the largest value of the tiles so far, which O
//   follows; the softmax weights are fp16 too, 2^7 at a row's maximum (below 2^-21 of
//   that they lose bits, below 2^-32 they are 0).  Where V's groups lie more than 2^16
//   apart the tiles are walked once per such range.
// S^T = K Q^T and O^T += V^T P^T run on v_mfma_f32_32x32x16_f16.  A row of q is scaled
// by a power of two to its largest value.
//
// What bounds it: VALU work that runs beside the products only in part (per score two
// scalings, an exponential with its argument, sum and rounding; the rebuilding), and
// registers, all 256 of which are taken, so that two waves per SIMD are the most.  512
// tokens of 28 query and 4 key/value heads of 128 over 33280 tokens of 8 bits: 358 us
// with the join (242 GFLOP, 677 TFLOP/s), of which a walk with K rounded to fp16 values
// saves 20 and loses two digits of lse.
//
// MFMA 32x32x16 lane layout as in sparse_attn.hip: A: row l % 32, K-slots 8 g ..
// 8 g + 7 (g = l / 32); B: column l % 32, the same slots; C: column l % 32, rows
// 8 * (v / 4) + 4 g + v % 4.
#include <type_traits>

#include "cache_plan.h"

namespace vecattn {
namespace {

typedef const __attribute__((address_space(4))) int32_t* ScalarInts;

constexpr int kTile = 64;       // tokens per tile
constexpr float kBias = 7.0f;   // log2 of the weight at a row's reference
constexpr int kBand = 16;       // powers of two that V's fp16 values hold at once

// Largest value over the wave, on every lane (a scalar).
__device__ __forceinline__ uint32_t wave_max(uint32_t x) {
  auto step = [&](auto ctrl, auto rows) __attribute__((always_inline)) {
    x = max(static_cast<uint32_t>(__builtin_amdgcn_update_dpp(
                0, static_cast<int>(x), decltype(ctrl)::value, decltype(rows)::value, 0xf, false)),
            x);   // 0 where no lane is read: max changes nothing, and takes the move in
  };
  using std::integral_constant;
  step(integral_constant<int, 0x111>{}, integral_constant<int, 0xf>{});   // row_shr:1
  step(integral_constant<int, 0x112>{}, integral_constant<int, 0xf>{});
  step(integral_constant<int, 0x114>{}, integral_constant<int, 0xf>{});
  step(integral_constant<int, 0x118>{}, integral_constant<int, 0xf>{});
  step(integral_constant<int, 0x142>{}, integral_constant<int, 0xa>{});   // row_bcast:15
  step(integral_constant<int, 0x143>{}, integral_constant<int, 0xc>{});   // row_bcast:31
  return __builtin_amdgcn_readlane(x, 63);
}

// Barrier for LDS alone: the wave's loads from memory stay in flight.
__device__ __forceinline__ void lds_barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0xC07F);   // lgkmcnt(0)
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// Eight codes as 1024 + u in fp16 (exact), in slot order.
template <int BITS>
__device__ __forceinline__ u32x4 codes_1024(const uint32_t* w) {
  const u32x4 x = codes_16<BITS>(w);
  return u32x4{x[0] | 0x64006400u, x[1] | 0x64006400u, x[2] | 0x64006400u, x[3] | 0x64006400u};
}

template <int D>
struct Shared {
  f16x8 k[2][D / 8][kTile];
  // K's steps of the last group, and of the first in units of them.
  __align__(16) float step[2][kTile], ratio[2][kTile];
  f16x8 v[2][2][4][D];
  uint32_t low[64];   // smallest magnitude of V's groups, by the lane that met it
  int redo;
};

// A second walk's first and last power of two of V.
struct Bands {
  int low, top;
};

// A workgroup's work, W waves of 32 rows.  Not CAREFUL: false, and nothing is written,
// if a careful walk has to follow.
template <int D, int BITS, int W, bool CAREFUL>
__device__ __forceinline__ bool walk(const AttnParams& a, Shared<D>& shared, Bands& bands) {
  using L = CacheLayout<D, BITS>;
  constexpr int G = L::kG, DW = L::kDw, DS = D / 16, DB = D / 32;
  constexpr int kChunks = L::kRun / 4;      // 1 KB pieces of a block's K or V codes
  constexpr int kUnits = 2 * kChunks;       // of a tile's
  constexpr bool kSplit = 2 * kUnits <= W;  // a wave takes a piece of K or one of V
  constexpr int kPer = kSplit ? 1 : kUnits / W;   // pieces a wave takes of either
  constexpr int kRows = 32 * W;
  constexpr int kItems = 4 / DW;            // octets of codes in a lane's 16 bytes
  auto& k_s = shared.k;
  auto& v_s = shared.v;
  auto &step_s = shared.step, &ratio_s = shared.ratio;

  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 5, ln = lane & 31;
  const int n16 = lane & 15, g16 = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);

  const int h = blockIdx.x % a.H;
  const int index = blockIdx.x / a.H;
  const Share share = find_share(a, kRows, index);
  if (share.unit < 0) return true;
  if (a.target && h == 0 && index == share.first && tid == 0)
    shares_of(a, kRows, D)[share.unit] = int2{share.first, share.count};
  const int64_t b = share.unit / a.tiles;
  const int row0 = share.unit % a.tiles * kRows;
  const Span s = span_of(a, b, row0, kRows);
  if (row0 >= s.rows) return true;
  const int t0 = (index - share.first) * (share.count > 1 ? share.chunk : 0);   // a multiple of 8
  const int t1 = share.count > 1 ? min(s.total, t0 + share.chunk) : s.total;
  const int ntiles = (t1 - t0 + 1) / 2;

  // This lane's row.
  const int row = row0 + 32 * wave + ln;
  const int tok = row / a.group, hq = h * a.group + row % a.group;
  const bool have = row < s.rows;
  const int pos = have ? s.p_first + tok : -1;
  // Positions of the wave's rows that exist.
  const int w_lo = s.p_first + (row0 + 32 * wave) / a.group;
  const int w_hi = s.p_first + (min(row0 + 32 * wave + 32, s.rows) - 1) / a.group;
  f16x8 qf[DS];
  bf16x8 q_sum;   // a group's sum of q in three parts, against (m, m) pairs (G = 1) or (m_0, m_1)
  float to_log2;
  {
    const u32x4* src =
        reinterpret_cast<const u32x4*>(a.q + b * a.q_sB + hq * a.q_sH + tok * a.q_sN);
    u32x4 w[DS];
    float top = 0x1p-100f;
#pragma unroll
    for (int st = 0; st < DS; ++st) {
      w[st] = u32x4{0, 0, 0, 0};
      if (have) w[st] = src[2 * st + g];
#pragma unroll
      for (int e = 0; e < 4; ++e)
        top = fmaxf(top, fmaxf(fabsf(low_of(w[st][e])), fabsf(high_of(w[st][e]))));
    }
    const int k = 15 - __builtin_amdgcn_frexp_expf(wave_max_xor32(top));
    float sum[2] = {0.0f, 0.0f};
#pragma unroll
    for (int st = 0; st < DS; ++st) {
      u32x4 x;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float lo = low_of(w[st][e]), hi = high_of(w[st][e]);
        sum[st / 4] += lo + hi;
        x[e] = to_f16(__builtin_amdgcn_ldexpf(lo, k), __builtin_amdgcn_ldexpf(hi, k));
      }
      qf[st] = __builtin_bit_cast(f16x8, x);
    }
    float part[2][3];
#pragma unroll
    for (int gi = 0; gi < 2; ++gi) {
      float x = __builtin_amdgcn_ldexpf(sum[gi] + __shfl_xor(sum[gi], 32), k - kCodeExp<BITS>);
#pragma unroll
      for (int i = 0; i < 3; ++i) {
        part[gi][i] = static_cast<float>(static_cast<__bf16>(x));
        x -= part[gi][i];
      }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) q_sum[i] = static_cast<__bf16>(0.0f);
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      if constexpr (G == 2) {
        q_sum[2 * i] = static_cast<__bf16>(part[0][i]);
        q_sum[2 * i + 1] = static_cast<__bf16>(part[1][i]);
      } else {
        q_sum[i] = static_cast<__bf16>(part[0][i]);
      }
    }
    to_log2 = fmaxf(a.scale_log2 * __builtin_amdgcn_ldexpf(1.0f, kCodeExp<BITS> - k), 0x1p-126f);  // -inf * 0
  }

  f32x16 oacc[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) oacc[db] = f32x16{};
  float m_run = kUnseen, l_run = 0.0f;
  int v_exp = -200;   // O is in units of 2^v_exp

  const int sh = a.page_shift - 5;
  const ScalarInts pages = (ScalarInts)(a.table + b * a.cols);
  // A block of the chunk: its first token, and where it lies (NULL: not held, or past
  // the chunk).
  auto first_token = [&](int t) __attribute__((always_inline)) {
    return (t < s.ns ? t : s.nb0 + (t - s.ns)) * kCacheBlock;
  };
  auto place = [&](int t) __attribute__((always_inline)) -> const uint8_t* {
    if (t >= t1) return nullptr;
    const int jb = first_token(t) / kCacheBlock;
    const int page = pages[jb >> sh];
    if (page < 0 || page >= a.pages) return nullptr;
    return a.data + (((static_cast<int64_t>(page) * a.H + h) << sh) + (jb & ((1 << sh) - 1))) *
                        L::kBytes;
  };

  // What a wave holds of a tile before it is rebuilt: its pieces' codes, the (m, s) that
  // V's need (they share a block and a group), and every token's, one per lane.
  struct Raw {
    u32x4 kc[kPer], vc[kPer];
    uint32_t vp[8], km[G], vm[G];
    uint32_t held;   // bit per block
  };
  // Which piece: block u / kChunks, 1 KB u % kChunks.
  auto k_unit = [&](int i) __attribute__((always_inline)) { return kSplit ? wave % kUnits : wave * kPer + i; };
  const bool do_k = !kSplit || wave < kUnits;
  const bool do_v = !kSplit || (wave >= kUnits && wave < 2 * kUnits);
  // Of octet i of a K piece: the 16 tokens it is of, and its 32 head-dim values.
  auto k_token16 = [&](int c, int i) __attribute__((always_inline)) { return (c * kItems + i) / (D / 32); };
  auto k_step = [&](int c, int i) __attribute__((always_inline)) { return (c * kItems + i) % (D / 32); };

  auto fetch = [&](Raw& x, int tile) __attribute__((always_inline)) {
    const uint8_t* at[2] = {place(t0 + 2 * tile), place(t0 + 2 * tile + 1)};
    x.held = (at[0] ? 1u : 0u) | (at[1] ? 2u : 0u);
    // A block that is not held is read from the cache's start and not used.
    const uint8_t* blk[2] = {at[0] ? at[0] : a.data, at[1] ? at[1] : a.data};
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int u = k_unit(i), c = u % kChunks;
      const uint8_t* p = u / kChunks ? blk[1] : blk[0];
      if (do_k) x.kc[i] = *reinterpret_cast<const u32x4*>(p + (c * 64 + lane) * 16);
      if (do_v) {
        p += L::kHalf;
        const uint32_t* par = reinterpret_cast<const uint32_t*>(p + L::kCodes);
        x.vc[i] = *reinterpret_cast<const u32x4*>(p + (c * 64 + lane) * 16);
        if (i == 0) {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            x.vp[e] = par[((e >> 2) * 16 + 4 * g16 + (e & 3)) * G + c / DW];
        }
      }
    }
    const uint8_t* p = (lane & 32 ? blk[1] : blk[0]) + L::kCodes + ln * G * 4;
#pragma unroll
    for (int gi = 0; gi < G; ++gi) {
      x.km[gi] = *reinterpret_cast<const uint32_t*>(p + 4 * gi);
      x.vm[gi] = *reinterpret_cast<const uint32_t*>(p + L::kHalf + 4 * gi);
    }
  };
  const int end = s.p_hi + 1;   // tokens from here on are nobody's
  auto left_in = [&](const Raw& x, int tile, int bl) __attribute__((always_inline)) {
    return x.held >> bl & 1u ? min(kCacheBlock, end - first_token(t0 + 2 * tile + bl)) : 0;
  };
  // The larger of a group's |m| and |m + s M|; NaN where it stands for NaN.
  auto group_top = [&](uint32_t w) __attribute__((always_inline)) {
    constexpr float M = BITS == 4 ? 15.0f : 255.0f;
    const float m = low_of(w), hi = __builtin_fmaf(high_of(w), M, m);
    return m == m ? fmaxf(fabsf(m), fabsf(hi)) : m;
  };
  constexpr float kTiny = 0x1p-110f, kHuge = 3.4028234663852886e38f;
  auto exponent_of = [&](float top) __attribute__((always_inline)) {
    return __builtin_amdgcn_frexp_expf(fminf(fmaxf(top, kTiny), kHuge));
  };
  // Rebuilding a tile: prepare, then its pieces (octets of a lane's codes: kPer * kItems
  // of K, as many of V).
  struct Rebuilt {
    f16x2 m2[4], d2[4];   // V's
    uint32_t km;          // K's m of this lane's token, as a pair for the product with q_sum
  };
  const f16x2 minus = {_Float16(-1024.0f), _Float16(-1024.0f)};
  // Raises v_next to V's power.  CAREFUL: V's groups that stand for NaN, and those of
  // another magnitude than 2^band to 2^(band + kBand), become 0.
  auto left_out = [&](uint32_t w, int band) __attribute__((always_inline)) {
    const float t = group_top(w);
    return CAREFUL && (!(t == t) || exponent_of(t) < band || exponent_of(t) > band + kBand);
  };
  auto prepare_k = [&](Raw& x, Rebuilt& y, int tile, int st) __attribute__((always_inline)) {
    // Tokens of no page and those that no row of the workgroup sees: as if m = s = 0.
    const int left[2] = {left_in(x, tile, 0), left_in(x, tile, 1)};
    const int j0[2] = {first_token(t0 + 2 * tile), first_token(t0 + 2 * tile + 1)};
    // Tokens up to `gone` that are no sinks are behind every row's window.
    const int gone = s.p_lo - a.window;
    auto behind = [&](int j) __attribute__((always_inline)) { return j <= gone && j >= a.sinks; };
    if (min(left[0], left[1]) < kCacheBlock || (j0[0] <= gone && j0[0] + 31 >= a.sinks) ||
        (j0[1] <= gone && j0[1] + 31 >= a.sinks)) {
      // (A lane number that is not seen through: nothing of this rare part is held over.)
      int l = lane;
      asm volatile("" : "+v"(l));
      const bool no = (l & 31) >= (l & 32 ? left[1] : left[0]) ||
                      behind((l & 32 ? j0[1] : j0[0]) + (l & 31));
#pragma unroll
      for (int gi = 0; gi < G; ++gi)
        if (no) x.km[gi] = x.vm[gi] = 0u;
      const int bl = k_unit(0) / kChunks;
      const int lim = bl ? left[1] : left[0], first = bl ? j0[1] : j0[0];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int i = (e >> 2) * 16 + (l >> 4 << 2) + (e & 3);
        if (i >= lim || behind(first + i)) x.vp[e] = 0u;
      }
    }
    if (wave == 0) {
      // Scores are step * (ratio * first group's + last group's).  Steps are 0 or from
      // 2^-100 on, and the reciprocal takes no subnormal numbers: a last step of 0 (its
      // codes are 0) is held as 2^-126.  One more than 2^100 below the first is raised
      // to that, so that the ratio is at most 2^100.  (NaN is in m too.)
      const float first = high_of(x.km[0]);
      float step = high_of(x.km[G - 1]);
      if (G == 2) {
        step = fmaxf(fmaxf(step, first * 0x1p-100f), 0x1p-126f);
        ratio_s[st][lane] = first * __builtin_amdgcn_rcpf(step);
      }
      step_s[st][lane] = step;
    }
    y.km = __builtin_amdgcn_perm(x.km[G - 1], x.km[0], 0x05040100u);
  };
  auto prepare_power = [&](const Raw& x, int& v_next, int band) __attribute__((always_inline)) {
    float top = 0.0f, low = kHuge;   // of the token's groups that are not 0
#pragma unroll
    for (int gi = 0; gi < G; ++gi) {
      const float t = left_out(x.vm[gi], band) ? 0.0f : group_top(x.vm[gi]);
      top = fmaxf(top, t);   // NaN: left out
      low = t > 0.0f ? fminf(low, t) : low;
    }
    if (!CAREFUL && wave == 1)
      __hip_atomic_fetch_min(&shared.low[lane], __float_as_uint(low), __ATOMIC_RELAXED,
                             __HIP_MEMORY_SCOPE_WORKGROUP);
    v_next = max(v_next, exponent_of(__uint_as_float(wave_max(__float_as_uint(top)))) - 15);
  };
  auto prepare_v = [&](const Raw& x, Rebuilt& y, int half, int v_next, int band)
                       __attribute__((always_inline)) {
#pragma unroll
    for (int e = 2 * half; e < 2 * half + 2; ++e) {
      float m[2], d[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        uint32_t w = x.vp[2 * e + i];
        if (left_out(w, band)) w = 0u;
        m[i] = __builtin_amdgcn_ldexpf(low_of(w), -v_next);
        d[i] = __builtin_amdgcn_ldexpf(high_of(w), -v_next);
      }
      y.m2[e] = __builtin_bit_cast(f16x2, to_f16(m[0], m[1]));
      y.d2[e] = __builtin_bit_cast(f16x2, to_f16(d[0], d[1]));
    }
  };
  constexpr int kPrepare = 4;
  auto prepare = [&](Raw& x, Rebuilt& y, int step, int tile, int st, int& v_next, int band)
                     __attribute__((always_inline)) {
    if (step == 0) prepare_k(x, y, tile, st);
    else if (step == 1) prepare_power(x, v_next, band);
    else prepare_v(x, y, step - 2, v_next, band);
  };
  constexpr int kPieces = 2 * kPer * kItems;
  auto piece = [&](const Raw& x, const Rebuilt& y, int i, int st) __attribute__((always_inline)) {
    const int per = i % (kPer * kItems) / kItems, it = i % kItems;
    const int u = k_unit(per), c = u % kChunks, bl = u / kChunks;
    uint32_t cw[DW];
    if (i < kPer * kItems) {
      if (!do_k) return;
#pragma unroll
      for (int e = 0; e < DW; ++e) cw[e] = x.kc[per][it * DW + e];
      k_s[st][4 * k_step(c, it) + g16][32 * bl + 16 * k_token16(c, it) + n16] =
          __builtin_bit_cast(f16x8, codes_f16<BITS>(cw));
    } else {
      if (!do_v) return;
#pragma unroll
      for (int e = 0; e < DW; ++e) cw[e] = x.vc[per][it * DW + e];
      u32x4 r = codes_1024<BITS>(cw);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t pair = r[e];
        r[e] = __builtin_bit_cast(uint32_t,
                                  __builtin_elementwise_fma(__builtin_bit_cast(f16x2, pair) + minus,
                                                            y.d2[e], y.m2[e]));
      }
      v_s[st][bl][g16][16 * (c * kItems + it) + n16] = __builtin_bit_cast(f16x8, r);
    }
  };

  auto sees = [&](int j) __attribute__((always_inline)) {
    return j <= pos && (j > pos - a.window || j < a.sinks);
  };
  // Tile `tile` in stage st (km: its tokens' m): scores, weights, products.  Operands
  // are read four instructions ahead; `between` runs beside the score products.
  constexpr int kAhead = 4;
  auto work = [&](int tile, int st, uint32_t km, uint32_t blocks, auto&& between)
                  __attribute__((always_inline)) {
    f32x16 sc[2];
    {
      f16x8 ring[kAhead];
      f32x16 acc[2] = {f32x16{}, f32x16{}};
      // Instruction i: half i / 4 % 2, 16 head-dim values of group i / 8.
      auto read = [&](int i) __attribute__((always_inline)) {
        if (i < 2 * DS)
          ring[i % kAhead] = k_s[st][2 * (i / 8 * 4 + i % 4) + g][32 * (i / 4 % 2) + ln];
      };
      // What the scores need beside the products, four values of a lane at a time, one per
      // instruction from the fifth on: with two groups first the first one's sums into the
      // second's steps (before those are added), then the steps and the m's share.  The
      // factors are read two instructions before.
      constexpr int kJobs = 8 * G;
      f32x4 factor[3];
      auto read_factor = [&](int job) __attribute__((always_inline)) {
        if (job < 0 || job >= kJobs) return;
        const float* x = job < 8 * (G - 1) ? ratio_s[st] : step_s[st];
        factor[job % 3] = *reinterpret_cast<const f32x4*>(x + 32 * (job / 4 % 2) + 8 * (job % 4) + 4 * g);
      };
      auto apply = [&](int job) __attribute__((always_inline)) {
        if (job < 0) return;
        const int hf = job / 4 % 2;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int at = 4 * (job % 4) + e;
          if (job < 8 * (G - 1)) acc[hf][at] *= factor[job % 3][e];
          else sc[hf][at] = __builtin_fmaf(acc[hf][at], factor[job % 3][e], sc[hf][at]);
        }
      };
      // sum_G m_G sum(q_G): lanes 32 hf .. + 31 hold the half's tokens.
      auto m_share = [&](int hf) __attribute__((always_inline)) {
        const uint32_t m = g == hf ? km : 0u;
        sc[hf] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
            __builtin_bit_cast(bf16x8, u32x4{m, m, m, 0u}), q_sum, f32x16{}, 0, 0, 0);
      };
#pragma unroll
      for (int i = 0; i < kAhead; ++i) read(i);
#pragma unroll
      for (int i = 0; i < 2 * DS; ++i) {
        const int hf = i / 4 % 2;
        __builtin_amdgcn_sched_barrier(0);
        acc[hf] = __builtin_amdgcn_mfma_f32_32x32x16_f16(ring[i % kAhead], qf[i / 8 * 4 + i % 4],
                                                         acc[hf], 0, 0, 0);
        read(i + kAhead);
        read_factor(i - 2);
        between(i);
        apply(i - 4);
        if (i == 2 * DS - 5) m_share(0);
      }
      __builtin_amdgcn_sched_barrier(0);
      m_share(1);
#pragma unroll
      for (int i = 2 * DS; i < 2 * DS + 4; ++i) {
        read_factor(i - 2);
        apply(i - 4);
      }
    }
#pragma unroll
    for (int hf = 0; hf < 2; ++hf) {
      const int j0 = first_token(t0 + 2 * tile + hf);
      const bool held = blocks >> hf & 1u;
      if (held && j0 + 31 <= w_lo && (j0 > w_hi - a.window || j0 + 31 < a.sinks)) continue;
      int l = lane;
      asm volatile("" : "+v"(l));
#pragma unroll
      for (int e = 0; e < 16; ++e)
        sc[hf][e] = held && sees(j0 + 8 * (e / 4) + (l >> 5 << 2) + e % 4) ? sc[hf][e] : kNegInf;
    }
    u32x4 pw[4];   // the weights as operands: of 16 tokens each, pairs in the order of V's
    float sum;
    auto weigh = [&]() __attribute__((always_inline)) {
      sum = 0.0f;
#pragma unroll
      for (int e = 0; e < 32; e += 4) {
        float p[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
          p[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[e / 16][e % 16 + i], to_log2, -m_run));
        sum += (p[0] + p[1]) + (p[2] + p[3]);
        const int k = 2 * (e / 16) + e / 4 % 2, at = 2 * (e % 16 / 8);
        pw[k][at] = to_f16(p[0], p[1]);
        pw[k][at + 1] = to_f16(p[2], p[3]);
      }
    };
    weigh();
    // A row that has met no key, or whose weights would leave fp16, takes its
    // reference from the tile's maximum first.
    if (__any(sum > 32768.0f)) {
      float top = kNegInf;
#pragma unroll
      for (int hf = 0; hf < 2; ++hf)
#pragma unroll
        for (int e = 0; e < 16; ++e) top = fmaxf(top, sc[hf][e]);
      top = wave_max_xor32(top) * to_log2 - kBias;
      const float m_new = fmaxf(m_run, top);
      const float alpha = __builtin_amdgcn_exp2f(m_run - m_new);
      m_run = m_new;
      l_run *= alpha;
#pragma unroll
      for (int db = 0; db < DB; ++db) oacc[db] *= alpha;
      weigh();
    }
    l_run += sum;
    f16x8 ring[kAhead];
    auto read = [&](int i) __attribute__((always_inline)) {
      const int k = i / DB;
      if (k < 4) ring[i % kAhead] = v_s[st][k / 2][2 * (k % 2) + g][32 * (i % DB) + ln];
    };
#pragma unroll
    for (int i = 0; i < kAhead; ++i) read(i);
#pragma unroll
    for (int i = 0; i < 4 * DB; ++i) {
      __builtin_amdgcn_sched_barrier(0);
      oacc[i % DB] = __builtin_amdgcn_mfma_f32_32x32x16_f16(
          ring[i % kAhead], __builtin_bit_cast(f16x8, pw[i / DB]), oacc[i % DB], 0, 0, 0);
      read(i + kAhead);
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  // O follows V's power.
  auto follow = [&](int v_next) __attribute__((always_inline)) {
    if (v_next == v_exp) return;
    const float f = __builtin_amdgcn_ldexpf(1.0f, v_exp - v_next);
#pragma unroll
    for (int db = 0; db < DB; ++db) oacc[db] *= f;
    v_exp = v_next;
  };

  if constexpr (!CAREFUL) {
    if (tid == 0) shared.redo = 0;
    if (wave == 1) shared.low[lane] = __float_as_uint(kHuge);
    if (ntiles > 0) {
      Raw raw;
      Rebuilt re;
      int v_next = v_exp;
      fetch(raw, 0);
#pragma unroll
      for (int i = 0; i < kPrepare; ++i) prepare(raw, re, i, 0, 0, v_next, 0);
#pragma unroll
      for (int i = 0; i < kPieces; ++i) piece(raw, re, i, 0);
      uint32_t km = re.km;
      uint32_t blocks = raw.held;
      if (ntiles > 1) fetch(raw, 1);
      auto turn = [&](int t, int st) __attribute__((always_inline)) {
        lds_barrier();
        follow(v_next);
        const uint32_t blocks1 = raw.held;
        // The next tile is prepared and rebuilt: K's pieces in the first half, V's in the
        // second.  The last tile does so with what it was itself, into a stage that
        // nothing reads.
        work(t, st, km, blocks, [&](int i) __attribute__((always_inline)) {
          constexpr int every = 2 * DS / kPieces;
          static_assert(every * kPieces == 2 * DS && kPrepare <= DS, "fits the score products");
          if (i < kPrepare) prepare(raw, re, i, t + 1, st ^ 1, v_next, 0);
          if (i % every == every - 1) piece(raw, re, i / every, st ^ 1);
          if (i == 2 * DS - 1 && t + 2 < ntiles) fetch(raw, t + 2);
        });
        km = re.km;
        blocks = blocks1;
      };
      int t = 0;
      for (; t + 1 < ntiles; t += 2) {
        turn(t, 0);
        turn(t + 1, 1);
      }
      if (t < ntiles) turn(t, 0);
    }
    float fin = l_run * 0.0f;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int e = 0; e < 16; ++e) fin = __builtin_fmaf(oacc[db][e], 0.0f, fin);
    __syncthreads();
    if (__any(have && fin != 0.0f) && lane == 0) shared.redo = 1;
    __syncthreads();
    bands.top = v_exp + 15;
    bands.low = min(bands.top, exponent_of(__uint_as_float(~wave_max(~shared.low[lane]))));
    if (__builtin_amdgcn_readfirstlane(shared.redo) || bands.low < bands.top - kBand) return false;
  } else {
#pragma unroll 1
    for (int band = bands.low; band <= bands.top; band += kBand + 1) {
      const float l_band = l_run;
#pragma unroll 1
      for (int t = 0; t < ntiles; ++t) {
        Raw raw;
        Rebuilt re;
        int v_next = v_exp;
        fetch(raw, t);
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kPrepare; ++i) prepare(raw, re, i, t, 0, v_next, band);
#pragma unroll
        for (int i = 0; i < kPieces; ++i) piece(raw, re, i, 0);
        __syncthreads();
        follow(v_next);
        work(t, 0, re.km, raw.held, [](int) {});
#pragma unroll
        for (int gi = 0; gi < G; ++gi) {
          const bool nan = !(low_of(raw.vm[gi]) == low_of(raw.vm[gi]));   // 0 where hidden
          for (uint64_t left = __ballot(nan); left; left &= left - 1) {
            const int i = __builtin_ctzll(left);
            if (!sees(first_token(t0 + 2 * t + (i >> 5)) + (i & 31))) continue;
#pragma unroll
            for (int db = 2 * gi; db < 2 * gi + 2; ++db)
#pragma unroll
              for (int e = 0; e < 16; ++e) oacc[db][e] = __builtin_nanf("");
          }
        }
      }
      // The weights' sums are whole after the first (and the references do not move).
      if (band > bands.low) l_run = l_band;
    }
  }

  l_run += __shfl_xor(l_run, 32);
  if (!have) return true;
  if (share.count > 1) {
    const float back = __builtin_amdgcn_ldexpf(1.0f, v_exp);
    const int64_t at = static_cast<int64_t>(blockIdx.x) * kRows + 32 * wave + ln;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int vq = 0; vq < 4; ++vq) {
        f32x4 y;
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = oacc[db][4 * vq + e] * back;
        *reinterpret_cast<f32x4*>(a.part + at * D + 32 * db + 8 * vq + 4 * g) = y;
      }
    if (g == 0) {
      float* ml = a.part + static_cast<int64_t>(a.items) * kRows * D + at * 2;
      ml[0] = m_run;
      ml[1] = l_run;
    }
    return true;
  }
  // No key: 0; NaN stays.  2^60: O of a row that saw none of V's largest stays normal.
  const float inv = (l_run > 0.0f ? 1.0f / l_run : l_run) * 0x1p60f;
  uint16_t* orow = a.o + b * a.o_sB + hq * a.o_sH + tok * a.o_sN;
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int vq = 0; vq < 4; ++vq) {
      f32x4 y;
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = __builtin_amdgcn_ldexpf(oacc[db][4 * vq + e] * inv, v_exp - 60);
      *reinterpret_cast<bf16x4*>(orow + 32 * db + 8 * vq + 4 * g) = __builtin_convertvector(y, bf16x4);
    }
  if (a.lse && g == 0)
    a.lse[(b * a.H * a.group + hq) * a.n + tok] =
        l_run == 0.0f ? kNegInf : (m_run + __builtin_log2f(l_run)) * kLn2;
  return true;
}

// A group of V that stands for NaN reaches rows that do not see its token (0 * NaN in
// the product), and one above 2^kBand times another costs that one bits in fp16.  So a
// workgroup with anything not finite, or with V's magnitudes that far apart, walks its
// tiles again: once for each kBand powers of two, the smallest first, with the other
// groups taken out of V; NaN is added to the rows that see it.
template <int D, int BITS, int W>
__global__ __launch_bounds__(64 * W) __attribute__((amdgpu_waves_per_eu(2))) void k_cache_chunk(
    const AttnParams a) {
  __shared__ __align__(16) Shared<D> shared;
  Bands bands;
  if (!walk<D, BITS, W, false>(a, shared, bands)) walk<D, BITS, W, true>(a, shared, bands);
}

}  // namespace

hipError_t launch_cache_chunk(const AttnParams& a, int32_t D, int32_t bits, int32_t waves,
                              int64_t items, hipStream_t stream) {
  auto run = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(items)),
                       dim3(static_cast<unsigned>(64 * waves)), 0, stream, a);
  };
  if (waves == 8) {
    if (D == 128) bits == 4 ? run(k_cache_chunk<128, 4, 8>) : run(k_cache_chunk<128, 8, 8>);
    else bits == 4 ? run(k_cache_chunk<64, 4, 8>) : run(k_cache_chunk<64, 8, 8>);
  } else {
    if (D == 128) bits == 4 ? run(k_cache_chunk<128, 4, 4>) : run(k_cache_chunk<128, 8, 4>);
    else bits == 4 ? run(k_cache_chunk<64, 4, 4>) : run(k_cache_chunk<64, 8, 4>);
  }
  return hipGetLastError();
}

}  // namespace vecattn
