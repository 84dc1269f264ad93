// Attention with a sliding window and sinks: query position p sees the keys
// j with p - window < j (and j <= p causal, or j < p + window), and the first
// `sinks` keys (causal: those at or before p).
//
// One workgroup owns 128 query rows of one head (four waves of 32) and walks the
// tiles of 64 keys that one of its rows sees: those of the sinks, then those of
// the window.  A tile's K and V rows go straight from memory to LDS (16 bytes per
// lane) while the tile before is worked on, stored with the swizzle of
// device_common.h.  Each wave computes S^T = K Q^T and O^T += V^T P^T for the
// whole tile on v_mfma_f32_32x32x16_bf16 (lane layout as in sparse_attn.hip) with
// the softmax state in registers.  Only tiles that some row of a wave does not
// see whole are masked.  The weights are rounded to bf16 (half a step, 2^-9) before
// they meet V, as the operands are; their sum is of what was not rounded.
//
// 4 D operations per visible pair of positions bound it, at the rate that the card's
// power allows: 40 heads of 128 over 75600 tokens, two-sided window 3600 and 3600
// sinks, take 13.75 ms (1168 TFLOP/s; a 16384-wide matrix product reaches 1359), and
// 9.3 ms on zeros; half the LDS reads save 4%.  28 heads over 4, 32768 tokens, causal,
// window 4096: 1.65 ms (1099 TFLOP/s).  Tiles of 64 keys in two stages leave LDS for
// two workgroups per CU; a wave's own skipping of tiles that it does not see cost 92
// spilled registers (36 ms).
#include <algorithm>
#include <type_traits>

#include "device_common.h"
#include "launch.h"

namespace vecattn {
namespace {

constexpr int kTile = 64;
constexpr int kRows = kWindowRows;
constexpr float kUnseen = -3.4028234663852886e38f;

struct WindowParams {
  const uint16_t *q, *k, *v;
  int64_t q_sB, q_sH, q_sN, k_sB, k_sH, k_sN, v_sB, v_sH, v_sN;
  uint16_t* o;
  int64_t o_sB, o_sH, o_sN;
  float* lse;
  const int32_t* lens;
  int32_t Hq, Hkv, group, Nq, Nk, window, sinks, causal, row_tiles, run;
  int64_t items;
  float scale_log2;
};

template <int D>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2))) void k_window_attn(
    const WindowParams a) {
  constexpr int CH = D / 8;
  constexpr int U = kTile * CH / 256;   // direct-load instructions per wave and matrix
  constexpr int DS = D / 16, DB = D / 32, RB = 2 * D;
  __shared__ __align__(16) uint16_t k_s0[kTile * D];
  __shared__ __align__(16) uint16_t k_s1[kTile * D];
  __shared__ __align__(16) uint16_t v_s0[kTile * D];
  __shared__ __align__(16) uint16_t v_s1[kTile * D];
  auto kbuf = [&](int st) __attribute__((always_inline)) { return st ? k_s1 : k_s0; };
  auto vbuf = [&](int st) __attribute__((always_inline)) { return st ? v_s1 : v_s0; };

  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 5, ln = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // Work item: batch and key/value head, then row tile, then the query heads that
  // share them.  The hardware deals workgroup x to XCD x % 8; an XCD takes `run`
  // consecutive items at a time, whose windows overlap, so that it finds most of
  // their keys in its own L2.
  const int64_t slot = blockIdx.x >> 3;
  int64_t item = (slot / a.run * 8 + (blockIdx.x & 7)) * a.run + slot % a.run;
  if (item >= a.items) return;
  const int hg = static_cast<int>(item % a.group);
  item /= a.group;
  const int rt = static_cast<int>(item % a.row_tiles);
  item /= a.row_tiles;
  const int hk = static_cast<int>(item % a.Hkv), h = hk * a.group + hg;
  const int64_t b = item / a.Hkv;
  const int off = a.Nk - a.Nq;                       // position of row 0
  const int len = a.lens ? min(max(a.lens[b], 0), a.Nk) : a.Nk;
  const int rows_end = min(a.Nq, len - off);         // rows past it are padding
  const int row0 = rt * kRows;
  if (row0 >= rows_end) return;
  const int p_lo = row0 + off, p_hi = min(row0 + kRows, rows_end) - 1 + off;
  // Keys of the window, [near, far] (with two-sided sinks past it), and the tiles:
  // ns of the sinks before it, then from nt0.
  const int near = max(0, p_lo - a.window + 1);
  const int far = a.causal ? p_hi : min(len, max(p_hi + a.window, a.sinks)) - 1;
  const int nt0 = near / kTile;
  const int ns = min(nt0, (min(a.sinks, near) + kTile - 1) / kTile);
  const int ntiles = ns + far / kTile + 1 - nt0;
  auto tile_key = [&](int t) __attribute__((always_inline)) {
    return (t < ns ? t : nt0 + (t - ns)) * kTile;
  };

  const uint16_t* kh = a.k + b * a.k_sB + hk * a.k_sH;
  const uint16_t* vh = a.v + b * a.v_sB + hk * a.v_sH;
  const uint32_t k_rowb = static_cast<uint32_t>(a.k_sN) * 2u;
  const uint32_t v_rowb = static_cast<uint32_t>(a.v_sN) * 2u;
  // Direct-load instruction u of this wave for the tile at key j0, through a buffer
  // resource of the tile's own (rows at or past len read 0).
  auto gather = [&](const uint16_t* base, int64_t sN, uint32_t rowb, int j0, int u, uint16_t* dst)
                    __attribute__((always_inline)) {
    const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<uint16_t*>(base + j0 * sN), 0, (min(kTile, len - j0) - 1) * rowb + RB,
        0x00020000);
    const int i = (wave * U + u) * 64 + lane, r = i / CH;
    gather16_to_lds(rs, r * rowb + 16u * ((i % CH) ^ swz<D>(r)), dst + (wave * U + u) * 64 * 8);
  };
  auto gather_k = [&](int j0, int u, int st) __attribute__((always_inline)) {
    gather(kh, a.k_sN, k_rowb, j0, u, kbuf(st));
  };
  auto gather_v = [&](int j0, int u, int st) __attribute__((always_inline)) {
    gather(vh, a.v_sN, v_rowb, j0, u, vbuf(st));
  };

  const int my_row = row0 + 32 * wave + ln;
  const int my_pos = my_row + off;
  const bool have = my_row < rows_end;
  bf16x8 qf[DS];
  {
    const u32x4* qr = reinterpret_cast<const u32x4*>(
        a.q + b * a.q_sB + h * a.q_sH + static_cast<int64_t>(have ? my_row : row0) * a.q_sN);
#pragma unroll
    for (int s = 0; s < DS; ++s) {
      const u32x4 t = have ? qr[2 * s + g] : u32x4{0, 0, 0, 0};
      qf[s] = __builtin_bit_cast(bf16x8, t);
    }
  }
  // Positions of the wave's rows that exist (w_hi < w_lo: none).
  const int w_lo = row0 + 32 * wave + off, w_hi = min(w_lo + 31, rows_end - 1 + off);

  f32x16 oacc[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) oacc[db] = f32x16{};
  float m_run = kUnseen, l_run = 0.0f;

  const int j16 = lane & 15, tq = j16 >> 2, tp = j16 & 3, vhalf = (lane >> 4) & 1;
  uint32_t koff[DS], voff[DB][2];
#pragma unroll
  for (int s2 = 0; s2 < DS; ++s2) koff[s2] = ln * RB + 16 * ((2 * s2 + g) ^ swz<D>(ln));
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int hi = 0; hi < 2; ++hi) {
      const int d = 32 * db + 16 * vhalf + 4 * tp;
      const int k0 = 4 * g + tq + 8 * hi;
      voff[db][hi] = k0 * RB + 16 * ((d >> 3) ^ swz<D>(k0)) + 8 * ((d >> 2) & 1);
    }

  // This lane's row sees the keys in (v_lo, v_hi] and those up to v_first.
  const int v_lo = my_pos - a.window;
  const int v_hi = min(len - 1, a.causal ? my_pos : my_pos + a.window - 1);
  const int v_first = min(a.causal ? min(a.sinks - 1, my_pos) : a.sinks - 1, len - 1);
  // Every row of the wave sees keys j0 .. j0 + 63.
  auto whole = [&](int j0) __attribute__((always_inline)) {
    return j0 + kTile <= len && (!a.causal || j0 + kTile - 1 <= w_lo) &&
           (j0 + kTile <= a.sinks ||
            (j0 > w_hi - a.window && (a.causal || j0 + kTile - 1 < w_lo + a.window)));
  };
  // S^T of keys 32 hf .. + 31 of the tile in stage st.
  auto score = [&](f32x16& s, int st, int hf) __attribute__((always_inline)) {
    const char* kb = reinterpret_cast<const char*>(kbuf(st)) + hf * 32 * RB;
    s = f32x16{};
#pragma unroll
    for (int s2 = 0; s2 < DS; ++s2) {
      const u32x4 kf = *reinterpret_cast<const u32x4*>(kb + koff[s2]);
      s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kf), qf[s2], s, 0, 0,
                                                  0);
    }
  };
  auto mask = [&](f32x16 (&s)[2], int j0) __attribute__((always_inline)) {
    const int lo = v_lo - j0 - 4 * g, hi = v_hi - j0 - 4 * g, first = v_first - j0 - 4 * g;
#pragma unroll
    for (int hf = 0; hf < 2; ++hf)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int j = 32 * hf + 8 * (e / 4) + e % 4;
        s[hf][e] = (j > lo && j <= hi) || j <= first ? s[hf][e] : kNegInf;
      }
  };
  // A row's reference moves when its maximum has grown by more than 8 (log2 units).
  auto refer = [&](const f32x16 (&s)[2], bool mine) __attribute__((always_inline)) {
    float top = kNegInf;
#pragma unroll
    for (int hf = 0; hf < 2; ++hf)
#pragma unroll
      for (int e = 0; e < 16; ++e) top = fmaxf(top, s[hf][e]);
    top = wave_max_xor32(top) * a.scale_log2;
    const bool up = mine && top > m_run + 8.0f;
    if (__any(up)) {
      const float m_new = up ? top : m_run;
      const float alpha = __builtin_amdgcn_exp2f(m_run - m_new);
      m_run = m_new;
      l_run *= alpha;
#pragma unroll
      for (int db = 0; db < DB; ++db) oacc[db] *= alpha;
    }
  };
  auto vread = [&](int ks, int db, int st) __attribute__((always_inline)) {
    const char* vb = reinterpret_cast<const char*>(vbuf(st));
    const char* a0 = vb + voff[db][0] + 16 * ks * RB;  // the swizzle repeats every 16 rows
    const char* a1 = vb + voff[db][1] + 16 * ks * RB;
    const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS_PTR(i16x4, a0));
    const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS_PTR(i16x4, a1));
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  };
  // Weights above 256 went into O and l as they are; the row's reference moves up by
  // a power of two for the tiles to come.  A weight, or its product with V, past fp32
  // range leaves O or l infinite, which the end of the walk sees.
  auto move = [&](float tsum) __attribute__((always_inline)) {
    if (__any(tsum > 256.0f)) {
      const float top = wave_max_xor32(tsum);
      const int up = top > 256.0f ? __builtin_amdgcn_frexp_expf(top) : 0;
      const float alpha = __builtin_amdgcn_ldexpf(1.0f, -up);
      l_run *= alpha;
#pragma unroll
      for (int db = 0; db < DB; ++db) oacc[db] *= alpha;
      m_run += static_cast<float>(up);
    }
  };
  // The weights of keys 16 ks .. + 15 of a tile, times alpha, and their sum.
  auto weigh = [&](const f32x16 (&s)[2], int ks, float alpha, float& sum)
                   __attribute__((always_inline)) {
    f32x8 p;
#pragma unroll
    for (int e = 0; e < 8; ++e)
      p[e] = __builtin_amdgcn_exp2f(
                 __builtin_fmaf(s[ks >> 1][8 * (ks & 1) + e], a.scale_log2, -m_run)) *
             alpha;
    sum = ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
    return __builtin_convertvector(p, bf16x8);
  };
  // One step: the scores of tile t + 1 (K of stage st ^ 1) while tile t (scores cur,
  // V of stage st) is weighed and multiplied, so that matrix instructions run beside
  // exponentials.  The order is fixed: between two matrix instructions one operand
  // read kAhead instructions ahead of its use, one weight (two where the product
  // waits for them) and, in the first half, one of the gathers.
  auto step = [&](f32x16 (&cur)[2], f32x16 (&nxt)[2], int st, auto more_tag, auto&& fetch)
                  __attribute__((always_inline)) {
    constexpr bool MORE = decltype(more_tag)::value;
    constexpr int NS = MORE ? 2 * DS : 0, NP = 4 * DB;   // matrix instructions of either kind
    constexpr int kAhead = 4;
    i16x8 ring[kAhead];
    f32x8 p[4];
    float sum[4];
    bf16x8 pb[4];
    auto read = [&](int i) __attribute__((always_inline)) {   // operand of instruction i
      if (i < NS) {
        const char* kb = reinterpret_cast<const char*>(kbuf(st ^ 1)) + i / DS * 32 * RB;
        ring[i % kAhead] = *reinterpret_cast<const i16x8*>(kb + koff[i % DS]);
      } else if (i < NS + NP) {
        ring[i % kAhead] = vread((i - NS) / DB, (i - NS) % DB, st);
      }
    };
    auto weight = [&](int e) __attribute__((always_inline)) {   // of element e of 32
      if (e >= 32) return;
      const int ks = e / 8;
      p[ks][e % 8] =
          __builtin_amdgcn_exp2f(__builtin_fmaf(cur[e / 16][e % 16], a.scale_log2, -m_run));
      if (e % 8 == 7) {
        sum[ks] = ((p[ks][0] + p[ks][1]) + (p[ks][2] + p[ks][3])) +
                  ((p[ks][4] + p[ks][5]) + (p[ks][6] + p[ks][7]));
        pb[ks] = __builtin_convertvector(p[ks], bf16x8);
      }
    };
#pragma unroll
    for (int i = 0; i < kAhead; ++i) read(i);
    if constexpr (!MORE) {
#pragma unroll
      for (int e = 0; e < 16; ++e) weight(e);
    }
    if constexpr (MORE) nxt[0] = nxt[1] = f32x16{};
#pragma unroll
    for (int i = 0; i < NS; ++i) {
      __builtin_amdgcn_sched_barrier(0);
      nxt[i / DS] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
          __builtin_bit_cast(bf16x8, ring[i % kAhead]), qf[i % DS], nxt[i / DS], 0, 0, 0);
      read(i + kAhead);
      fetch(i);
#pragma unroll
      for (int x = 0; x < 16 / NS; ++x) weight(16 / NS * i + x);
    }
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      __builtin_amdgcn_sched_barrier(0);
      oacc[i % DB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
          __builtin_bit_cast(bf16x8, ring[(NS + i) % kAhead]), pb[i / DB], oacc[i % DB], 0, 0, 0);
      read(NS + i + kAhead);
#pragma unroll
      for (int x = 0; x < 32 / NP; ++x) weight(16 + 32 / NP * i + x);
    }
    __builtin_amdgcn_sched_barrier(0);
    const float tsum = (sum[0] + sum[1]) + (sum[2] + sum[3]);
    l_run += tsum;
    move(tsum);
  };
  int settled = 0;   // every row of the wave has a reference
  auto ready = [&](f32x16 (&s)[2], int j0) __attribute__((always_inline)) {
    if (!whole(j0)) mask(s, j0);
    if (!settled) {
      refer(s, true);
      settled = __builtin_amdgcn_readfirstlane(!__any(m_run == kUnseen));
    }
  };

  __shared__ int s_redo;
  if (tid == 0) s_redo = 0;
  // K runs one tile ahead of V.
  f32x16 sa[2], sb[2];
#pragma unroll
  for (int u = 0; u < U; ++u) gather_k(tile_key(0), u, 0);
#pragma unroll
  for (int u = 0; u < U; ++u) gather_v(tile_key(0), u, 0);
  wait_all();
  __builtin_amdgcn_s_barrier();
  if (ntiles > 1) {
#pragma unroll
    for (int u = 0; u < U; ++u) gather_k(tile_key(1), u, 1);
  }
  score(sa[0], 0, 0);
  score(sa[1], 0, 1);
  ready(sa, tile_key(0));
  int t = 0;
  auto turn = [&](f32x16 (&cur)[2], f32x16 (&nxt)[2], int st) __attribute__((always_inline)) {
    wait_all();
    __builtin_amdgcn_s_barrier();
    // Past the last tile K is fetched once more (into a buffer nothing reads).
    const int jk = tile_key(min(t + 2, ntiles - 1)), jv = tile_key(t + 1);
    step(cur, nxt, st, std::true_type{}, [&](int i) __attribute__((always_inline)) {
      if (i < U) gather_v(jv, i, st ^ 1);
      else if (i < 2 * U) gather_k(jk, i - U, st);
    });
    ready(nxt, tile_key(t + 1));
    ++t;
  };
  while (t + 2 < ntiles) {
    turn(sa, sb, 0);
    turn(sb, sa, 1);
  }
  if (t + 1 < ntiles) {
    turn(sa, sb, 0);
    wait_all();
    __builtin_amdgcn_s_barrier();
    step(sb, sa, 1, std::false_type{}, [](int) {});
  } else {
    wait_all();
    __builtin_amdgcn_s_barrier();
    step(sa, sb, 0, std::false_type{}, [](int) {});
  }

  // A NaN or an infinity of a V row reaches rows of its tile that do not see it
  // (0 * NaN in the product), and a weight taken before its row's reference has moved
  // may be past fp32 range, by itself or times V.  So a workgroup with anything not
  // finite walks its tiles again, with such values taken out of the products and added
  // to the rows that see them, and references moved first.
  float fin = l_run * 0.0f;
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int e = 0; e < 16; ++e) fin = __builtin_fmaf(oacc[db][e], 0.0f, fin);
  __syncthreads();
  if (__any(have && fin != 0.0f) && lane == 0) s_redo = 1;
  __syncthreads();
  if (__builtin_amdgcn_readfirstlane(s_redo)) {
    auto not_finite = [](uint16_t x) __attribute__((always_inline)) {
      return (x & 0x7F80u) == 0x7F80u;
    };
    m_run = kUnseen;
    l_run = 0.0f;
    settled = 0;
#pragma unroll
    for (int db = 0; db < DB; ++db) oacc[db] = f32x16{};
    for (t = 0; t < ntiles; ++t) {
      const int j0 = tile_key(t);
      __syncthreads();
#pragma unroll
      for (int u = 0; u < U; ++u) {
        gather_k(j0, u, 0);
        gather_v(j0, u, 0);
      }
      wait_all();
      __syncthreads();
      f32x16 s[2];
      score(s[0], 0, 0);
      score(s[1], 0, 1);
      ready(s, j0);
      // A row whose weights are past fp32 range takes its reference from the tile first.
      // The others' references move as after a first walk's tile, by the same power of
      // two, but before the products, which a large V would take past fp32 range:
      // (O + P V) 2^-up = O 2^-up + (P 2^-up) V to the bit.
      float sum[4], alpha = 1.0f;
      bf16x8 pb[4];
      auto weights = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) pb[ks] = weigh(s, ks, alpha, sum[ks]);
        return (sum[0] + sum[1]) + (sum[2] + sum[3]);
      };
      float tsum = weights();
      const int past = !(tsum < INFINITY);
      const bool over = (past | __shfl_xor(past, 32)) != 0;
      if (__any(over)) {
        refer(s, over);
        tsum = weights();
      }
      float shift = 0.0f;
      if (__any(tsum > 256.0f)) {
        const float top = wave_max_xor32(tsum);
        const int up = top > 256.0f ? __builtin_amdgcn_frexp_expf(top) : 0;
        shift = static_cast<float>(up);
        alpha = __builtin_amdgcn_ldexpf(1.0f, -up);
        tsum = weights();
        l_run *= alpha;
#pragma unroll
        for (int db = 0; db < DB; ++db) oacc[db] *= alpha;
      }
      m_run += shift;
      l_run += tsum;
#pragma unroll
      for (int ks = 0; ks < 4; ++ks) {
#pragma unroll
        for (int db = 0; db < DB; ++db) {
          i16x8 x = vread(ks, db, 0);
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] = not_finite(x[e]) ? short(0) : x[e];
          oacc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, x), pb[ks],
                                                             oacc[db], 0, 0, 0);
        }
      }
#pragma unroll 1
      for (int j = 0; j < kTile; ++j) {
        if (!((j0 + j > v_lo && j0 + j <= v_hi) || j0 + j <= v_first)) continue;
        const char* row = reinterpret_cast<const char*>(v_s0) + j * RB;
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const int d = 32 * db + 8 * (e / 4) + 4 * g + e % 4;
            const uint16_t x = *reinterpret_cast<const uint16_t*>(
                row + 16 * ((d >> 3) ^ swz<D>(j)) + 2 * (d & 7));
            if (not_finite(x)) oacc[db][e] += bf16_bits_to_f32(x);
          }
      }
    }
  }

  l_run += __shfl_xor(l_run, 32);
  if (!have) return;
  const float inv = 1.0f / l_run;   // a row sees its own key at least
  if (a.lse && g == 0)
    a.lse[(b * a.Hq + h) * a.Nq + my_row] =
        (m_run + __builtin_log2f(l_run)) * 0.69314718055994531f;
  uint16_t* orow = a.o + b * a.o_sB + h * a.o_sH + static_cast<int64_t>(my_row) * a.o_sN;
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int vq = 0; vq < 4; ++vq) {
      f32x4 r;
#pragma unroll
      for (int e = 0; e < 4; ++e) r[e] = oacc[db][4 * vq + e] * inv;
      *reinterpret_cast<bf16x4*>(orow + 32 * db + 8 * vq + 4 * g) = __builtin_convertvector(r, bf16x4);
    }
}

}  // namespace

hipError_t launch_window_attn(const WindowArgs& x, hipStream_t stream) {
  WindowParams a;
  a.q = static_cast<const uint16_t*>(x.q.ptr);
  a.k = static_cast<const uint16_t*>(x.k.ptr);
  a.v = static_cast<const uint16_t*>(x.v.ptr);
  a.q_sB = x.q.sB, a.q_sH = x.q.sH, a.q_sN = x.q.sN;
  a.k_sB = x.k.sB, a.k_sH = x.k.sH, a.k_sN = x.k.sN;
  a.v_sB = x.v.sB, a.v_sH = x.v.sH, a.v_sN = x.v.sN;
  a.o = static_cast<uint16_t*>(x.o);
  a.o_sB = x.o_sB, a.o_sH = x.o_sH, a.o_sN = x.o_sN;
  a.lse = x.lse;
  a.lens = x.lens;
  a.Hq = static_cast<int32_t>(x.q.H);
  a.Hkv = static_cast<int32_t>(x.k.H);
  a.group = a.Hq / a.Hkv;
  a.Nq = static_cast<int32_t>(x.q.N);
  a.Nk = static_cast<int32_t>(x.k.N);
  // A window or sinks past the keys is all of them (and keeps the positions'
  // sums and differences in range: N <= 2^30).
  a.window = static_cast<int32_t>(std::min(x.window, x.k.N));
  a.sinks = static_cast<int32_t>(std::min(x.sinks, x.k.N));
  a.causal = x.causal;
  a.row_tiles = static_cast<int32_t>((x.q.N + kRows - 1) / kRows);
  const float scale = x.scale != 0.0f ? x.scale : 1.0f / sqrtf(static_cast<float>(x.q.D));
  a.scale_log2 = std::max(scale * 1.4426950408889634f, 0x1p-126f);   // -inf * 0 is no mask
  a.items = x.q.B * a.Hq * static_cast<int64_t>(a.row_tiles);
  // Runs of the 64 workgroups that an XCD holds at a time (75600 tokens: 14.1 ms, 15.7
  // without; 16 to 128 differ by 2%), shorter ones where that would leave an XCD fewer
  // than four.
  a.run = static_cast<int32_t>(std::min<int64_t>(64, std::max<int64_t>(1, a.items / 32)));
  const int64_t rounds = (a.items + 8 * a.run - 1) / (8 * a.run);
  const dim3 grid(static_cast<unsigned>(rounds * 8 * a.run));
  if (x.q.D == 128) hipLaunchKernelGGL(k_window_attn<128>, grid, dim3(256), 0, stream, a);
  else hipLaunchKernelGGL(k_window_attn<64>, grid, dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace vecattn
