// The quantised key/value cache: K and V rows into it (4 or 8 bits a value) and
// back to bf16.
//
// A group of 64 head-dim values of one token and head has the smallest value
// m = min x (bf16 as it came), the step s = bf16((max x - min x) / M), M = 2^bits
// - 1, and codes u = min(M, rint((x - m) / s)), the range, both quotients and the
// difference in fp32; it stands for m + s u.  Steps below 2^-100 are held as 0
// (and u = 0); a group with a NaN or an infinity, or whose range is past fp32,
// holds NaN.
//
// A workgroup takes one block of 32 tokens of one head, so that no two write the
// same bytes (V's codes of eight tokens share a dword).  Both kernels are bound by
// memory for long prompts: 32768 tokens, 4 heads of 128, 4 bits (86 MB) are written in
// 19.5 us (4.4 TB/s) and read back in 15 (5.7, the codes still in cache), 131072 tokens
// (344 MB) in 79 us (4.4 TB/s).  A call for single tokens takes 5 us, most of it the
// chain of loads length, table, store.
#include "cache_common.h"

namespace vecattn {
namespace {

// Where sequence b's tokens are, shared by both directions.
struct PageMap {
  uint8_t* data;
  const int32_t* table;
  int64_t cols;
  int64_t pages;
  int32_t H;
  int32_t page_shift;  // log2 of the tokens per page
};

// Base of the block of tokens [32 jb, 32 jb + 32) of head h, or NULL where no
// page is held for it.
template <int BYTES>
__device__ __forceinline__ uint8_t* block_ptr(const PageMap& m, int64_t b, int h, int64_t jb) {
  const int sh = m.page_shift - 5;  // log2 of the blocks per page
  const int64_t col = jb >> sh;
  if (col >= m.cols) return nullptr;
  const int64_t page = m.table[b * m.cols + col];
  if (page < 0 || page >= m.pages) return nullptr;
  return m.data + (((page * m.H + h) << sh) + (jb & ((1 << sh) - 1))) * BYTES;
}

typedef short i16x2 __attribute__((ext_vector_type(2)));

// bf16 bits as integers of the same order, and back, two at a time.
__device__ __forceinline__ i16x2 ordered(uint32_t bits) {
  const i16x2 b = __builtin_bit_cast(i16x2, bits);
  return b ^ ((b >> 15) & short(0x7FFF));
}

// Eight codes from two dwords of bytes into the nibbles of their slots.
__device__ __forceinline__ uint32_t nibbles(uint32_t lo, uint32_t hi) {
  // Slots 0, 2, 4, 6 from nibble 0 on, slots 1, 3, 5, 7 from nibble 4 on.
  const uint32_t even = __builtin_amdgcn_perm(hi, lo, 0x06040200u);
  const uint32_t odd = __builtin_amdgcn_perm(hi, lo, 0x07050301u);
  const uint32_t e = even | even >> 4, o = odd | odd >> 4;   // pairs in bytes 0 and 2
  return __builtin_amdgcn_perm(o, e, 0x06040200u);
}

// Half a group, 32 values of a token (the other half is on the lane beside): codes
// (0..M) as bytes, four to a dword, and, on both lanes, the group's (m, s) dword.
template <int BITS>
__device__ __forceinline__ uint32_t quantise32(const u32x4 (&w)[4], uint32_t (&bytes)[8]) {
  constexpr float M = BITS == 4 ? 15.0f : 255.0f;
  // Extremes on the bits: bf16 pairs take one instruction, and NaN has its place.
  i16x2 lo2 = ordered(w[0][0]), hi2 = lo2;
#pragma unroll
  for (int e = 1; e < 16; ++e) {
    const i16x2 k = ordered(w[e / 4][e % 4]);
    lo2 = __builtin_elementwise_min(lo2, k);
    hi2 = __builtin_elementwise_max(hi2, k);
  }
  auto beside = [](i16x2 x) __attribute__((always_inline)) {
    const int y = __builtin_bit_cast(int, x);
    return __builtin_bit_cast(i16x2, __builtin_amdgcn_update_dpp(y, y, 0xB1, 0xf, 0xf, false));
  };
  lo2 = __builtin_elementwise_min(lo2, beside(lo2));   // quad_perm [1, 0, 3, 2]
  hi2 = __builtin_elementwise_max(hi2, beside(hi2));
  const short lo_key = min(lo2[0], lo2[1]), hi_key = max(hi2[0], hi2[1]);
  const uint32_t both = __builtin_bit_cast(
      uint32_t, ordered(__builtin_bit_cast(uint32_t, i16x2{lo_key, hi_key})));
  const float lo = __uint_as_float(both << 16), hi = __uint_as_float(both & 0xFFFF0000u);
  const float range = hi - lo;
  // Infinities (keys 0x7F80 and its mirror) and NaN lie outside the finite keys.
  if (hi_key >= 0x7F80 || lo_key < -0x7F80 || !(range < INFINITY)) {
#pragma unroll
    for (int e = 0; e < 8; ++e) bytes[e] = 0;
    return 0x7FC07FC0u;
  }
  const __bf16 sb = static_cast<__bf16>(range / M);
  float s = static_cast<float>(sb);
  uint32_t sbits = __builtin_bit_cast(uint16_t, sb);
  if (s < 0x1p-100f) {
    s = 0.0f;
    sbits = 0;
  }
  // The nearest float to (x - m) / s from the nearest to 1 / s: one step with the
  // exact remainder leaves the product off by 2^-46 of it before it is rounded, and a
  // quotient by s, eight bits, is 2^-33 from the midpoint of two floats at least (none
  // is one).  Adding 2^23 rounds it to an integer in the low bits, ties to even.
  // s = 0: r = 0, u = 0.
  const float r = s == 0.0f ? 0.0f : 1.0f / s;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    uint32_t u[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t pair = w[i / 2][2 * (i % 2) + e / 2];
      const float d = __uint_as_float(e % 2 ? pair & 0xFFFF0000u : pair << 16) - lo;
      float q = d * r;
      q = __builtin_fmaf(__builtin_fmaf(-q, s, d), r, q);
      q = __uint_as_float(min(__float_as_uint(q), __float_as_uint(M)));   // neither below 0
      u[e] = __float_as_uint(q + 8388608.0f);
    }
    bytes[i] = __builtin_amdgcn_perm(__builtin_amdgcn_perm(u[3], u[2], 0x0C0C0400u),
                                     __builtin_amdgcn_perm(u[1], u[0], 0x0C0C0400u), 0x05040100u);
  }
  return (both & 0xFFFFu) | (sbits << 16);
}

// Dword x of the codes of eight tokens, for four head-dim values: c[e] holds the four
// values' codes of the token in slot e, a byte each.
template <int BITS>
__device__ __forceinline__ void transpose_codes(const uint32_t (&c)[8], int x, uint32_t (&out)[4]) {
  uint32_t p[4];   // byte i of the dwords to come, of four values
  if constexpr (BITS == 4) {   // nibbles 2 i and 2 i + 1
    p[0] = c[0] | c[2] << 4, p[1] = c[4] | c[6] << 4;
    p[2] = c[1] | c[3] << 4, p[3] = c[5] | c[7] << 4;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) p[i] = c[4 * x + i];
  }
  const uint32_t a0 = __builtin_amdgcn_perm(p[1], p[0], 0x05010400u);   // values 0, 1: bytes 0, 1
  const uint32_t a1 = __builtin_amdgcn_perm(p[1], p[0], 0x07030602u);   // values 2, 3
  const uint32_t b0 = __builtin_amdgcn_perm(p[3], p[2], 0x05010400u);
  const uint32_t b1 = __builtin_amdgcn_perm(p[3], p[2], 0x07030602u);
  out[0] = __builtin_amdgcn_perm(b0, a0, 0x05040100u);
  out[1] = __builtin_amdgcn_perm(b0, a0, 0x07060302u);
  out[2] = __builtin_amdgcn_perm(b1, a1, 0x05040100u);
  out[3] = __builtin_amdgcn_perm(b1, a1, 0x07060302u);
}

// Half of a workgroup's threads take K, half V, each half a group of a token.  A whole
// block is put together in LDS and stored 16 bytes a lane; of a part of one only the
// new tokens' codes are stored, V's within the dwords they share with others.
template <int D, int BITS>
__global__ __launch_bounds__(2 * D) void k_cache_write(
    const uint16_t* __restrict__ k, int64_t k_sB, int64_t k_sH, int64_t k_sN,
    const uint16_t* __restrict__ v, int64_t v_sB, int64_t v_sH, int64_t v_sN, int32_t n,
    const int32_t* __restrict__ lens, const int32_t* __restrict__ n_new, PageMap map) {
  using L = CacheLayout<D, BITS>;
  constexpr int PARTS = D / 32;   // threads per row
  const int64_t b = blockIdx.z;
  const int h = blockIdx.y;
  const int len = min(max(lens[b], 0), 1 << 30);
  const int nb = n_new ? min(max(n_new[b], 0), n) : n;
  const int p0 = len - nb;        // position of row 0
  const int jb = (max(p0, 0) >> 5) + blockIdx.x;
  const int j0 = jb * kCacheBlock;
  if (nb == 0 || j0 >= len) return;
  uint8_t* blk = block_ptr<L::kBytes>(map, b, h, jb);
  if (!blk) return;
  // Tokens [from, to) of the block are written.
  const int from = max(p0 - j0, 0), to = min(len - j0, kCacheBlock);
  const bool whole = from == 0 && to == kCacheBlock;
  __shared__ __align__(16) uint8_t image[L::kBytes];               // the block
  __shared__ __align__(16) uint32_t codes[kCacheBlock][D / 4 + 4];   // V's, a byte each

  const bool is_v = threadIdx.x >= D;
  const int t = threadIdx.x % D, key = t / PARTS, part = t % PARTS;
  if (key >= from && key < to) {
    const int64_t row = j0 + key - p0;
    const u32x4* src = reinterpret_cast<const u32x4*>(
        is_v ? v + b * v_sB + h * v_sH + row * v_sN + 32 * part
             : k + b * k_sB + h * k_sH + row * k_sN + 32 * part);
    u32x4 w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = src[i];
    uint32_t bytes[8];
    const uint32_t par = quantise32<BITS>(w, bytes);
    uint8_t* to_blk = whole ? image : blk;
    if (part % 2 == 0)
      reinterpret_cast<uint32_t*>(to_blk + (is_v ? L::kHalf : 0) +
                                  L::kCodes)[key * L::kG + part / 2] = par;
    if (is_v) {
#pragma unroll
      for (int i = 0; i < 2; ++i)
        *reinterpret_cast<u32x4*>(&codes[key][8 * part + 4 * i]) =
            u32x4{bytes[4 * i], bytes[4 * i + 1], bytes[4 * i + 2], bytes[4 * i + 3]};
    } else {
      const int w0 = ((key >> 4) * PARTS + part) * L::kDw;
#pragma unroll
      for (int g = 0; g < 4; ++g)   // eight values each
#pragma unroll
        for (int x = 0; x < L::kDw; ++x)
          *reinterpret_cast<uint32_t*>(to_blk + code_byte(w0 + x, g * 16 + (key & 15))) =
              BITS == 4 ? nibbles(bytes[2 * g], bytes[2 * g + 1]) : bytes[2 * g + x];
    }
  }
  __syncthreads();
  // V's codes: eight tokens of four head-dim values at a time, as bytes transposed.
  for (int it = threadIdx.x; it < D; it += 2 * D) {
    const int d = it % (D / 4) * 4, g = it / (D / 4);
    uint32_t c[8], have = 0;   // slot e: four values' codes; bit e: written
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int token = (e >> 2) * 16 + 4 * g + (e & 3);
      const bool here = token >= from && token < to;
      c[e] = here ? codes[token][d / 4] : 0u;   // not written: undefined
      have |= here ? 1u << e : 0u;
    }
#pragma unroll
    for (int x = 0; x < L::kDw; ++x) {
      uint32_t out[4];
      transpose_codes<BITS>(c, x, out);
      auto byte_of = [&](int i) __attribute__((always_inline)) {
        return L::kHalf + code_byte((d + i) / 16 * L::kDw + x, g * 16 + (d + i) % 16);
      };
      if (whole) {
#pragma unroll
        for (int i = 0; i < 4; ++i) *reinterpret_cast<uint32_t*>(image + byte_of(i)) = out[i];
        continue;
      }
      uint32_t mask = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if constexpr (BITS == 4) mask |= have >> e & 1u ? 0xFu << (4 * nibble_of(e)) : 0u;
        else if (e / 4 == x) mask |= have >> e & 1u ? 0xFFu << (8 * (e & 3)) : 0u;
      }
      if (mask == 0) continue;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint32_t* at = reinterpret_cast<uint32_t*>(blk + byte_of(i));
        *at = (*at & ~mask) | (out[i] & mask);
      }
    }
  }
  if (!whole) return;
  __syncthreads();
  for (int i = threadIdx.x; i < L::kBytes / 16; i += 2 * D)
    *reinterpret_cast<u32x4*>(blk + 16 * i) = *reinterpret_cast<const u32x4*>(image + 16 * i);
}

// m + s u for eight codes, rounded to bf16 once.
__device__ __forceinline__ u32x4 values8(uint32_t par, const int (&u)[8]) {
  const float m = __uint_as_float(par << 16), s = __uint_as_float(par & 0xFFFF0000u);
  u32x4 out;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    const f32x2 y = {__builtin_fmaf(s, static_cast<float>(u[2 * e]), m),
                     __builtin_fmaf(s, static_cast<float>(u[2 * e + 1]), m)};
    out[e] = __builtin_bit_cast(uint32_t, __builtin_convertvector(y, bf16x2));
  }
  return out;
}

template <int BITS>
__device__ __forceinline__ void unpack8(const uint32_t (&dw)[BITS / 4], int (&u)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    if constexpr (BITS == 4) u[e] = (dw[0] >> (4 * nibble_of(e))) & 0xF;
    else u[e] = (dw[e >> 2] >> (8 * (e & 3))) & 0xFF;
  }
}

template <int D, int BITS>
__global__ __launch_bounds__(256) void k_cache_read(
    PageMap map, const int32_t* __restrict__ lens, int64_t start, int64_t n,
    uint16_t* __restrict__ k, int64_t k_sB, int64_t k_sH, int64_t k_sN, uint16_t* __restrict__ v,
    int64_t v_sB, int64_t v_sH, int64_t v_sN, bool clear) {
  using L = CacheLayout<D, BITS>;
  constexpr int CH = D / 8;
  constexpr int RPP = 256 / CH;
  const int64_t b = blockIdx.z;
  const int h = blockIdx.y;
  const int64_t len = min(max(lens[b], 0), 1 << 30);
  const int64_t jb = (start >> 5) + blockIdx.x;
  const int64_t j0 = jb * kCacheBlock;
  const int c = threadIdx.x % CH;
  auto k_row = [&](int64_t r) __attribute__((always_inline)) {
    return reinterpret_cast<u32x4*>(k + b * k_sB + h * k_sH + r * k_sN + 8 * c);
  };
  auto v_row = [&](int64_t r) __attribute__((always_inline)) {
    return reinterpret_cast<u32x4*>(v + b * v_sB + h * v_sH + r * v_sN + 8 * c);
  };
  const uint8_t* blk = j0 < len ? block_ptr<L::kBytes>(map, b, h, jb) : nullptr;
  if (clear) {   // rows of tokens that are not held
#pragma unroll
    for (int pass = 0; pass < kCacheBlock / RPP; ++pass) {
      const int64_t j = j0 + pass * RPP + threadIdx.x / CH, r = j - start;
      if (r < 0 || r >= n || (blk && j < len)) continue;
      *k_row(r) = *v_row(r) = u32x4{0, 0, 0, 0};
    }
  }
  if (!blk) return;
  __shared__ uint8_t codes[kCacheBlock][D];  // V's, token-major
  for (int it = threadIdx.x; it < 4 * D; it += 256) {
    const int d = it % D, g = it / D;
    uint32_t dw[L::kDw];
#pragma unroll
    for (int x = 0; x < L::kDw; ++x)
      dw[x] = *reinterpret_cast<const uint32_t*>(
          blk + L::kHalf + code_byte((d >> 4) * L::kDw + x, g * 16 + (d & 15)));
    int u[8];
    unpack8<BITS>(dw, u);
#pragma unroll
    for (int e = 0; e < 8; ++e) codes[(e >> 2) * 16 + 4 * g + (e & 3)][d] = static_cast<uint8_t>(u[e]);
  }
  __syncthreads();
#pragma unroll
  for (int pass = 0; pass < kCacheBlock / RPP; ++pass) {
    const int key = pass * RPP + threadIdx.x / CH;
    const int64_t j = j0 + key, r = j - start;
    if (r < 0 || r >= n || j >= len) continue;
    int u[8];
    uint32_t dw[L::kDw];
    const int w0 = ((key >> 4) * (D / 32) + (c >> 2)) * L::kDw, l = (c & 3) * 16 + (key & 15);
#pragma unroll
    for (int x = 0; x < L::kDw; ++x)
      dw[x] = *reinterpret_cast<const uint32_t*>(blk + code_byte(w0 + x, l));
    unpack8<BITS>(dw, u);
    const int gi = key * L::kG + c / 8;
    *k_row(r) =
        values8(reinterpret_cast<const uint32_t*>(blk + L::kCodes)[gi], u);
#pragma unroll
    for (int e = 0; e < 8; ++e) u[e] = codes[key][8 * c + e];
    *v_row(r) =
        values8(reinterpret_cast<const uint32_t*>(blk + L::kHalf + L::kCodes)[gi], u);
  }
}

// Chosen tokens of a head into pages of their own: slot i takes the codes and (m, s) of
// token idx[i] as they are.  A workgroup puts two blocks of 32 slots together in LDS and
// stores them whole.  Of K a token's codes lie in four runs; of V, whose dwords eight
// tokens share, its codes are picked out to bytes and put together anew.  The lines that the
// kept tokens touch bound it, at about three quarters of a copy's rate: 2048 of up to 8192
// tokens of 64 x 8 heads of 128 in 4 bits take 118 us, 16384 of 131072 of 4 x 4 heads 60.
struct GatherTo {
  uint8_t* data;
  const int32_t* table;
  int64_t cols, pages;
  int32_t page_shift;
};

template <int D, int BITS>
__global__ __launch_bounds__(256) void k_cache_gather(PageMap map, GatherTo to,
                                                      const int32_t* __restrict__ idx,
                                                      const int32_t* __restrict__ kept,
                                                      int64_t budget,
                                                      const float* __restrict__ mass, int64_t M,
                                                      float* __restrict__ mass_out, int64_t M_out,
                                                      bool clear) {
  using L = CacheLayout<D, BITS>;
  constexpr int RUN = D / 32 * L::kDw;   // dwords of a token's codes of K on a lane
  constexpr int NB = 2, SLOTS = NB * kCacheBlock;
  const int64_t b = blockIdx.z;
  const int h = blockIdx.y;
  const int64_t n = min(max(static_cast<int64_t>(kept[b]), int64_t(0)), budget);
  const int64_t jb = static_cast<int64_t>(blockIdx.x) * NB, j0 = jb * kCacheBlock;
  const int64_t bh = b * map.H + h;
  if (mass_out && clear) {
    const int64_t i = j0 + threadIdx.x;
    if (threadIdx.x < SLOTS && i >= n && i < budget) mass_out[bh * M_out + i] = 0.0f;
    // Entries past the budget, of tokens to come.
    const int64_t step = static_cast<int64_t>(gridDim.x) * 256;
    for (int64_t x = budget + blockIdx.x * int64_t(256) + threadIdx.x; x < M_out; x += step)
      mass_out[bh * M_out + x] = 0.0f;
  }
  if (j0 >= n) return;
  const int count = static_cast<int>(min<int64_t>(n - j0, SLOTS));
  const PageMap dst_map{to.data, to.table, to.cols, to.pages, map.H, to.page_shift};

  __shared__ __align__(16) uint8_t image[NB][L::kBytes];
  __shared__ __align__(16) uint32_t codes[SLOTS][D / 4 + 4];   // V's, a byte each
  __shared__ const uint8_t* s_blk[SLOTS];                      // NULL: no such token
  __shared__ int s_token[SLOTS];                               // within its block
  if (threadIdx.x < SLOTS) {
    const int slot = threadIdx.x;
    const uint8_t* blk = nullptr;
    int64_t j = -1;
    if (slot < count) {
      j = idx[bh * budget + j0 + slot];
      if (j >= 0) blk = block_ptr<L::kBytes>(map, b, h, j >> 5);
      if (mass_out)
        mass_out[bh * M_out + j0 + slot] =
            j >= 0 && j < M ? mass[bh * M + j] : __builtin_nanf("");
    }
    s_blk[slot] = blk;
    s_token[slot] = static_cast<int>(j & 31);
  }
  uint8_t* dst[NB];
#pragma unroll
  for (int x = 0; x < NB; ++x)
    dst[x] = x * kCacheBlock < count ? block_ptr<L::kBytes>(dst_map, b, h, jb + x) : nullptr;
  __syncthreads();
  // All loads first: K's codes, the groups of both, and V, sixteen lanes a token, 16 bytes
  // at a time.
  static_assert(SLOTS * 4 == 256 && SLOTS * 2 * L::kG <= 256, "one item per thread");
  uint32_t k_run[RUN], par = 0x7FC07FC0u;
  const int ks = threadIdx.x & (SLOTS - 1), kg = threadIdx.x / SLOTS;
  {
    const uint8_t* blk = s_blk[ks];
    const int from = s_token[ks], a = (from >> 4) * RUN;
#pragma unroll
    for (int x = 0; x < RUN; ++x)
      k_run[x] = blk ? *reinterpret_cast<const uint32_t*>(blk + code_byte(a + x, kg * 16 + (from & 15)))
                     : 0u;
  }
  const int ps = threadIdx.x / L::kG % SLOTS, gi = threadIdx.x % L::kG;
  const int group_at = (threadIdx.x / (L::kG * SLOTS) ? L::kHalf : 0) + L::kCodes;
  const bool has_par = threadIdx.x < SLOTS * 2 * L::kG;
  if (has_par && s_blk[ps])
    par = reinterpret_cast<const uint32_t*>(s_blk[ps] + group_at)[s_token[ps] * L::kG + gi];
  constexpr int VI = SLOTS * 16 / 256, VC = L::kRun / 4;
  const int ln = threadIdx.x & 15;
  u32x4 v[VI][VC];
#pragma unroll
  for (int i = 0; i < VI; ++i) {
    const int slot = 16 * i + (threadIdx.x >> 4);
    const uint8_t* blk = s_blk[slot];
    const int g = (s_token[slot] >> 2) & 3;   // token = 16 (e / 4) + 4 g + e % 4
#pragma unroll
    for (int c = 0; c < VC; ++c)
      v[i][c] = blk ? *reinterpret_cast<const u32x4*>(blk + L::kHalf + code_byte(4 * c, g * 16 + ln))
                    : u32x4{0, 0, 0, 0};
  }
  {
    const int slot = ks & 31, c = (slot >> 4) * RUN;
#pragma unroll
    for (int x = 0; x < RUN; ++x)
      *reinterpret_cast<uint32_t*>(image[ks >> 5] + code_byte(c + x, kg * 16 + (slot & 15))) = k_run[x];
  }
  if (has_par)
    reinterpret_cast<uint32_t*>(image[ps >> 5] + group_at)[(ps & 31) * L::kG + gi] = par;
  // Of V a dword is of one head-dim value (4 bits) or of half its tokens (8 bits).
  uint8_t* bytes = reinterpret_cast<uint8_t*>(codes);
  constexpr int kRow = 4 * (D / 4 + 4);
#pragma unroll
  for (int i = 0; i < VI; ++i) {
    const int slot = 16 * i + (threadIdx.x >> 4), token = s_token[slot];
    const int e = (token >> 4) * 4 + (token & 3);
#pragma unroll
    for (int c = 0; c < VC; ++c) {
      if constexpr (BITS == 4) {
#pragma unroll
        for (int y = 0; y < 4; ++y)
          bytes[slot * kRow + 16 * (4 * c + y) + ln] =
              static_cast<uint8_t>(v[i][c][y] >> (4 * nibble_of(e)) & 0xFu);
      } else {
#pragma unroll
        for (int y = 0; y < 2; ++y)
          bytes[slot * kRow + 16 * (2 * c + y) + ln] =
              static_cast<uint8_t>((e >> 2 ? v[i][c][2 * y + 1] : v[i][c][2 * y]) >> (8 * (e & 3)));
      }
    }
  }
  __syncthreads();
  for (int it = threadIdx.x; it < NB * D; it += 256) {
    const int x0 = it / D, d = it % (D / 4) * 4, g = it % D / (D / 4);
    uint32_t c[8];
#pragma unroll
    for (int e = 0; e < 8; ++e)
      c[e] = codes[x0 * kCacheBlock + (e >> 2) * 16 + 4 * g + (e & 3)][d / 4];
#pragma unroll
    for (int x = 0; x < L::kDw; ++x) {
      uint32_t out[4];
      transpose_codes<BITS>(c, x, out);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<uint32_t*>(image[x0] + L::kHalf +
                                     code_byte((d + i) / 16 * L::kDw + x, g * 16 + (d + i) % 16)) =
            out[i];
    }
  }
  __syncthreads();
#pragma unroll
  for (int x = 0; x < NB; ++x)
    if (dst[x])
      for (int i = threadIdx.x; i < L::kBytes / 16; i += 256)
        *reinterpret_cast<u32x4*>(dst[x] + 16 * i) =
            *reinterpret_cast<const u32x4*>(image[x] + 16 * i);
}

PageMap page_map(const CacheArgs& c) {
  return PageMap{static_cast<uint8_t*>(c.data), c.table, c.cols, c.pages, c.H,
                 __builtin_ctz(static_cast<unsigned>(c.page))};
}

}  // namespace

hipError_t launch_cache_write(const Tensor4& k, const Tensor4& v, const CacheArgs& c,
                              const int32_t* n_new, hipStream_t stream) {
  // Blocks that n consecutive tokens can touch.
  const int64_t blocks = (k.N + 2 * kCacheBlock - 2) / kCacheBlock;
  const dim3 grid(static_cast<unsigned>(blocks), static_cast<unsigned>(k.H),
                  static_cast<unsigned>(k.B));
  auto run = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, dim3(static_cast<unsigned>(2 * c.D)), 0, stream,
                       static_cast<const uint16_t*>(k.ptr), k.sB, k.sH, k.sN, static_cast<const uint16_t*>(v.ptr), v.sB, v.sH, v.sN,
                       static_cast<int32_t>(k.N), c.lens, n_new, page_map(c));
  };
  if (c.D == 128) c.bits == 4 ? run(k_cache_write<128, 4>) : run(k_cache_write<128, 8>);
  else c.bits == 4 ? run(k_cache_write<64, 4>) : run(k_cache_write<64, 8>);
  return hipGetLastError();
}

hipError_t launch_cache_read(const CacheArgs& c, int64_t start, const Tensor4& k, const Tensor4& v,
                             bool clear, hipStream_t stream) {
  const int64_t blocks = (start + k.N + kCacheBlock - 1) / kCacheBlock - start / kCacheBlock;
  const dim3 grid(static_cast<unsigned>(blocks), static_cast<unsigned>(k.H),
                  static_cast<unsigned>(k.B));
  auto run = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, dim3(256), 0, stream, page_map(c), c.lens, start, k.N,
                       static_cast<uint16_t*>(const_cast<void*>(k.ptr)), k.sB, k.sH, k.sN,
                       static_cast<uint16_t*>(const_cast<void*>(v.ptr)), v.sB, v.sH, v.sN, clear);
  };
  if (c.D == 128) c.bits == 4 ? run(k_cache_read<128, 4>) : run(k_cache_read<128, 8>);
  else c.bits == 4 ? run(k_cache_read<64, 4>) : run(k_cache_read<64, 8>);
  return hipGetLastError();
}

hipError_t launch_cache_gather(const CacheArgs& c, const CacheArgs& to, int64_t B,
                               const int32_t* idx, const int32_t* kept, int64_t budget,
                               const float* mass, int64_t M, float* mass_out, int64_t M_out,
                               bool clear, hipStream_t stream) {
  const dim3 grid(static_cast<unsigned>((budget + 2 * kCacheBlock - 1) / (2 * kCacheBlock)),
                  static_cast<unsigned>(c.H), static_cast<unsigned>(B));
  const GatherTo g{static_cast<uint8_t*>(to.data), to.table, to.cols, to.pages,
                   __builtin_ctz(static_cast<unsigned>(to.page))};
  auto run = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, dim3(256), 0, stream, page_map(c), g, idx, kept, budget, mass, M,
                       mass_out, M_out, clear);
  };
  if (c.D == 128) c.bits == 4 ? run(k_cache_gather<128, 4>) : run(k_cache_gather<128, 8>);
  else c.bits == 4 ? run(k_cache_gather<64, 4>) : run(k_cache_gather<64, 8>);
  return hipGetLastError();
}

}  // namespace vecattn
