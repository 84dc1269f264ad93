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
      const uint32_t out[4] = {__builtin_amdgcn_perm(b0, a0, 0x05040100u),
                               __builtin_amdgcn_perm(b0, a0, 0x07060302u),
                               __builtin_amdgcn_perm(b1, a1, 0x05040100u),
                               __builtin_amdgcn_perm(b1, a1, 0x07060302u)};
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
    int64_t v_sB, int64_t v_sH, int64_t v_sN) {
  using L = CacheLayout<D, BITS>;
  constexpr int CH = D / 8;
  constexpr int RPP = 256 / CH;
  const int64_t b = blockIdx.z;
  const int h = blockIdx.y;
  const int64_t len = min(max(lens[b], 0), 1 << 30);
  const int64_t jb = (start >> 5) + blockIdx.x;
  const int64_t j0 = jb * kCacheBlock;
  if (j0 >= len) return;
  const uint8_t* blk = block_ptr<L::kBytes>(map, b, h, jb);
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
  const int c = threadIdx.x % CH;
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
    *reinterpret_cast<u32x4*>(k + b * k_sB + h * k_sH + r * k_sN + 8 * c) =
        values8(reinterpret_cast<const uint32_t*>(blk + L::kCodes)[gi], u);
#pragma unroll
    for (int e = 0; e < 8; ++e) u[e] = codes[key][8 * c + e];
    *reinterpret_cast<u32x4*>(v + b * v_sB + h * v_sH + r * v_sN + 8 * c) =
        values8(reinterpret_cast<const uint32_t*>(blk + L::kHalf + L::kCodes)[gi], u);
  }
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
                             hipStream_t stream) {
  const int64_t blocks = (start + k.N + kCacheBlock - 1) / kCacheBlock - start / kCacheBlock;
  const dim3 grid(static_cast<unsigned>(blocks), static_cast<unsigned>(k.H),
                  static_cast<unsigned>(k.B));
  auto run = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, dim3(256), 0, stream, page_map(c), c.lens, start, k.N,
                       static_cast<uint16_t*>(const_cast<void*>(k.ptr)), k.sB, k.sH, k.sN,
                       static_cast<uint16_t*>(const_cast<void*>(v.ptr)), v.sB, v.sH, v.sN);
  };
  if (c.D == 128) c.bits == 4 ? run(k_cache_read<128, 4>) : run(k_cache_read<128, 8>);
  else c.bits == 4 ? run(k_cache_read<64, 4>) : run(k_cache_read<64, 8>);
  return hipGetLastError();
}

}  // namespace vecattn
