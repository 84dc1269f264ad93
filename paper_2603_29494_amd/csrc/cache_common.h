// Layout of the quantised key/value cache, shared by the kernels that write it,
// read it back (cache.hip) and attend to it (cache_attn.hip).
//
// A page holds `page` tokens of every head; a head's part of it is page / 32
// blocks of 32 tokens, and a block is
//   K codes | K groups | V codes | V groups.
// Groups: one dword per token and 64 values (token-major), the smallest value m
// in its low half and the step s in its high half, both bf16; a code u stands
// for m + s u.  Codes lie as the matrix instructions take them, so that the
// attention moves them from memory to registers without a shuffle: as chunks of
// 64 lanes x 16 bytes, lane l of a wave holding dwords 4c .. 4c + 3 of its run in
// chunk c.  With kDw dwords per 8 codes and lane l = 16 g + n:
//   K: dword (t * D/32 + st) * kDw + x holds codes of token 16 t + n (t = 0, 1),
//      head-dim values 32 st + 8 g + 0..7 (A operand: rows tokens, K-slots
//      head-dim values);
//   V: dword db * kDw + x holds codes of head-dim value 16 db + n, tokens
//      4 g + 0..3 and 16 + 4 g + 0..3 (A operand: rows head-dim values, K-slots
//      tokens, in the order in which the scores' C layout leaves the weights).
// Eight codes of 4 bits: slot 2 i in nibble i, slot 2 i + 1 in nibble i + 4, so that
// one shift and one mask give the pair (2 i, 2 i + 1).  Of 8 bits: slots 0..3 in the
// first dword's bytes, 4..7 in the second's.
#pragma once

#include "device_common.h"
#include "launch.h"

namespace vecattn {

constexpr int kCacheBlock = 32;   // tokens per block
constexpr int kCacheGroup = 64;   // head-dim values that share a step and a smallest value

template <int D, int BITS>
struct CacheLayout {
  static constexpr int kG = D / kCacheGroup;             // groups per token
  static constexpr int kDw = BITS / 4;                   // dwords per 8 codes
  static constexpr int kCodes = D * kCacheBlock * BITS / 8;   // bytes of a block's K or V codes
  static constexpr int kParams = kCacheBlock * kG * 4;
  static constexpr int kHalf = kCodes + kParams;
  static constexpr int kBytes = 2 * kHalf;               // bytes of a block
  static constexpr int kRun = kCodes / 256;              // dwords of codes a lane holds
};

// Byte of dword w of lane l's run.
__host__ __device__ __forceinline__ constexpr int code_byte(int w, int l) {
  return ((w >> 2) * 64 + l) * 16 + (w & 3) * 4;
}

// Nibble of slot e (0..7).
__host__ __device__ __forceinline__ constexpr int nibble_of(int e) { return (e >> 1) + 4 * (e & 1); }

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint32_t to_f16(float x, float y) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{x, y}, f16x2));
}

// The values in a pair of bf16, such as a group's m (low) and s (high).
__device__ __forceinline__ float low_of(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float high_of(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// Eight codes, in slot order, in the low bits of 16 each.
template <int BITS>
__device__ __forceinline__ u32x4 codes_16(const uint32_t* w) {
  if constexpr (BITS == 4) {
    const uint32_t x = w[0];
    return u32x4{x & 0x000F000Fu, (x >> 4) & 0x000F000Fu, (x >> 8) & 0x000F000Fu,
                 (x >> 12) & 0x000F000Fu};
  } else {
    return u32x4{__builtin_amdgcn_perm(0u, w[0], 0x0C010C00u), __builtin_amdgcn_perm(0u, w[0], 0x0C030C02u),
                 __builtin_amdgcn_perm(0u, w[1], 0x0C010C00u), __builtin_amdgcn_perm(0u, w[1], 0x0C030C02u)};
  }
}

// The same as fp16 u 2^-kCodeExp: subnormal numbers, whose bits are the code.  Codes of
// 4 bits are moved up by 6: the matrix instructions line subnormal operands up as if
// they were 2^-14, and their sums lose what lies that far below (the log-sum-exp of
// 3000 tokens: off by 2.0e-6 at 2^-24, 4e-7 with 8 bits).
template <int BITS>
constexpr int kCodeExp = BITS == 4 ? 18 : 24;
template <int BITS>
__device__ __forceinline__ u32x4 codes_f16(const uint32_t* w) {
  if constexpr (BITS == 4) {
    const uint32_t x = w[0];
    return u32x4{(x << 6) & 0x03C003C0u, (x << 2) & 0x03C003C0u, (x >> 2) & 0x03C003C0u,
                 (x >> 6) & 0x03C003C0u};
  } else {
    return codes_16<8>(w);
  }
}

}  // namespace vecattn
