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
// Eight codes of 4 bits: of K slot e in nibble 2 e and slot 4 + e in nibble 2 e + 1
// (e < 4: a mask makes bytes of either four); of V slot 2 i in nibble i, slot 2 i + 1
// in nibble i + 4 (a shift and an and-or make the bf16 pair (2 i, 2 i + 1)).  Of 8
// bits: slots 0..3 in the first dword's bytes, 4..7 in the second's.
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

// Nibble of slot e (0..7) of K's and of V's dwords.
__host__ __device__ __forceinline__ constexpr int k_nibble(int e) { return 2 * (e & 3) + (e >> 2); }
__host__ __device__ __forceinline__ constexpr int v_nibble(int e) { return (e >> 1) + 4 * (e & 1); }

}  // namespace vecattn
