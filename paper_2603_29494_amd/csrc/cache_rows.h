// Rows of q against the cache's codes on the 16x16x32 matrix instructions, shared by
// the attention of a few rows (cache_attn.hip) and the weights' sums (cache_mass.hip).
//
// Lane layout (lane l = 16 g + n): A: row n, K-slots 8 g .. 8 g + 7; B: column n, the
// same slots; C: column n, rows 4 g .. 4 g + 3.
#pragma once

#include "cache_common.h"

namespace vecattn {

// Over the four lanes that hold a column (n = lane % 16).
__device__ __forceinline__ float col_max(float x) {
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}
__device__ __forceinline__ float col_sum(float x) {
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
}

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

}  // namespace vecattn
