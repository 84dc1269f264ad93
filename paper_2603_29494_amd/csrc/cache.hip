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
// memory.
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

// Eight values of a token: codes (0..M) and, on every lane of the eight that
// hold the group, its (m, s) dword.
template <int BITS>
__device__ __forceinline__ uint32_t quantise8(const u32x4 w, int (&u)[8]) {
  constexpr float M = BITS == 4 ? 15.0f : 255.0f;
  float x[8];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    x[2 * e] = __uint_as_float(w[e] << 16);
    x[2 * e + 1] = __uint_as_float(w[e] & 0xFFFF0000u);
  }
  float lo = x[0], hi = x[0], bad = x[0] * 0.0f;  // bad: 0, or NaN
#pragma unroll
  for (int e = 1; e < 8; ++e) {
    lo = fminf(lo, x[e]);
    hi = fmaxf(hi, x[e]);
    bad += x[e] * 0.0f;
  }
#pragma unroll
  for (int o = 1; o < 8; o <<= 1) {
    lo = fminf(lo, __shfl_xor(lo, o));
    hi = fmaxf(hi, __shfl_xor(hi, o));
    bad += __shfl_xor(bad, o);
  }
  const float range = hi - lo;
  if (!(bad == 0.0f) || !(range < INFINITY)) {
#pragma unroll
    for (int e = 0; e < 8; ++e) u[e] = 0;
    return 0x7FC07FC0u;
  }
  const __bf16 sb = static_cast<__bf16>(range / M);
  float s = static_cast<float>(sb);
  uint32_t sbits = __builtin_bit_cast(uint16_t, sb);
  if (s < 0x1p-100f) {
    s = 0.0f;
    sbits = 0;
  }
#pragma unroll
  for (int e = 0; e < 8; ++e)
    u[e] = s == 0.0f ? 0 : static_cast<int>(fminf(M, __builtin_rintf((x[e] - lo) / s)));
  return (__float_as_uint(lo) >> 16) | (sbits << 16);
}

template <int D, int BITS>
__global__ __launch_bounds__(256) void k_cache_write(
    const uint16_t* __restrict__ k, int64_t k_sB, int64_t k_sH, int64_t k_sN,
    const uint16_t* __restrict__ v, int64_t v_sB, int64_t v_sH, int64_t v_sN, int32_t n,
    const int32_t* __restrict__ lens, const int32_t* __restrict__ n_new, PageMap map) {
  using L = CacheLayout<D, BITS>;
  constexpr int CH = D / 8;               // 8-value chunks per row
  constexpr int RPP = 256 / CH;           // rows per pass
  const int64_t b = blockIdx.z;
  const int h = blockIdx.y;
  const int64_t len = min(max(lens[b], 0), 1 << 30);
  const int64_t nb = n_new ? min(max(n_new[b], 0), n) : n;
  const int64_t p0 = len - nb;            // position of row 0
  const int64_t jb = (max(p0, int64_t(0)) >> 5) + blockIdx.x;
  const int64_t j0 = jb * kCacheBlock;
  if (nb == 0 || j0 >= len) return;
  uint8_t* blk = block_ptr<L::kBytes>(map, b, h, jb);
  if (!blk) return;
  __shared__ uint8_t codes[kCacheBlock][D];  // V's

  const int c = threadIdx.x % CH;
#pragma unroll
  for (int pass = 0; pass < kCacheBlock / RPP; ++pass) {
    const int key = pass * RPP + threadIdx.x / CH;
    const int64_t r = j0 + key - p0;
    const bool have = r >= 0 && r < nb;   // the same for the lanes of a group
    u32x4 kw = {0, 0, 0, 0}, vw = {0, 0, 0, 0};
    if (have) {
      kw = *reinterpret_cast<const u32x4*>(k + b * k_sB + h * k_sH + r * k_sN + 8 * c);
      vw = *reinterpret_cast<const u32x4*>(v + b * v_sB + h * v_sH + r * v_sN + 8 * c);
    }
    int u[8];
    uint32_t par = quantise8<BITS>(kw, u);
    if (have) {
      uint32_t dw[L::kDw] = {};
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if constexpr (BITS == 4) dw[0] |= static_cast<uint32_t>(u[e]) << (4 * k_nibble(e));
        else dw[e >> 2] |= static_cast<uint32_t>(u[e]) << (8 * (e & 3));
      }
      const int w0 = ((key >> 4) * (D / 32) + (c >> 2)) * L::kDw, l = (c & 3) * 16 + (key & 15);
#pragma unroll
      for (int x = 0; x < L::kDw; ++x)
        *reinterpret_cast<uint32_t*>(blk + code_byte(w0 + x, l)) = dw[x];
      if (c % 8 == 0)
        reinterpret_cast<uint32_t*>(blk + L::kCodes)[key * L::kG + c / 8] = par;
    }
    par = quantise8<BITS>(vw, u);
    uint32_t pk[2] = {0, 0};
#pragma unroll
    for (int e = 0; e < 8; ++e) pk[e >> 2] |= static_cast<uint32_t>(u[e]) << (8 * (e & 3));
    *reinterpret_cast<u32x2*>(&codes[key][8 * c]) = u32x2{pk[0], pk[1]};
    if (have && c % 8 == 0)
      reinterpret_cast<uint32_t*>(blk + L::kHalf + L::kCodes)[key * L::kG + c / 8] = par;
  }
  __syncthreads();
  // V's codes, eight tokens of a head-dim value at a time; codes of tokens that
  // this call does not write stay as they are.
  for (int it = threadIdx.x; it < 4 * D; it += 256) {
    const int d = it % D, g = it / D;
    uint32_t dw[L::kDw] = {}, mask[L::kDw] = {};
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int key = (e >> 2) * 16 + 4 * g + (e & 3);
      const int64_t r = j0 + key - p0;
      const bool have = r >= 0 && r < nb;
      const uint32_t u = codes[key][d];
      const int x = BITS == 4 ? 0 : e >> 2, sh = BITS == 4 ? 4 * v_nibble(e) : 8 * (e & 3);
      if (have) {
        dw[x] |= u << sh;
        mask[x] |= (BITS == 4 ? 0xFu : 0xFFu) << sh;
      }
    }
#pragma unroll
    for (int x = 0; x < L::kDw; ++x) {
      if (mask[x] == 0) continue;
      uint32_t* at = reinterpret_cast<uint32_t*>(
          blk + L::kHalf + code_byte((d >> 4) * L::kDw + x, g * 16 + (d & 15)));
      *at = mask[x] == 0xFFFFFFFFu ? dw[x] : (*at & ~mask[x]) | dw[x];
    }
  }
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

template <int BITS, bool V>
__device__ __forceinline__ void unpack8(const uint32_t (&dw)[BITS / 4], int (&u)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    if constexpr (BITS == 4) u[e] = (dw[0] >> (4 * (V ? v_nibble(e) : k_nibble(e)))) & 0xF;
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
    unpack8<BITS, true>(dw, u);
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
    unpack8<BITS, false>(dw, u);
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
    hipLaunchKernelGGL(kernel, grid, dim3(256), 0, stream, static_cast<const uint16_t*>(k.ptr),
                       k.sB, k.sH, k.sN, static_cast<const uint16_t*>(v.ptr), v.sB, v.sH, v.sN,
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
