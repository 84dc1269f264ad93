// Rotary positions: pairs of a row's values turned by the row's position times
// the pair's frequency, (a, b) -> f (a cos t - b sin t, a sin t + b cos t), the
// transposed turn with -t.
//
// Angles.  Frequencies come as turns per position in fp64 (off by 2^-52 of themselves);
// position x turns less the nearest quarter turn is one fused multiply-add, so that the
// reduction of a far position costs no digits, and what is left, at most an eighth of a
// turn, goes to fp32.  Its sine and cosine are Taylor sums (the next terms are below 2^-29),
// swapped and signed by the quarter.  Products and their sum are fp32, rounded
// to bf16 once.
//
// A wave takes a token and walks over its heads, q's and then k's; a lane computes the
// angle of one pair, and the others read it from LDS.  Where rows of a head lie beside
// each other (head-major tensors) its rows are consecutive tokens of one head instead, and
// every thread computes the angles that it needs, for all heads.  A thread holds 32 bytes
// of a row: 16-byte chunks c and c + half of the turned values, which are partners in the
// half layout.
//
// Bound by memory, 131072 tokens of 28 + 4 heads of 128: 377 us, 5.7 TB/s; 75600 of 40 + 40:
// 606 us, 5.1 TB/s.  With each thread computing the angles of its own pairs these took 487
// and 650.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "device_common.h"
#include "launch.h"

namespace vecattn {
namespace {

enum Layout { kInterleaved, kHalfChunks, kHalfAny };

struct RopeParams {
  const uint16_t *q, *k;
  uint16_t *qo, *ko;
  int64_t q_sB, q_sH, q_sN, k_sB, k_sH, k_sN;
  int64_t qo_sB, qo_sH, qo_sN, ko_sB, ko_sH, ko_sN;
  const int32_t* pos;
  int64_t pos_sA, pos_sB;
  const int32_t *lens, *n_new;
  int64_t start;
  int64_t N;
  int64_t units;      // runs of tokens, of all sequences
  int32_t runs;       // runs of tokens per sequence
  int32_t Hq, heads;  // q's heads, and k's with them
  int32_t token_log2; // a wave's rows are 1 << token_log2 tokens by the rest in heads
  int32_t split;      // waves that share a run's heads
  int32_t rot, in_place, clear;
  float factor;       // negated sines for the transposed turn
  float sine;
  double turns[kRopeMaxPairs];
  uint8_t axis[kRopeMaxPairs];
};

struct Turn {
  float c, s;
};

// Cosine and sine of 2 pi (pos x turns), times f and fs.
__device__ __forceinline__ Turn turn_of(double pos, double turns, float f, float fs) {
  const double quarters = 4.0 * turns;   // exact
  // Beside 2^52 a sum is an integer, in its low bits too (here below 2^41).
  const double big = __builtin_fma(pos, quarters, 0x1.8p52), n = big - 0x1.8p52;
  const float r = static_cast<float>(__builtin_fma(pos, quarters, -n));   // quarter turns, |r| <= 1/2
  const int quad = static_cast<int>(__double_as_longlong(big)) & 3;
  const float x = r * 1.57079632679489662f;   // pi / 2
  const float x2 = x * x;
  float s = __builtin_fmaf(x2, 1.0f / 362880.0f, -1.0f / 5040.0f);
  s = __builtin_fmaf(x2, s, 1.0f / 120.0f);
  s = __builtin_fmaf(x2, s, -1.0f / 6.0f);
  s = __builtin_fmaf(x2 * x, s, x);
  float c = __builtin_fmaf(x2, -1.0f / 3628800.0f, 1.0f / 40320.0f);
  c = __builtin_fmaf(x2, c, -1.0f / 720.0f);
  c = __builtin_fmaf(x2, c, 1.0f / 24.0f);
  c = __builtin_fmaf(x2, c, -0.5f);
  c = __builtin_fmaf(x2, c, 1.0f);
  float cq = quad & 1 ? -s : c, sq = quad & 1 ? c : s;
  if (quad & 2) cq = -cq, sq = -sq;
  return Turn{cq * f, sq * fs};
}

__device__ __forceinline__ float lo16(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi16(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }
__device__ __forceinline__ uint32_t pack16(float lo, float hi) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{lo, hi}, bf16x2));
}

// A 16-byte chunk; STREAM: past the caches.
template <bool STREAM>
__device__ __forceinline__ u32x4 load_chunk(const uint16_t* row, int c) {
  const u32x4* at = reinterpret_cast<const u32x4*>(row) + c;
  if constexpr (STREAM) return __builtin_nontemporal_load(at);
  return *at;
}
template <bool STREAM>
__device__ __forceinline__ void store_chunk(uint16_t* row, int c, u32x4 x) {
  u32x4* at = reinterpret_cast<u32x4*>(row) + c;
  if constexpr (STREAM) __builtin_nontemporal_store(x, at);
  else *at = x;
}

template <int D, int LAYOUT, bool STREAM>
__global__ __launch_bounds__(256) void k_rope(const RopeParams a) {
  constexpr int TH = D / 16;          // threads per row
  constexpr int ROWS = 64 / TH;       // rows of a wave
  constexpr int PAIRS = LAYOUT == kHalfAny ? 16 : 8;   // angles a thread needs
  const int lane = threadIdx.x & 63, j = lane % TH, r = lane / TH;
  const int64_t block = blockIdx.y * static_cast<int64_t>(gridDim.x) + blockIdx.x;
  const int64_t wave = block * 4 + (threadIdx.x >> 6);
  const int64_t unit = wave / a.split;
  if (unit >= a.units) return;
  const int part = static_cast<int>(wave % a.split);
  const int64_t b = unit / a.runs;
  const int tokens = 1 << a.token_log2, heads = ROWS >> a.token_log2;
  const int64_t n = (unit % a.runs) * tokens + (r & (tokens - 1));
  const int64_t rows = a.n_new ? min(max(static_cast<int64_t>(a.n_new[b]), int64_t(0)), a.N) : a.N;
  const bool gone = n >= rows;
  if (n >= a.N || (gone && !a.clear)) return;

  // Chunks (of eight values) that this thread holds.
  const int half = a.rot >> 1;
  int c0 = j, c1 = j + TH;
  if constexpr (LAYOUT == kHalfChunks) {
    const int pairs8 = half >> 3;
    c1 = j + pairs8;
    if (j >= pairs8) c0 = 2 * j, c1 = 2 * j + 1;   // behind the turned values
  }
  const bool turned0 = 8 * c0 < a.rot, turned1 = 8 * c1 < a.rot;
  const bool store0 = turned0 || gone || !a.in_place, store1 = turned1 || gone || !a.in_place;
  // Values of chunk 0 or 1 belong to pair index:
  Turn t[PAIRS];
  const double p0 = a.pos ? 0.0
                          : static_cast<double>(a.lens ? static_cast<int64_t>(a.lens[b]) - rows + n
                                                       : a.start + n);
  auto angle = [&](int pair) __attribute__((always_inline)) {
    double p = p0;
    if (a.pos) p = a.pos[a.axis[pair] * a.pos_sA + b * a.pos_sB + n];
    return turn_of(p, a.turns[pair], a.factor, a.sine);
  };
  __shared__ Turn table[4][kRopeMaxPairs];
  Turn* shared = table[threadIdx.x >> 6];
  if (a.token_log2 == 0 && lane < half) shared[lane] = angle(lane);
  __builtin_amdgcn_wave_barrier();   // a wave's LDS accesses keep their order
  if (turned0 || turned1) {
#pragma unroll
    for (int i = 0; i < PAIRS; ++i) {
      int pair;
      if constexpr (LAYOUT == kInterleaved) pair = 4 * (i < 4 ? c0 : c1) + (i & 3);
      else if constexpr (LAYOUT == kHalfChunks) pair = 8 * c0 + i;
      else {
        const int d = 8 * (i < 8 ? c0 : c1) + (i & 7);
        pair = d < half ? d : d - half;
      }
      pair = min(pair, half - 1);   // of those past the turned values nothing is used
      t[i] = a.token_log2 == 0 ? shared[pair] : angle(pair);
    }
  }
  for (int h = part * heads + (r >> a.token_log2); h < a.heads; h += a.split * heads) {
    const bool is_q = h < a.Hq;
    const int hh = is_q ? h : h - a.Hq;
    const uint16_t* src = is_q ? a.q + b * a.q_sB + hh * a.q_sH + n * a.q_sN
                               : a.k + b * a.k_sB + hh * a.k_sH + n * a.k_sN;
    uint16_t* dst = is_q ? a.qo + b * a.qo_sB + hh * a.qo_sH + n * a.qo_sN
                         : a.ko + b * a.ko_sB + hh * a.ko_sH + n * a.ko_sN;
    u32x4 x0 = {}, x1 = {};
    if (store0) x0 = load_chunk<STREAM>(src, c0);
    if (store1) x1 = load_chunk<STREAM>(src, c1);
    if constexpr (LAYOUT == kInterleaved) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float a0 = lo16(x0[e]), b0 = hi16(x0[e]), a1 = lo16(x1[e]), b1 = hi16(x1[e]);
        const uint32_t y0 = pack16(__builtin_fmaf(a0, t[e].c, -(b0 * t[e].s)),
                                   __builtin_fmaf(a0, t[e].s, b0 * t[e].c));
        const uint32_t y1 = pack16(__builtin_fmaf(a1, t[4 + e].c, -(b1 * t[4 + e].s)),
                                   __builtin_fmaf(a1, t[4 + e].s, b1 * t[4 + e].c));
        if (8 * c0 + 2 * e < a.rot) x0[e] = y0;
        if (8 * c1 + 2 * e < a.rot) x1[e] = y1;
      }
    } else if constexpr (LAYOUT == kHalfChunks) {
      if (turned0) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const Turn u = t[2 * e], w = t[2 * e + 1];
          const float a0 = lo16(x0[e]), b0 = lo16(x1[e]), a1 = hi16(x0[e]), b1 = hi16(x1[e]);
          x0[e] = pack16(__builtin_fmaf(a0, u.c, -(b0 * u.s)), __builtin_fmaf(a1, w.c, -(b1 * w.s)));
          x1[e] = pack16(__builtin_fmaf(a0, u.s, b0 * u.c), __builtin_fmaf(a1, w.s, b1 * w.c));
        }
      }
    } else {
      // Partners lie anywhere in the row: one value at a time.  All of the row is read
      // by this wave before any of it is written (the barrier below keeps it so).
      float y[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int d = 8 * (i < 8 ? c0 : c1) + (i & 7);
        const u32x4& x = i < 8 ? x0 : x1;
        const float own = (i & 1) ? hi16(x[(i & 7) / 2]) : lo16(x[(i & 7) / 2]);
        y[i] = own;
        if (d < a.rot) {
          const float other = bf16_bits_to_f32(src[d < half ? d + half : d - half]);
          y[i] = d < half ? __builtin_fmaf(own, t[i].c, -(other * t[i].s))
                          : __builtin_fmaf(other, t[i].s, own * t[i].c);
        }
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t y0 = pack16(y[2 * e], y[2 * e + 1]), y1 = pack16(y[8 + 2 * e], y[9 + 2 * e]);
        if (8 * c0 + 2 * e < a.rot) x0[e] = y0;
        if (8 * c1 + 2 * e < a.rot) x1[e] = y1;
      }
      __builtin_amdgcn_wave_barrier();
    }
    if (gone) x0 = x1 = u32x4{0, 0, 0, 0};
    if (store0) store_chunk<STREAM>(dst, c0, x0);
    if (store1) store_chunk<STREAM>(dst, c1, x1);
  }
}

}  // namespace

hipError_t launch_rope(const RopeArgs& x, hipStream_t stream) {
  RopeParams a;
  const bool with_k = x.k.ptr != nullptr;
  a.q = static_cast<const uint16_t*>(x.q.ptr);
  a.q_sB = x.q.sB, a.q_sH = x.q.sH, a.q_sN = x.q.sN;
  a.qo = static_cast<uint16_t*>(const_cast<void*>(x.qo.ptr));
  a.qo_sB = x.qo.sB, a.qo_sH = x.qo.sH, a.qo_sN = x.qo.sN;
  a.k = static_cast<const uint16_t*>(x.k.ptr);
  a.k_sB = x.k.sB, a.k_sH = x.k.sH, a.k_sN = x.k.sN;
  a.ko = static_cast<uint16_t*>(const_cast<void*>(x.ko.ptr));
  a.ko_sB = x.ko.sB, a.ko_sH = x.ko.sH, a.ko_sN = x.ko.sN;
  a.pos = x.pos, a.pos_sA = x.pos_sA, a.pos_sB = x.pos_sB;
  a.lens = x.lens, a.n_new = x.n_new;
  a.start = x.start;
  a.N = x.q.N;
  a.Hq = static_cast<int32_t>(x.q.H);
  a.heads = static_cast<int32_t>(x.q.H + (with_k ? x.k.H : 0));
  a.rot = x.rot;
  // Values behind the turned ones stay where they are if both tensors do.
  a.in_place = x.q.ptr == x.qo.ptr && (!with_k || x.k.ptr == x.ko.ptr);
  a.clear = x.clear;
  a.factor = static_cast<float>(x.factor);
  a.sine = x.transposed ? -a.factor : a.factor;
  for (int i = 0; i < x.rot / 2; ++i) {
    a.turns[i] = x.freq[i] * 0.15915494309189533577;   // 1 / (2 pi)
    a.axis[i] = static_cast<uint8_t>(x.axis ? x.axis[i] : 0);
  }
  const int rows = 64 / static_cast<int>(x.q.D / 16);
  // Rows of a wave: tokens of a head where those lie closer together than heads do.
  a.token_log2 = x.q.sH > x.q.sN && x.q.N > 1 ? __builtin_ctz(static_cast<unsigned>(rows)) : 0;
  const int64_t tokens = int64_t(1) << a.token_log2;
  a.runs = static_cast<int32_t>((x.q.N + tokens - 1) / tokens);
  a.units = x.q.B * a.runs;
  // Few tokens: their heads are shared by as many waves as it takes to fill the chip.
  const int64_t passes = (a.heads + rows / tokens - 1) / (rows / tokens);
  a.split = static_cast<int32_t>(std::min(passes, std::max<int64_t>(1, 8192 / a.units)));
  // A dimension of a launch holds fewer than 2^32 threads (the API takes more without an error,
  // and runs what is left of them).
  const int64_t blocks = (a.units * a.split + 3) / 4, most = int64_t(1) << 22;
  const dim3 grid(static_cast<unsigned>(std::min(blocks, most)),
                  static_cast<unsigned>((blocks + most - 1) / most));
  const int layout = !x.half ? kInterleaved : x.rot % 16 == 0 ? kHalfChunks : kHalfAny;
  // What is turned, in and out, is past 256 MB: no cache holds it until it is read (131072
  // tokens of 32 heads: 399 us through the caches, 377 past them).
  const bool stream_past = 4 * x.q.B * x.q.N * a.heads * x.q.D > (int64_t(256) << 20);
  auto run = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, stream, a); };
  auto pick = [&](auto dim, auto past) {
    constexpr int D = decltype(dim)::value;
    constexpr bool PAST = decltype(past)::value;
    if (layout == kInterleaved) run(k_rope<D, kInterleaved, PAST>);
    else if (layout == kHalfChunks) run(k_rope<D, kHalfChunks, PAST>);
    else run(k_rope<D, kHalfAny, PAST>);
  };
  using std::integral_constant;
  if (x.q.D == 128)
    stream_past ? pick(integral_constant<int, 128>{}, std::true_type{})
                : pick(integral_constant<int, 128>{}, std::false_type{});
  else
    stream_past ? pick(integral_constant<int, 64>{}, std::true_type{})
                : pick(integral_constant<int, 64>{}, std::false_type{});
  return hipGetLastError();
}

}  // namespace vecattn
