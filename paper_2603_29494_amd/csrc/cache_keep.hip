// Which tokens of each head a budget keeps: those at the start (sinks) and the end
// (recent) of the sequence, then the heaviest by the attention weight that they have
// collected, the lower index first among equals.
//
// A workgroup takes a row (a sequence and key/value head).  Weights become 32-bit keys of
// the same order (a protected token the largest, NaN the smallest), and three rounds
// over 11, 11 and 10 bits of them find the key of the last token that is kept: integer
// counts, so that nothing depends on their order.  The tokens above it, and the first of
// those equal to it, are then written in ascending order, each wave its own range.
#include <algorithm>

#include "device_common.h"
#include "launch.h"

namespace vecattn {
namespace {

struct KeepParams {
  const float* mass;
  const int32_t* table;
  const int32_t* lens;
  int32_t* idx;
  int32_t* kept;
  int64_t M, budget, cols, pages;
  int32_t page_shift, H, sinks, recent;
};

constexpr int kThreads = 1024, kWaves = kThreads / 64, kBins = 2048;

// The whole wave's sum, on every lane.
__device__ __forceinline__ int wave_sum(int x) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) x += __shfl_xor(x, o);
  return x;
}

// ITEMS: keys that a thread holds; 0: they are made anew each time they are used.
template <int ITEMS>
__global__ __launch_bounds__(kThreads) void k_cache_keep(const KeepParams a) {
  __shared__ int hist[kBins];
  __shared__ int s_wave[kWaves], s_more[kWaves];
  __shared__ int s_bin, s_above;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int h = blockIdx.x;
  const int64_t b = blockIdx.y, bh = b * a.H + h;
  const int len = min(max(a.lens[b], 0), 1 << 30);
  const int end = static_cast<int>(min<int64_t>(min<int64_t>(len, a.M), a.cols << a.page_shift));
  const float* mass = a.mass + bh * a.M;
  const int32_t* table = a.table + b * a.cols;
  int32_t* idx = a.idx + bh * a.budget;

  // Wave w takes tokens [w span, (w + 1) span).
  const int rounds = (end + kThreads - 1) / kThreads, span = 64 * rounds;
  const int from = wave * span;
  uint64_t held[ITEMS > 0 ? ITEMS : 1];
  uint32_t keys[ITEMS > 0 ? ITEMS : 1];
  auto make = [&](int i, bool& is) __attribute__((always_inline)) {
    const int j = from + 64 * i + lane;
    is = false;
    if (j >= end) return 0u;
    const int64_t page = table[j >> a.page_shift];
    is = page >= 0 && page < a.pages;
    if (!is) return 0u;
    if (j < a.sinks || j >= len - a.recent) return 0xFFFFFFFFu;
    const float x = mass[j] + 0.0f;   // one zero
    const uint32_t bits = __float_as_uint(x);
    return x != x ? 0u : bits & 0x80000000u ? ~bits : bits | 0x80000000u;
  };
  auto each = [&](auto&& f) __attribute__((always_inline)) {
    if constexpr (ITEMS > 0) {
#pragma unroll
      for (int i = 0; i < ITEMS; ++i)
        if (i < rounds) f(i, keys[i], (held[i] >> lane & 1) != 0);
    } else {
#pragma unroll 4
      for (int i = 0; i < rounds; ++i) {
        bool is;
        const uint32_t key = make(i, is);
        f(i, key, is);
      }
    }
  };
  if constexpr (ITEMS > 0) {
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      bool is = false;
      keys[i] = i < rounds ? make(i, is) : 0u;
      held[i] = __ballot(is);
    }
  }
  // Sum over the workgroup of a value that is the same on a wave's lanes.
  auto total = [&](int mine, int* buf) __attribute__((always_inline)) {
    if (lane == 0) buf[wave] = mine;
    __syncthreads();
    int sum = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) sum += buf[w];
    __syncthreads();
    return sum;
  };
  int mine = 0;
  each([&](int, uint32_t, bool is) { mine += is ? 1 : 0; });
  const int n_held = total(wave_sum(mine), s_wave);
  const int n = static_cast<int>(min<int64_t>(n_held, a.budget));
  if (h == 0 && tid == 0) a.kept[b] = n;

  uint32_t last = 0;   // bits of the last key that is kept, from the top
  int need = n;        // of the tokens whose key has those bits
  if (n > 0) {
    int bits = 32;     // still open
#pragma unroll 1
    for (int round = 0; round < 3; ++round) {
      const int take = round == 2 ? 10 : 11, shift = bits - take;
      for (int i = tid; i < kBins; i += kThreads) hist[i] = 0;
      __syncthreads();
      each([&](int, uint32_t key, bool is) {
        if (is && (bits == 32 || key >> bits == last))
          atomicAdd(&hist[key >> shift & ((1u << take) - 1u)], 1);
      });
      __syncthreads();
      // The bin of the need-th largest: each thread two bins, from the top.
      const int top = kBins - 2 - 2 * tid;
      const int c1 = hist[top + 1], c0 = hist[top];
      int incl = c0 + c1;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const int y = __shfl_up(incl, o);
        if (lane >= o) incl += y;
      }
      if (lane == 63) s_wave[wave] = incl;
      __syncthreads();
      int before = 0;
      for (int w = 0; w < wave; ++w) before += s_wave[w];
      const int above = before + incl - c0 - c1;   // in bins above this thread's
      if (above < need && need <= above + c0 + c1) {
        const bool upper = need <= above + c1;
        s_bin = upper ? top + 1 : top;
        s_above = upper ? above : above + c1;
      }
      __syncthreads();
      last = last << take | static_cast<uint32_t>(s_bin);
      need -= s_above;
      bits = shift;
      __syncthreads();
    }
    // Tokens above it, and equal to it, per wave; what the waves before write.
    int more = 0, same = 0;
    each([&](int, uint32_t key, bool is) {
      more += is && key > last ? 1 : 0;
      same += is && key == last ? 1 : 0;
    });
    more = wave_sum(more), same = wave_sum(same);
    if (lane == 0) s_wave[wave] = more, s_more[wave] = same;
    __syncthreads();
    int at = 0, ties = 0;
    for (int w = 0; w < wave; ++w) at += s_wave[w], ties += s_more[w];
    at += min(ties, need);
    const uint64_t below = (uint64_t(1) << lane) - 1;
    each([&](int i, uint32_t key, bool is) {
      const bool tie = is && key == last;
      const uint64_t tie_set = __ballot(tie);
      const bool keep = (is && key > last) ||
                        (tie && ties + __builtin_popcountll(tie_set & below) < need);
      const uint64_t set = __ballot(keep);
      if (keep) idx[at + __builtin_popcountll(set & below)] = from + 64 * i + lane;
      at += __builtin_popcountll(set);
      ties += __builtin_popcountll(tie_set);
    });
  }
  for (int64_t i = n + tid; i < a.budget; i += kThreads) idx[i] = -1;
}

}  // namespace

hipError_t launch_cache_keep(const CacheArgs& c, int64_t B, const float* mass, int64_t M,
                             int64_t budget, int64_t sinks, int64_t recent, int32_t* idx,
                             int32_t* kept, hipStream_t stream) {
  KeepParams a;
  a.mass = mass;
  a.table = c.table;
  a.lens = c.lens;
  a.idx = idx;
  a.kept = kept;
  a.M = M, a.budget = budget, a.cols = c.cols, a.pages = c.pages;
  a.page_shift = __builtin_ctz(static_cast<unsigned>(c.page));
  a.H = c.H;
  a.sinks = static_cast<int32_t>(sinks), a.recent = static_cast<int32_t>(recent);
  const int64_t most = std::min(M, c.cols * c.page);
  const dim3 grid(static_cast<unsigned>(c.H), static_cast<unsigned>(B));
  auto run = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, stream, a); };
  if (most <= 8 * kThreads) run(k_cache_keep<8>);
  else if (most <= 24 * kThreads) run(k_cache_keep<24>);
  else run(k_cache_keep<0>);
  return hipGetLastError();
}

}  // namespace vecattn
