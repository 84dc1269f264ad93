// Which tokens of each head a budget keeps: those at the start (sinks) and the end
// (recent) of the sequence, then the heaviest by the attention weight that they have
// collected, the lower index first among equals.
//
// Weights become 32-bit keys of the same order (a protected token the largest, NaN the
// smallest, 0 no token), and three rounds over 11, 11 and 10 bits of them find the key of the
// last token that is kept: integer counts, so that nothing depends on their order.  The
// tokens above it, and the first of those equal to it, are then written in ascending order,
// each wave its own range.
//
// A row (a sequence and key/value head) of up to 32768 tokens is one workgroup's, its keys
// in registers: 9 us for 700 tokens, 14 for 8192, 36 for 32768 (in six launches the same, and
// 242 instead of 85 for 512 such rows).  Longer ones are cut into segments of 8192, a
// workgroup each, with a launch per round, and counts that meet in the workspace: 16 rows of
// 131072 tokens take 43 us in six launches of 5 to 9 us each, against 330 us for a CU alone
// per row.  What bounds either is the chain of rounds, each a load, counts in LDS and a scan
// over its bins.
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
  int32_t* work;      // [row] of work_size counts
  int64_t work_size;
};

constexpr int kThreads = 1024, kWaves = kThreads / 64, kItems = 8, kBins = 2048;
constexpr int kSegment = kThreads * kItems;

// A row's counts in the workspace: of each round's bins, of the tokens that a page holds,
// what each round has found (bits of the last kept key, and how many of the tokens with
// those bits are kept), and per segment the tokens above and equal to that key.
constexpr int kHeld = 2 * kBins + kBins / 2, kState = kHeld + 1, kSegments = kState + 6;

__device__ __forceinline__ int wave_sum(int x) {   // on every lane
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) x += __shfl_xor(x, o);
  return x;
}

// A workgroup's tokens, up to kSegment from `base` on: wave w takes [span w, span (w + 1))
// of them.
template <int ITEMS>
struct Keys {
  uint32_t key[ITEMS];   // 0: no token that a page holds
  int from, rounds;

  __device__ __forceinline__ void load(const KeepParams& a, int64_t b, int64_t bh, int base, int end,
                                       int len, int lane, int wave) {
    rounds = (min(end - base, ITEMS * kThreads) + kThreads - 1) / kThreads;
    from = base + wave * 64 * rounds;
    const float* mass = a.mass + bh * a.M;
    const int32_t* table = a.table + b * a.cols;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      const int j = from + 64 * i + lane;
      uint32_t k = 0;
      if (i < rounds && j < end) {
        const float x = mass[j] + 0.0f;   // one zero
        const int64_t page = table[j >> a.page_shift];
        const uint32_t bits = __float_as_uint(x);
        k = x != x ? 1u : bits & 0x80000000u ? ~bits : bits | 0x80000000u;
        if (j < a.sinks || j >= len - a.recent) k = 0xFFFFFFFFu;
        if (page < 0 || page >= a.pages) k = 0;
      }
      key[i] = k;
    }
  }
  template <typename F>
  __device__ __forceinline__ void each(F&& f) const {
#pragma unroll
    for (int i = 0; i < ITEMS; ++i)
      if (i < rounds) f(i, key[i], key[i] != 0);
  }
};

struct Row {
  int64_t b, bh;
  int len, end;   // tokens, and of them those that have an entry and a place in the table
};
__device__ __forceinline__ Row row_of(const KeepParams& a, int64_t b, int h) {
  Row r;
  r.b = b;
  r.bh = b * a.H + h;
  r.len = min(max(a.lens[b], 0), 1 << 30);
  r.end = static_cast<int>(min<int64_t>(min<int64_t>(r.len, a.M), a.cols << a.page_shift));
  return r;
}

constexpr int bits_of(int round) { return round == 2 ? 10 : 11; }
constexpr int shift_of(int round) { return round == 0 ? 21 : round == 1 ? 10 : 0; }

struct Shared {
  int hist[kBins];
  int wave[kWaves], more[kWaves];
  int bin, above;
};

// Counts, into hist, the held keys whose bits above the round's are `last`.
template <int ITEMS>
__device__ __forceinline__ void count_bins(const Keys<ITEMS>& k, Shared& s, int round, uint32_t last) {
  const int shift = shift_of(round), take = bits_of(round);
  for (int i = threadIdx.x; i < kBins; i += kThreads) s.hist[i] = 0;
  __syncthreads();
  k.each([&](int, uint32_t key, bool is) {
    if (is && (round == 0 || key >> (shift + take) == last))
      atomicAdd(&s.hist[key >> shift & ((1u << take) - 1u)], 1);
  });
  __syncthreads();
}

// The bin of the need-th largest (need >= 1, of as many at least): `last` takes its bits,
// `need` becomes what is left for it.  Each thread two bins, from the top.
__device__ __forceinline__ void find_bin(Shared& s, int round, uint32_t& last, int& need) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int top = kBins - 2 - 2 * tid;
  const int c1 = s.hist[top + 1], c0 = s.hist[top];
  int incl = c0 + c1;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int y = __shfl_up(incl, o);
    if (lane >= o) incl += y;
  }
  if (lane == 63) s.wave[wave] = incl;
  __syncthreads();
  int before = 0;
  for (int w = 0; w < wave; ++w) before += s.wave[w];
  const int above = before + incl - c0 - c1;   // in bins above this thread's
  if (above < need && need <= above + c0 + c1) {
    const bool upper = need <= above + c1;
    s.bin = upper ? top + 1 : top;
    s.above = upper ? above : above + c1;
  }
  __syncthreads();
  last = last << bits_of(round) | static_cast<uint32_t>(s.bin);
  need -= s.above;
  __syncthreads();
}

// Tokens above the last kept key, and equal to it, of the waves before this one, and of
// all.
struct Before {
  int more, same, all_more, all_same;
};
template <int ITEMS>
__device__ __forceinline__ Before count_kept(const Keys<ITEMS>& k, Shared& s, uint32_t last) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int more = 0, same = 0;
  k.each([&](int, uint32_t key, bool is) {
    more += is && key > last ? 1 : 0;
    same += is && key == last ? 1 : 0;
  });
  more = wave_sum(more), same = wave_sum(same);
  if (lane == 0) s.wave[wave] = more, s.more[wave] = same;
  __syncthreads();
  Before r{0, 0, 0, 0};
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    if (w < wave) r.more += s.wave[w], r.same += s.more[w];
    r.all_more += s.wave[w], r.all_same += s.more[w];
  }
  __syncthreads();
  return r;
}

// Writes the kept ones of a wave; more and same: kept and equal ones before them.
template <int ITEMS>
__device__ __forceinline__ void write_kept(const Keys<ITEMS>& k, int32_t* idx, uint32_t last, int need,
                                           int more, int same) {
  const int lane = threadIdx.x & 63;
  const uint64_t below = (uint64_t(1) << lane) - 1;
  int at = more + min(same, need);
  k.each([&](int i, uint32_t key, bool is) {
    const bool tie = is && key == last;
    const uint64_t ties = __ballot(tie);
    const bool keep = (is && key > last) || (tie && same + __builtin_popcountll(ties & below) < need);
    const uint64_t set = __ballot(keep);
    if (keep) idx[at + __builtin_popcountll(set & below)] = k.from + 64 * i + lane;
    at += __builtin_popcountll(set);
    same += __builtin_popcountll(ties);
  });
}

template <int ITEMS>
__device__ __forceinline__ int count_held(const Keys<ITEMS>& k, Shared& s) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  int mine = 0;
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) mine += __builtin_popcountll(__ballot(k.key[i] != 0));
  if (lane == 0) s.wave[wave] = mine;
  __syncthreads();
  int sum = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) sum += s.wave[w];
  __syncthreads();
  return sum;
}

// Rows of one workgroup.
template <int ITEMS>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(ITEMS > 8 ? 4 : 8)))
void k_keep_row(const KeepParams a) {
  __shared__ Shared s;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Row r = row_of(a, blockIdx.y, blockIdx.x);
  int32_t* idx = a.idx + r.bh * a.budget;
  Keys<ITEMS> k;
  k.load(a, r.b, r.bh, 0, r.end, r.len, lane, wave);
  const int n = static_cast<int>(min<int64_t>(count_held(k, s), a.budget));
  if (blockIdx.x == 0 && threadIdx.x == 0) a.kept[r.b] = n;
  if (n > 0) {
    uint32_t last = 0;
    int need = n;
#pragma unroll 1
    for (int round = 0; round < 3; ++round) {
      count_bins(k, s, round, last);
      find_bin(s, round, last, need);
    }
    const Before before = count_kept(k, s, last);
    write_kept(k, idx, last, need, before.more, before.same);
  }
  for (int64_t i = n + threadIdx.x; i < a.budget; i += kThreads) idx[i] = -1;
}

// Rows of several segments: a launch per round.
__global__ __launch_bounds__(256) void k_keep_clear(const KeepParams a) {
  int32_t* work = a.work + (static_cast<int64_t>(blockIdx.y) * a.H + blockIdx.x) * a.work_size;
  for (int i = threadIdx.x; i < kState; i += 256) work[i] = 0;
}

// ROUND 0 .. 2 count bins, 3 counts each segment's kept tokens, 4 writes them.
template <int ROUND>
__global__ __launch_bounds__(kThreads) void k_keep_round(const KeepParams a) {
  __shared__ Shared s;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int64_t b = blockIdx.z;
  const int h = blockIdx.y, seg = blockIdx.x;
  const Row r = row_of(a, b, h);
  const int base = seg * kSegment;
  int32_t* work = a.work + r.bh * a.work_size;
  int32_t* segs = work + kSegments;
  if (base >= r.end && (ROUND < 4 || seg > 0)) return;   // the first one fills the list
  uint32_t last = 0;
  int need = 0, n = 0;
  if constexpr (ROUND > 0) n = static_cast<int>(min<int64_t>(work[kHeld], a.budget));
  if constexpr (ROUND > 0 && ROUND < 4) {
    if (n == 0) return;
    // What the round before has found, and its bins.
    need = n;
    if constexpr (ROUND > 1) {
      last = static_cast<uint32_t>(work[kState + 2 * (ROUND - 2)]);
      need = work[kState + 2 * (ROUND - 2) + 1];
    }
    const int bins = 1 << bits_of(ROUND - 1);
    for (int i = tid; i < kBins; i += kThreads)
      s.hist[i] = i < bins ? work[(ROUND - 1) * kBins + i] : 0;
    __syncthreads();
    find_bin(s, ROUND - 1, last, need);
    if (seg == 0 && tid == 0) {
      work[kState + 2 * (ROUND - 1)] = static_cast<int>(last);
      work[kState + 2 * (ROUND - 1) + 1] = need;
    }
  }
  Keys<kItems> k;
  k.load(a, b, r.bh, base, r.end, r.len, lane, wave);
  if constexpr (ROUND < 3) {
    if constexpr (ROUND == 0) {
      const int held = count_held(k, s);
      if (tid == 0) atomicAdd(&work[kHeld], held);
    }
    count_bins(k, s, ROUND, last);
    for (int i = tid; i < kBins; i += kThreads)
      if (s.hist[i] > 0) atomicAdd(&work[ROUND * kBins + i], s.hist[i]);
  } else if constexpr (ROUND == 3) {
    const Before all = count_kept(k, s, last);
    if (tid == 0) segs[2 * seg] = all.all_more, segs[2 * seg + 1] = all.all_same;
  } else {
    if (h == 0 && seg == 0 && tid == 0) a.kept[b] = n;
    int32_t* idx = a.idx + r.bh * a.budget;
    if (n > 0) {
      last = static_cast<uint32_t>(work[kState + 4]);
      need = work[kState + 5];
      // Tokens of the segments before.
      int more = 0, same = 0;
      for (int i = tid; i < seg; i += kThreads) more += segs[2 * i], same += segs[2 * i + 1];
      more = wave_sum(more), same = wave_sum(same);
      if (lane == 0) s.wave[wave] = more, s.more[wave] = same;
      __syncthreads();
      more = same = 0;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) more += s.wave[w], same += s.more[w];
      __syncthreads();
      const Before before = count_kept(k, s, last);
      write_kept(k, idx, last, need, more + before.more, same + before.same);
    }
    if (seg == 0)
      for (int64_t i = n + tid; i < a.budget; i += kThreads) idx[i] = -1;
  }
}

int64_t tokens_of(int64_t M, const CacheArgs& c) { return std::min(M, c.cols * c.page); }
constexpr int64_t kWholeRow = 4 * kSegment;   // tokens that one workgroup takes
int64_t segments_of(int64_t M, const CacheArgs& c) {
  return (tokens_of(M, c) + kSegment - 1) / kSegment;
}

}  // namespace

size_t cache_keep_workspace_bytes(const CacheArgs& c, int64_t B, int64_t M) {
  if (tokens_of(M, c) <= kWholeRow) return 0;
  const int64_t segments = segments_of(M, c);
  return static_cast<size_t>(B) * c.H * (kSegments + 2 * segments) * sizeof(int32_t);
}

hipError_t launch_cache_keep(const CacheArgs& c, int64_t B, const float* mass, int64_t M,
                             int64_t budget, int64_t sinks, int64_t recent, int32_t* idx,
                             int32_t* kept, void* workspace, hipStream_t stream) {
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
  const int64_t segments = segments_of(M, c);
  a.work = static_cast<int32_t*>(workspace);
  a.work_size = kSegments + 2 * segments;
  const dim3 rows(static_cast<unsigned>(c.H), static_cast<unsigned>(B));
  const int64_t tokens = tokens_of(M, c);
  if (tokens <= kWholeRow) {
    auto run = [&](auto kernel) { hipLaunchKernelGGL(kernel, rows, dim3(kThreads), 0, stream, a); };
    if (tokens <= kSegment) run(k_keep_row<8>);
    else if (tokens <= 2 * kSegment) run(k_keep_row<16>);
    else run(k_keep_row<32>);
    return hipGetLastError();
  }
  const dim3 grid(static_cast<unsigned>(segments), static_cast<unsigned>(c.H),
                  static_cast<unsigned>(B));
  hipLaunchKernelGGL(k_keep_clear, rows, dim3(256), 0, stream, a);
  hipLaunchKernelGGL(k_keep_round<0>, grid, dim3(kThreads), 0, stream, a);
  hipLaunchKernelGGL(k_keep_round<1>, grid, dim3(kThreads), 0, stream, a);
  hipLaunchKernelGGL(k_keep_round<2>, grid, dim3(kThreads), 0, stream, a);
  hipLaunchKernelGGL(k_keep_round<3>, grid, dim3(kThreads), 0, stream, a);
  hipLaunchKernelGGL(k_keep_round<4>, grid, dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace vecattn
