// How the attention over the cache deals its work out: what a row tile sees of a
// sequence's tokens, and the chunks that the blocks of all row tiles are cut into.
// Shared by the kernels of a few rows (cache_attn.hip) and of many (cache_chunk.hip).
#pragma once

#include "cache_common.h"
#include "wave_scan.h"

namespace vecattn {

constexpr float kUnseen = -3.4028234663852886e38f;  // reference of a row that has met no key
constexpr int32_t kMaxLen = 1 << 30;                 // positions stay in 32 bits
constexpr float kLn2 = 0.69314718055994531f;

struct AttnParams {
  const uint16_t* q;
  int64_t q_sB, q_sH, q_sN;
  uint16_t* o;
  int64_t o_sB, o_sH, o_sN;
  float* lse;
  const uint8_t* data;
  const int32_t* table;
  const int32_t* lens;
  const int32_t* n_new;
  float* part;       // [item][rows of a tile][D] sums, then [item][rows of a tile] (m, l)
  int32_t cols, pages;   // pages past the first 2^31 - 1 cannot be named
  int32_t window, sinks;
  int32_t H, n, group, page_shift;
  int32_t tiles;     // row tiles per head
  int32_t units;     // row tiles of all sequences
  int32_t items;     // chunks that partial results have room for
  int32_t target;    // most chunks, of all heads (0: one per row tile)
  int32_t least;     // blocks of a chunk at least
  float scale_log2;
};

// What one row tile sees, in blocks of 32 tokens: the first `ns` blocks (sinks),
// then blocks nb0 ..; `total` of both.
struct Span {
  int32_t p_first;      // position of the sequence's row 0
  int32_t p_lo, p_hi;   // positions of the tile's rows
  int32_t ns, nb0, total;
  int32_t rows;         // rows of the sequence (all tiles)
};

__device__ __forceinline__ Span span_of(const AttnParams& a, int64_t b, int row0, int nrows) {
  Span s;
  const int len = min(max(a.lens[b], 0), kMaxLen);
  const int nb = a.n_new ? min(max(a.n_new[b], 0), a.n) : a.n;
  s.p_first = len - nb;
  s.rows = nb * a.group;
  s.p_lo = s.p_first + row0 / a.group;
  s.p_hi = s.p_first + (min(row0 + nrows, s.rows) - 1) / a.group;
  s.ns = s.nb0 = s.total = 0;
  if (row0 >= s.rows || s.p_hi < 0) return s;
  const int near = max(0, s.p_lo - a.window + 1);
  s.nb0 = near >> 5;
  s.ns = min(s.nb0, (min(a.sinks, near) + 31) >> 5);
  // Tokens past the table are held nowhere.
  const int held = a.cols << (a.page_shift - 5);
  const int end = min((s.p_hi >> 5) + 1, held);
  s.ns = min(s.ns, held);
  s.total = s.ns + max(0, end - s.nb0);
  return s;
}

// Row tile `unit`'s chunks of `chunk` blocks are those from `first` on, `count` of them
// (stored for the join behind the partial results).
struct Share {
  int32_t unit, first, count, chunk;
};

constexpr int kMaxUnits = 256;   // row tiles that are dealt out by their lengths

// The share that chunk `index` belongs to; unit < 0 if there is none.  Every wave of
// every workgroup computes the same from the lengths: chunks of a size that makes at
// most `target` of them for all heads.
__device__ __forceinline__ Share find_share(const AttnParams& a, int tile_rows, int index) {
  if (a.target == 0) return Share{index < a.units ? index : -1, index, 1, kMaxLen};
  constexpr int kPasses = kMaxUnits / 64;
  const int lane = threadIdx.x & 63;
  int total[kPasses], sum = 0;   // a sum of 256 x 2^25 blocks, in units of 8
#pragma unroll
  for (int i = 0; i < kPasses; ++i) {
    const int u = 64 * i + lane;
    total[i] = 0;
    if (64 * i < a.units && u < a.units)
      total[i] = span_of(a, u / a.tiles, u % a.tiles * tile_rows, tile_rows).total;
    sum += (total[i] + 7) >> 3;
  }
  const int64_t blocks = static_cast<int64_t>(wave_total(sum)) * 8 * a.H;
  auto count_of = [&](int i, int chunk) __attribute__((always_inline)) {
    return 64 * i + lane < a.units ? max(1, (total[i] + chunk - 1) / chunk) : 0;
  };
  auto chunk_for = [&](int parts) __attribute__((always_inline)) {
    return (max(static_cast<int>((blocks + parts - 1) / parts), a.least) + 7) & ~7;
  };
  // As many blocks per chunk as fill `target`, unless the row tiles' last chunks make
  // more of them; the second size cannot (each row tile adds less than one).
  int chunk = chunk_for(a.target), chunks = 0;
#pragma unroll
  for (int i = 0; i < kPasses; ++i) chunks += count_of(i, chunk);
  if (static_cast<int64_t>(wave_total(chunks)) * a.H > a.target)
    chunk = chunk_for(a.target - a.units * a.H);
  int before = 0;
#pragma unroll
  for (int i = 0; i < kPasses; ++i) {
    if (64 * i >= a.units) break;
    const int count = count_of(i, chunk), incl = wave_incl_scan(count);
    const int first = before + incl - count;
    const uint64_t at = __ballot(index >= first && index < first + count);
    if (at) {
      const int l = __builtin_ctzll(at);
      return Share{64 * i + l, __builtin_amdgcn_readlane(first, l),
                   __builtin_amdgcn_readlane(count, l), chunk};
    }
    before += __builtin_amdgcn_readlane(incl, 63);
  }
  return Share{-1, 0, 0, 0};
}

__device__ __forceinline__ int2* shares_of(const AttnParams& a, int tile_rows, int D) {
  return reinterpret_cast<int2*>(a.part + static_cast<int64_t>(a.items) * tile_rows * (D + 2));
}

// How a call is dealt out; depends on its shapes alone, so that the workspace
// query and the launch agree.
struct Deal {
  bool many, half;   // which kernel takes it
  int32_t R, W, rows, tiles, target, least;
  int64_t units, items;
  bool merge;
};

// The kernel of many rows: 32 of them per wave, four or eight waves.
hipError_t launch_cache_chunk(const AttnParams& a, int32_t D, int32_t bits, int32_t waves,
                              int64_t items, hipStream_t stream);

}  // namespace vecattn
