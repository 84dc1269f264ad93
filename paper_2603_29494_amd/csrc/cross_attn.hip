// Attention over an encoder's states: every row of q sees the same keys of its
// sequence, those below its length that the mask leaves.
//
// The query heads that share a key/value head are rows beside each other (row = token *
// group + head), so that one token's heads read K and V once.  The matrix products are
// v_mfma_f32_32x32x16_bf16, S^T = K Q^T and O^T += V^T P^T, with a row's softmax state in
// its two lanes; K and V go from memory straight to LDS with the swizzle of
// device_common.h, and V is read back transposed.  Rows of masked keys of V are fetched
// from past the buffer's end, which reads 0: what such a key holds never meets a
// product, and its score is set to -inf.  The weights are rounded to bf16 (off by 2^-8 of a
// weight at most) before they meet V, as the operands are; their sum is of what was not
// rounded.  Up to 16 rows stand in the products' 32 columns twice, and a weight in two bf16
// numbers that add up to it (2^-16), which takes no more products.  Of more rows the second half
// would: 75600 rows of 40 heads over 512 keys 1138 us in place of 860, 4096 over 4096 keys 190
// in place of 135.
//
// Two kernels.  Of more than 32 rows, a workgroup owns 128 of them (a wave 32) and its
// waves share tiles of 32 keys.  Of up to 32, each of four waves takes tiles of 32 keys
// of its own, without barriers, and the waves' sums are joined at the end.  Where the
// rows alone do not fill the chip, the keys are cut into chunks, and a second kernel
// joins the chunks of a row.
//
// Many rows are bound by the matrix products and the exponentials beside them: 75600 rows
// of 40 heads of 128 over 512 keys take 864 us at best, 917 TFLOP/s with the first fetches
// and the last stores of each workgroup, which nothing of its own overlaps (1.24 to 1.29
// PFLOP/s over long keys).  Few rows by reading K and V: one token of 28 heads over 16
// sequences of up to 16384 keys, 4 heads of 128: 45 us (4.4 TB/s of the visible keys) and 5
// for the join.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "device_common.h"
#include "launch.h"
#include "wave_scan.h"

namespace vecattn {
namespace {

constexpr float kUnseen = -3.4028234663852886e38f;   // reference of a row that has met no key
constexpr float kLn2 = 0.69314718055994531f;

struct CrossParams {
  const uint16_t *q, *k, *v;
  int64_t q_sB, q_sH, q_sN, k_sB, k_sH, k_sN, v_sB, v_sH, v_sN;
  uint16_t* o;
  int64_t o_sB, o_sH, o_sN;
  float* lse;
  const int32_t* lens;
  const uint8_t* mask;
  int64_t mask_sB;
  const int32_t* n_q;
  int32_t clear;       // rows past n_q become 0
  float* part;         // [item][rows of a tile][D] sums, then [item][rows of a tile] (m, l)
  int32_t Hkv, group, Nq, Nk, row_tiles, chunks, chunk, batch;
  int32_t target, least;     // of few rows: most chunks, of all heads (0: one each); their tiles
  uint32_t items;
  float scale_log2;
};

typedef const __attribute__((address_space(4))) int32_t* ScalarInts;

struct Item {
  int64_t b, index;
  int hk, rt, c, len, rows, count;   // keys and rows that exist, chunks of the sequence
};

__device__ __forceinline__ int chunks_of(const CrossParams& a, int len) {
  return max(1, (len + a.chunk - 1) / a.chunk);
}
__device__ __forceinline__ int keys_of(const CrossParams& a, int64_t b) {
  return a.lens ? min(max(((ScalarInts)a.lens)[b], 0), a.Nk) : a.Nk;
}
__device__ __forceinline__ int rows_of(const CrossParams& a, int64_t b) {
  return (a.n_q ? min(max(((ScalarInts)a.n_q)[b], 0), a.Nq) : a.Nq) * a.group;
}

// Item i: sequence and key/value head, then row tile, then chunk; false where it has no rows
// or no keys to take.  Workgroups take items as the hardware deals them out, beside each
// other to the eight XCDs, so that these read rows that lie near each other (75600 rows of 40
// heads over 512 keys: 864 us; 888 with a range of heads for each XCD).
__device__ __forceinline__ bool decode(const CrossParams& a, int tile_rows, uint32_t i, Item& s) {
  const uint32_t rest = i / static_cast<uint32_t>(a.chunks);
  const uint32_t bh = rest / static_cast<uint32_t>(a.row_tiles);
  const uint32_t b = bh / static_cast<uint32_t>(a.Hkv);
  s.index = i;
  s.c = static_cast<int>(i - rest * a.chunks);
  s.rt = static_cast<int>(rest - bh * a.row_tiles);
  s.hk = static_cast<int>(bh - b * a.Hkv);
  s.b = b;
  s.len = keys_of(a, s.b);
  s.rows = rows_of(a, s.b);
  s.count = chunks_of(a, s.len);
  return s.rt * tile_rows < s.rows && s.c < s.count;
}

// Few rows: the chunks, of `tiles` tiles of kFewKeys, that a sequence's keys are cut into.
constexpr int kFewKeys = 32, kMaxDealt = 256;   // sequences that are dealt out by their lengths
struct Share {
  int b, first, count, tiles;
};

// The share that chunk `index` belongs to; b < 0 if there is none.  Every wave of every
// workgroup computes the same from the lengths: chunks of a size that makes at most
// `target` of them for all heads.
__device__ __forceinline__ Share find_share(const CrossParams& a, int index) {
  if (a.target == 0) return Share{index < a.batch ? index : -1, index, 1, a.Nk};
  constexpr int kPasses = kMaxDealt / 64;
  const int lane = threadIdx.x & 63;
  int total[kPasses], sum = 0;
#pragma unroll
  for (int i = 0; i < kPasses; ++i) {
    const int b = 64 * i + lane;
    total[i] = 64 * i < a.batch && b < a.batch ? (keys_of(a, b) + kFewKeys - 1) / kFewKeys : 0;
    sum += (total[i] + 7) >> 3;   // 256 x 2^25 tiles, in units of 8
  }
  const int64_t tiles = static_cast<int64_t>(wave_total(sum)) * 8 * a.Hkv;
  // Chunks of a multiple of four tiles, one for each wave at a time.
  auto size_for = [&](int parts) __attribute__((always_inline)) {
    return (max(static_cast<int>((tiles + parts - 1) / parts), a.least) + 3) & ~3;
  };
  auto count_of = [&](int i, int size) __attribute__((always_inline)) {
    return 64 * i + lane < a.batch ? max(1, (total[i] + size - 1) / size) : 0;
  };
  // As many tiles per chunk as fill `target`, unless the sequences' last chunks make more of
  // them; the second size cannot (each sequence adds less than one).
  int size = size_for(a.target), chunks = 0;
#pragma unroll
  for (int i = 0; i < kPasses; ++i) chunks += count_of(i, size);
  if (static_cast<int64_t>(wave_total(chunks)) * a.Hkv > a.target)
    size = size_for(a.target - a.batch * a.Hkv);
  int before = 0;
#pragma unroll
  for (int i = 0; i < kPasses; ++i) {
    if (64 * i >= a.batch) break;
    const int count = count_of(i, size), incl = wave_incl_scan(count);
    const int first = before + incl - count;
    const uint64_t at = __ballot(index >= first && index < first + count);
    if (at) {
      const int l = __builtin_ctzll(at);
      return Share{64 * i + l, __builtin_amdgcn_readlane(first, l),
                   __builtin_amdgcn_readlane(count, l), size};
    }
    before += __builtin_amdgcn_readlane(incl, 63);
  }
  return Share{-1, 0, 0, 0};
}

// Where a sequence's share is left for the join, behind the parts.
template <int D>
__device__ __forceinline__ int2* shares_of(const CrossParams& a) {
  return reinterpret_cast<int2*>(a.part + static_cast<int64_t>(a.items) * 32 * (D + 2));
}

__device__ __forceinline__ const uint16_t* q_row(const CrossParams& a, const Item& s, int row) {
  const int tok = row / a.group, h = s.hk * a.group + row % a.group;
  return a.q + s.b * a.q_sB + h * a.q_sH + tok * a.q_sN;
}
__device__ __forceinline__ uint16_t* o_row(const CrossParams& a, int64_t b, int hk, int row) {
  const int tok = row / a.group, h = hk * a.group + row % a.group;
  return a.o + b * a.o_sB + h * a.o_sH + tok * a.o_sN;
}
__device__ __forceinline__ void put_lse(const CrossParams& a, int64_t b, int hk, int row, float m,
                                        float l) {
  if (!a.lse) return;
  const int tok = row / a.group, h = hk * a.group + row % a.group;
  a.lse[(b * a.Hkv * a.group + h) * a.Nq + tok] =
      l == 0.0f ? kNegInf : (m + __builtin_log2f(l)) * kLn2;
}

// The rows of an item's tile that do not exist, where they become 0.
template <int D>
__device__ __forceinline__ void clear_rows(const CrossParams& a, const Item& s, int tile_rows) {
  if (!a.clear || s.c > 0) return;
  const int first = max(s.rows, s.rt * tile_rows);
  const int count = min((s.rt + 1) * tile_rows, a.Nq * a.group) - first;
  for (int i = threadIdx.x; i < count * (D / 8); i += blockDim.x) {
    const int row = first + i / (D / 8);
    reinterpret_cast<u32x4*>(o_row(a, s.b, s.hk, row))[i % (D / 8)] = u32x4{0, 0, 0, 0};
    if (a.lse && i % (D / 8) == 0) {
      const int tok = row / a.group, h = s.hk * a.group + row % a.group;
      a.lse[(s.b * a.Hkv * a.group + h) * a.Nq + tok] = 0.0f;
    }
  }
}

// Direct-to-LDS instruction u of a tile of KEYS rows from row j0 on (16 bytes a lane).  HIDE:
// rows that are not visible read 0; rows past `keys` do so always.
// col: 16 times the lane's chunk, swizzled for the instruction's first row; row: its row of the
// instruction's times rowb.
template <int D>
__device__ __forceinline__ uint32_t gather_col(int lane) {
  constexpr int CH = D / 8;
  return 16u * ((lane % CH) ^ swz<D>(lane / CH));
}
template <int D, int KEYS, bool HIDE>
__device__ __forceinline__ void gather(const uint16_t* base, uint32_t rowb, int j0, int keys, int u,
                                       int lane, uint32_t col, uint32_t row, uint64_t see,
                                       uint16_t* dst) {
  constexpr int CH = D / 8, R = 64 / CH;   // rows of an instruction
  const int n = min(KEYS, keys - j0);
  const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(
      const_cast<char*>(reinterpret_cast<const char*>(base) + static_cast<int64_t>(j0) * rowb), 0,
      n > 0 ? (n - 1) * rowb + 2 * D : 0, 0x00020000);
  // Row u R + lane / CH, whose swizzle is its parts' exclusive or.
  uint32_t at = (col ^ (16u * swz<D>(u * R))) + row + u * R * rowb;
  if constexpr (HIDE) at = static_cast<uint32_t>(see >> (u * R)) >> (lane / CH) & 1 ? at : 0x80000000u;
  gather16_to_lds(rs, at, dst + u * 64 * 8);
}

// x, not known to be the same as before: what follows from it is computed where it is used.
// Held over the walk, the operands' addresses would not fit the registers.
__device__ __forceinline__ uint32_t fresh(uint32_t x) {
  asm volatile("" : "+v"(x));
  return x;
}

// One wave's 32 rows against 32 keys at a time; TWICE: 16 rows, each with a weight's rounding to
// bf16 in one column of the products and the rounding of what that leaves in the other, 16 on.
template <int D, bool TWICE>
struct Wave {
  static constexpr int DS = D / 16, DB = D / 32, RB = 2 * D;
  bf16x8 qf[DS];
  f32x16 oacc[DB];
  float m_run, l_run;
  uint32_t kat, vat;   // where the lane's operands lie: of K's first values, of V's first keys
  int g, ln;
  float second;        // 1 in the columns of the weights' second parts

  __device__ __forceinline__ void clear() {
    m_run = kUnseen;
    l_run = 0.0f;
#pragma unroll
    for (int db = 0; db < DB; ++db) oacc[db] = f32x16{};
  }
  __device__ __forceinline__ void start(int lane) {
    g = lane >> 5, ln = lane & 31;
    second = TWICE && (ln & 16) ? 1.0f : 0.0f;
    clear();
    kat = ln * RB + 16 * (g ^ swz<D>(ln));
    const int j16 = lane & 15, tq = j16 >> 2, tp = j16 & 3, vhalf = (lane >> 4) & 1;
    const int k0 = 4 * g + tq;
    vat = k0 * RB + 16 * ((2 * vhalf + (tp >> 1)) ^ swz<D>(k0)) + 8 * (tp & 1);
  }
  __device__ __forceinline__ void load(const uint16_t* row, bool have) {
#pragma unroll
    for (int s = 0; s < DS; ++s) {
      u32x4 t = {0, 0, 0, 0};
      if (have) t = reinterpret_cast<const u32x4*>(row)[2 * s + g];
      qf[s] = __builtin_bit_cast(bf16x8, t);
    }
  }
  // Values 16 i .. + 15 of K (its chunk 2 i + g, swizzled).
  __device__ __forceinline__ i16x8 kread(int i, const uint16_t* k, uint32_t at) {
    return *reinterpret_cast<const i16x8*>(reinterpret_cast<const char*>(k) + (at ^ (32 * i)));
  }
  // Operands are read kAhead instructions ahead of their use, in a fixed order: the
  // compiler would read all of them first, which the registers have no room for.
  static constexpr int kAhead = 3;
  __device__ __forceinline__ void score(f32x16& s, const uint16_t* k) {
    const uint32_t at = kat;
    i16x8 ring[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) ring[i] = kread(i, k, at);
    s = f32x16{};
#pragma unroll
    for (int i = 0; i < DS; ++i) {
      __builtin_amdgcn_sched_barrier(0);
      s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, ring[i % kAhead]), qf[i],
                                                  s, 0, 0, 0);
      if (i + kAhead < DS) ring[i % kAhead] = kread(i + kAhead, k, at);
    }
    __builtin_amdgcn_sched_barrier(0);
  }
  // Element e of a lane is key 8 (e / 4) + 4 g + e % 4: a bit of either half of the wave, put
  // together on the scalar side.
  __device__ __forceinline__ void hide(f32x16& s, uint32_t see) {
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const int j = 8 * (e / 4) + e % 4;
      const uint32_t lo = static_cast<int32_t>(see << (31 - j)) >> 31;
      const uint32_t hi = static_cast<int32_t>(see << (27 - j)) >> 31;
      const bool there = __builtin_amdgcn_inverse_ballot_w64(uint64_t(hi) << 32 | lo);
      s[e] = there ? s[e] : kNegInf;
    }
  }
  static __device__ __forceinline__ float largest(const f32x16& s) {
    float top = kNegInf;
#pragma unroll
    for (int e = 0; e < 16; ++e) top = fmaxf(top, s[e]);
    return top;
  }
  // The sums times alpha.  In place by force: of products of its own on a rare branch the
  // compiler makes a second set of registers for O, and copies one to the other on the
  // common way.  It does not see what the instructions read and write: they wait for the
  // matrix instructions before them, and those after them wait for them, by themselves
  // (a 32x32x16 product's result can be read after 18 cycles).
  __device__ __forceinline__ void rescale(float alpha) {
    l_run *= alpha;
    asm volatile("s_nop 15\n\ts_nop 15");
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        float x = oacc[db][e];
        asm volatile("v_mul_f32_e32 %0, %1, %0" : "+v"(x) : "v"(alpha));
        oacc[db][e] = x;
      }
    asm volatile("s_nop 7");
  }
  // The weights against the reference as it is; a row whose sum is past 256 on one of its
  // lanes moves its reference first.
  __device__ __forceinline__ void weigh(const f32x16& s, float scale_log2, bf16x8 (&pb)[2]) {
    float sum;
    auto weights = [&]() __attribute__((always_inline)) {
      float part[2];
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        f32x8 y;
#pragma unroll
        for (int e = 0; e < 8; ++e)
          y[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[8 * x + e], scale_log2, -m_run));
        part[x] = ((y[0] + y[1]) + (y[2] + y[3])) + ((y[4] + y[5]) + (y[6] + y[7]));
        pb[x] = __builtin_convertvector(y, bf16x8);
        if constexpr (TWICE) {   // in the second columns what that leaves
          const f32x8 first = __builtin_convertvector(pb[x], f32x8);
#pragma unroll
          for (int e = 0; e < 8; ++e) y[e] = __builtin_fmaf(-first[e], second, y[e]);
          pb[x] = __builtin_convertvector(y, bf16x8);
        }
      }
      sum = part[0] + part[1];
    };
    weights();
    if (__any(sum > 256.0f)) {
      const bool up = wave_max_xor32(sum) > 256.0f;   // no row depends on its neighbours
      const float m_new = up ? fmaxf(m_run, wave_max_xor32(largest(s)) * scale_log2) : m_run;
      rescale(__builtin_amdgcn_exp2f(m_run - m_new));
      m_run = m_new;
      weights();
    }
    l_run += sum;
  }
  // Values 32 db .. + 31 of keys 16 ks .. + 15 of V, transposed.
  __device__ __forceinline__ i16x8 vread(int ks, int db, const uint16_t* v, uint32_t at) {
    const char* vb = reinterpret_cast<const char*>(v) + 16 * ks * RB;  // the swizzle repeats
    const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS_PTR(i16x4, vb + (at ^ (64 * db))));
    const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
        LDS_PTR(i16x4, vb + (at ^ (64 * db + 32)) + 8 * RB));   // eight keys on
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  }
  __device__ __forceinline__ void add(const bf16x8 (&pb)[2], const uint16_t* v) {
    const uint32_t at = vat;
    constexpr int N = 2 * DB;
    i16x8 ring[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) ring[i] = vread(i / DB, i % DB, v, at);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      __builtin_amdgcn_sched_barrier(0);
      oacc[i % DB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
          __builtin_bit_cast(bf16x8, ring[i % kAhead]), pb[i / DB], oacc[i % DB], 0, 0, 0);
      if (i + kAhead < N) ring[i % kAhead] = vread((i + kAhead) / DB, (i + kAhead) % DB, v, at);
    }
    __builtin_amdgcn_sched_barrier(0);
  }
};

// Sums of a row to where they go: o, or the chunk's part.  y: four values from d on.
template <int D>
__device__ __forceinline__ void put_part(const CrossParams& a, const Item& s, int tile_rows, int r,
                                         int d, f32x4 y) {
  *reinterpret_cast<f32x4*>(a.part + (s.index * tile_rows + r) * D + d) = y;
}
template <int D>
__device__ __forceinline__ float* part_ml(const CrossParams& a, int64_t index, int tile_rows, int r) {
  return a.part + static_cast<int64_t>(a.items) * tile_rows * D + (index * tile_rows + r) * 2;
}

// Many rows.  Tiles of 32 keys in three stages, one barrier each: a tile is fetched while
// the two before it are worked on.
template <int D, bool MASK>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(D == 128 ? 3 : 4))) void k_cross_many(
    const CrossParams a) {
  constexpr int KEYS = 32, U = KEYS * (D / 8) / 256;   // direct loads per wave and matrix
  using W = Wave<D, false>;
  constexpr int DB = W::DB;
  __shared__ __align__(16) uint16_t k_s0[KEYS * D];
  __shared__ __align__(16) uint16_t k_s1[KEYS * D];
  __shared__ __align__(16) uint16_t k_s2[KEYS * D];
  __shared__ __align__(16) uint16_t v_s0[KEYS * D];
  __shared__ __align__(16) uint16_t v_s1[KEYS * D];
  __shared__ __align__(16) uint16_t v_s2[KEYS * D];
  Item s;
  const bool some = decode(a, kCrossRows, blockIdx.x, s);
  clear_rows<D>(a, s, kCrossRows);
  if (!some) return;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int first = s.c * a.chunk, keys = min(s.len - first, a.chunk);
  const uint16_t* kh = a.k + s.b * a.k_sB + s.hk * a.k_sH + first * a.k_sN;
  const uint16_t* vh = a.v + s.b * a.v_sB + s.hk * a.v_sH + first * a.v_sN;
  const uint32_t k_rowb = static_cast<uint32_t>(a.k_sN) * 2u;
  const uint32_t v_rowb = static_cast<uint32_t>(a.v_sN) * 2u;
  const uint32_t col = gather_col<D>(lane), k_row = lane / (D / 8) * k_rowb,
                 v_row = lane / (D / 8) * v_rowb;
  const uint8_t* mask = MASK ? a.mask + s.b * a.mask_sB + first : nullptr;
  const int ntiles = (keys + KEYS - 1) / KEYS;

  auto fetch = [&](int t, uint32_t see, uint16_t* k, uint16_t* v) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < U; ++u)
      gather<D, KEYS, false>(kh, k_rowb, t * KEYS, keys, wave * U + u, lane, col, k_row, see, k);
#pragma unroll
    for (int u = 0; u < U; ++u)
      gather<D, KEYS, MASK>(vh, v_rowb, t * KEYS, keys, wave * U + u, lane, col, v_row, see, v);
  };
  // Visible keys of a tile; with a mask from its bytes, fetched a tile earlier.
  auto key_byte = [&](int t) __attribute__((always_inline)) {
    const int j = t * KEYS + (lane & 31);
    return MASK && j < keys ? mask[j] : 0;
  };
  auto visible = [&](int t, int byte) __attribute__((always_inline)) {
    if constexpr (MASK) {
      asm volatile("" : "+v"(byte));   // compared here, not where it is fetched
      return static_cast<uint32_t>(__ballot(byte != 0));
    }
    const int n = keys - t * KEYS;
    return n >= 32 ? ~0u : n <= 0 ? 0u : (1u << n) - 1u;
  };
  const int row = s.rt * kCrossRows + 32 * wave + (lane & 31);
  const bool have = row < s.rows;
  W w;
  w.start(lane);
  // Visible keys of the tile that is worked on and the two after it, the last as it came.
  uint32_t see = 0, see1 = 0;
  int byte2 = 0;
  if (ntiles > 0) {
    const int b0 = key_byte(0), b1 = key_byte(1);
    byte2 = key_byte(2);
    see = visible(0, b0), see1 = visible(1, b1);
    fetch(0, see, k_s0, v_s0);
    w.load(q_row(a, s, have ? row : 0), have);
    if (ntiles > 1) fetch(1, see1, k_s1, v_s1);
  }
  bool settled = false;
  auto turn = [&](int t, const uint16_t* k, const uint16_t* v, uint16_t* k2, uint16_t* v2)
                  __attribute__((always_inline)) {
    // Tile t is there, and every wave is through with the one whose stage is filled again.
    if (t + 1 < ntiles) wait_vmcnt<2 * U>();
    else wait_all();
    __builtin_amdgcn_s_barrier();
    const uint32_t see2 = visible(t + 2, byte2);
    byte2 = key_byte(t + 3);
    if (t + 2 < ntiles) fetch(t + 2, see2, k2, v2);
    f32x16 x;
    bf16x8 pb[2];
    w.score(x, k);
    if (see != ~0u) w.hide(x, see);
    if (!settled) {   // the first keys of which one is visible, the same for all rows
      w.m_run = fmaxf(w.m_run, wave_max_xor32(W::largest(x)) * a.scale_log2);
      settled = see != 0;
    }
    w.weigh(x, a.scale_log2, pb);
    w.add(pb, v);
    see = see1, see1 = see2;
  };
  for (int t = 0; t < ntiles; t += 3) {
    turn(t, k_s0, v_s0, k_s2, v_s2);
    if (t + 1 < ntiles) turn(t + 1, k_s1, v_s1, k_s0, v_s0);
    if (t + 2 < ntiles) turn(t + 2, k_s2, v_s2, k_s1, v_s1);
  }

  const float l = w.l_run + __shfl_xor(w.l_run, 32);
  if (s.count > 1) {
    if (!have) return;
    const int r = 32 * wave + w.ln;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int vq = 0; vq < 4; ++vq) {
        f32x4 y;
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = w.oacc[db][4 * vq + e];
        put_part<D>(a, s, kCrossRows, r, 32 * db + 8 * vq + 4 * w.g, y);
      }
    if (w.g == 0) {
      float* ml = part_ml<D>(a, s.index, kCrossRows, r);
      ml[0] = w.m_run, ml[1] = l;
    }
    return;
  }
  const float inv = l > 0.0f ? 1.0f / l : l;   // no key: 0; NaN stays
  if (have && w.g == 0) put_lse(a, s.b, s.hk, row, w.m_run, l);
  uint16_t* orow = o_row(a, s.b, s.hk, have ? row : 0);
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      // A lane of a row holds four values of every eight: after a swap, eight of every
      // sixteen.
      u32x2 y[2];
#pragma unroll
      for (int vq = 0; vq < 2; ++vq) {
        f32x4 z;
#pragma unroll
        for (int e = 0; e < 4; ++e) z[e] = w.oacc[db][8 * x + 4 * vq + e] * inv;
        y[vq] = __builtin_bit_cast(u32x2, __builtin_convertvector(z, bf16x4));
      }
      const auto lo = __builtin_amdgcn_permlane32_swap(y[0][0], y[1][0], false, false);
      const auto hi = __builtin_amdgcn_permlane32_swap(y[0][1], y[1][1], false, false);
      if (have)
        *reinterpret_cast<u32x4*>(orow + 32 * db + 16 * x + 8 * w.g) =
            u32x4{lo[0], hi[0], lo[1], hi[1]};
    }
}

// Few rows; TWICE: up to 16, each in two columns of the products (weights in two parts).  What it
// adds are the instructions that take a weight apart: nothing where K and V come from memory (one
// token of 28 heads over 16 x 16384 keys 48 us with or without), 3% of 12 heads over 257 keys (7.0
// and 6.8), 7% where they come from the caches (256 heads of 64 over 4000 keys 29.9 and 27.8).
// Products of their own would take as much more.
template <int D, bool TWICE>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(1))) void k_cross_few(
    const CrossParams a) {
  constexpr int KEYS = kFewKeys, U = KEYS * (D / 8) / 64, ROWS = 32;
  using W = Wave<D, TWICE>;
  __shared__ __align__(16) uint16_t k_s0[4][KEYS * D];
  __shared__ __align__(16) uint16_t k_s1[4][KEYS * D];
  __shared__ __align__(16) uint16_t v_s0[4][KEYS * D];
  __shared__ __align__(16) uint16_t v_s1[4][KEYS * D];
  __shared__ float s_m[4][ROWS], s_l[4][ROWS];
  const uint32_t chunk = blockIdx.x / static_cast<uint32_t>(a.Hkv);
  const Share share = find_share(a, static_cast<int>(chunk));
  if (share.b < 0) return;
  Item s;
  s.index = blockIdx.x;
  s.b = share.b;
  s.hk = static_cast<int>(blockIdx.x - chunk * a.Hkv);
  s.rt = 0;
  s.c = static_cast<int>(chunk) - share.first;
  s.count = share.count;
  s.len = keys_of(a, s.b);
  s.rows = rows_of(a, s.b);
  if (a.target && s.c == 0 && s.hk == 0 && threadIdx.x == 0)
    shares_of<D>(a)[s.b] = int2{share.first, share.count};
  clear_rows<D>(a, s, ROWS);
  if (s.rows == 0) return;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int first = s.count > 1 ? s.c * share.tiles * KEYS : 0;
  const int keys = s.count > 1 ? min(s.len - first, share.tiles * KEYS) : s.len;
  const uint16_t* kh = a.k + s.b * a.k_sB + s.hk * a.k_sH + first * a.k_sN;
  const uint16_t* vh = a.v + s.b * a.v_sB + s.hk * a.v_sH + first * a.v_sN;
  const uint32_t k_rowb = static_cast<uint32_t>(a.k_sN) * 2u;
  const uint32_t v_rowb = static_cast<uint32_t>(a.v_sN) * 2u;
  const uint32_t col = gather_col<D>(lane), k_row = lane / (D / 8) * k_rowb,
                 v_row = lane / (D / 8) * v_rowb;
  const uint8_t* mask = a.mask ? a.mask + s.b * a.mask_sB + first : nullptr;
  const int ntiles = (keys + KEYS - 1) / KEYS;
  const int row = lane & (TWICE ? 15 : 31);
  const bool have = row < s.rows;
  W w;
  w.start(lane);
  w.load(q_row(a, s, have ? row : 0), have);

  auto fetch = [&](int t, uint64_t see, uint16_t* k, uint16_t* v) __attribute__((always_inline)) {
    const int j0 = t * KEYS;
#pragma unroll
    for (int u = 0; u < U; ++u) gather<D, KEYS, false>(kh, k_rowb, j0, keys, u, lane, col, k_row, see, k);
#pragma unroll
    for (int u = 0; u < U; ++u) gather<D, KEYS, true>(vh, v_rowb, j0, keys, u, lane, col, v_row, see, v);
  };
  // A tile is worked on while the wave's next is fetched; past the last one the fetch
  // goes to the last again (into a buffer that nothing reads).
  auto tile = [&](int t) __attribute__((always_inline)) { return min(t, ntiles - 1); };
  // Visible keys of the tile that is worked on and of the next; of the one after that the
  // lane's byte, fetched before the next tile's keys, so that it does not wait for them.
  auto key_byte = [&](int t) __attribute__((always_inline)) {
    const int j = t * KEYS + (lane & 31);
    return j < keys ? (mask ? mask[j] : 1) : 0;
  };
  auto bits = [&](int byte) __attribute__((always_inline)) {
    asm volatile("" : "+v"(byte));   // compared here, not where it is fetched
    return static_cast<uint32_t>(__ballot(byte != 0));
  };
  int t = wave;
  uint32_t see = 0, see1 = 0;
  if (t < ntiles) {
    const int b0 = key_byte(t), b1 = key_byte(tile(t + 4));
    see = bits(b0), see1 = bits(b1);
    fetch(t, see, k_s0[wave], v_s0[wave]);
  }
  bool settled = false;
  auto turn = [&](const uint16_t* k, const uint16_t* v, uint16_t* k1, uint16_t* v1)
                  __attribute__((always_inline)) {
    const int byte2 = key_byte(tile(t + 8));
    fetch(tile(t + 4), see1, k1, v1);
    wait_vmcnt<2 * U>();
    f32x16 x;
    bf16x8 pb[2];
    w.score(x, k);
    if (see != ~0u) w.hide(x, see);
    if (!settled) {   // the first keys of which one is visible, the same for all rows
      w.m_run = fmaxf(w.m_run, wave_max_xor32(W::largest(x)) * a.scale_log2);
      settled = see != 0;
    }
    w.weigh(x, a.scale_log2, pb);
    w.add(pb, v);
    see = see1, see1 = bits(byte2);
    t += 4;
  };
  while (t < ntiles) {
    turn(k_s0[wave], v_s0[wave], k_s1[wave], v_s1[wave]);
    if (t >= ntiles) break;
    turn(k_s1[wave], v_s1[wave], k_s0[wave], v_s0[wave]);
  }
  wait_all();

  // Join the waves: each scales its sums to the largest reference.
  w.l_run += __shfl_xor(w.l_run, 32);
  if (w.g == 0) s_m[wave][w.ln] = w.m_run;
  __syncthreads();
  float m = kUnseen;
#pragma unroll
  for (int i = 0; i < 4; ++i) m = fmaxf(m, s_m[i][w.ln]);
  const float alpha = __builtin_amdgcn_exp2f(w.m_run - m);
  if (w.g == 0) s_l[wave][w.ln] = w.l_run * alpha;
  // Their sums go through LDS one wave after the other, over V's first stage.
  constexpr int kSo = D + 4;
  static_assert(sizeof(v_s0) >= ROWS * kSo * sizeof(float), "the sums of a tile fit a stage");
  float* buf = reinterpret_cast<float*>(v_s0);
  __syncthreads();
#pragma unroll 1
  for (int i = 3; i >= 0; --i) {
    if (wave == i) {
#pragma unroll
      for (int db = 0; db < W::DB; ++db)
#pragma unroll
        for (int vq = 0; vq < 4; ++vq) {
          const int d = 32 * db + 8 * vq + 4 * w.g;
          float* at = buf + w.ln * kSo + d;
          f32x4 y;
#pragma unroll
          for (int e = 0; e < 4; ++e) y[e] = w.oacc[db][4 * vq + e] * alpha;
          if (i < 3) y += *reinterpret_cast<const f32x4*>(at);
          *reinterpret_cast<f32x4*>(at) = y;
        }
    }
    __syncthreads();
  }
  // Eight threads a row.
  const int r = threadIdx.x >> 3;
  if (r >= s.rows) return;
  float lr = 0.0f, mr = kUnseen;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    lr += s_l[i][r];
    mr = fmaxf(mr, s_m[i][r]);
  }
  const float inv = s.count > 1 ? 1.0f : lr > 0.0f ? 1.0f / lr : lr;
#pragma unroll
  for (int i = 0; i < D / 32; ++i) {
    const int d = 32 * i + 4 * (threadIdx.x & 7);
    f32x4 y = *reinterpret_cast<const f32x4*>(buf + r * kSo + d);
    if constexpr (TWICE) {
      const f32x4 more = *reinterpret_cast<const f32x4*>(buf + (r + 16) * kSo + d);
#pragma unroll
      for (int e = 0; e < 4; ++e)   // an infinity of V is one of o, whatever the second part makes of it
        y[e] += fabsf(y[e]) < INFINITY ? more[e] : 0.0f;
    }
    if (s.count > 1) {
      put_part<D>(a, s, ROWS, r, d, y);
    } else {
      y *= inv;
      *reinterpret_cast<bf16x4*>(o_row(a, s.b, s.hk, r) + d) = __builtin_convertvector(y, bf16x4);
    }
  }
  if ((threadIdx.x & 7) == 0) {
    if (s.count > 1) {
      float* ml = part_ml<D>(a, s.index, ROWS, r);
      ml[0] = mr, ml[1] = lr;
    } else {
      put_lse(a, s.b, s.hk, r, mr, lr);
    }
  }
}

// Joins the chunks of a row, a wave per row, a lane D / 64 values.
template <int D, bool FEW>
__global__ __launch_bounds__(256) void k_cross_merge(const CrossParams a, int32_t tile_rows,
                                                     int64_t total) {
  constexpr int V = D / 64;
  const int lane = threadIdx.x & 63;
  const int64_t id = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6);
  if (id >= total) return;
  const int rows_all = a.Nq * a.group;
  const int row = static_cast<int>(id % rows_all);
  const int64_t bh = id / rows_all;
  const int hk = static_cast<int>(bh % a.Hkv);
  const int64_t b = bh / a.Hkv;
  // The row's parts: every `step`-th row of them from the first on.
  int count;
  int64_t at, step;
  if constexpr (FEW) {
    const int2 share = shares_of<D>(a)[b];   // first, count
    count = share.y;
    at = static_cast<int64_t>(share.x) * a.Hkv + hk;
    step = static_cast<int64_t>(a.Hkv) * tile_rows;
  } else {
    count = chunks_of(a, keys_of(a, b));
    at = (bh * a.row_tiles + row / tile_rows) * a.chunks;
    step = tile_rows;
  }
  if (count <= 1 || row >= rows_of(a, b)) return;
  const int r = row % tile_rows;
  const float* ml = part_ml<D>(a, at, tile_rows, r);
  const float* src = a.part + (at * tile_rows + r) * D + V * lane;
  float m = kUnseen;
  for (int i = lane; i < count; i += 64) m = fmaxf(m, ml[i * step * 2]);
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) m = fmaxf(m, __shfl_xor(m, o));
  float l = 0.0f, y[V] = {};
#pragma unroll 4
  for (int i = 0; i < count; ++i) {
    const float alpha = __builtin_amdgcn_exp2f(ml[i * step * 2] - m);
    l = __builtin_fmaf(ml[i * step * 2 + 1], alpha, l);
#pragma unroll
    for (int x = 0; x < V; ++x) y[x] = __builtin_fmaf(src[i * step * D + x], alpha, y[x]);
  }
  const float inv = l > 0.0f ? 1.0f / l : l;
  __bf16* orow = reinterpret_cast<__bf16*>(o_row(a, b, hk, row));
#pragma unroll
  for (int x = 0; x < V; ++x) orow[V * lane + x] = static_cast<__bf16>(y[x] * inv);
  if (lane == 0) put_lse(a, b, hk, row, m, l);
}

// How a call is dealt out; depends on its shapes alone, so that the workspace query and
// the launch agree.
struct Deal {
  bool few;
  int32_t rows, tiles, chunks, chunk, target, least;
  int64_t items;
};

Deal deal(int64_t B, int64_t Hq, int64_t Hkv, int64_t Nq, int64_t Nk, int64_t D) {
  Deal d;
  const int64_t rows = Nq * (Hq / Hkv);
  d.few = rows <= 32;
  d.rows = d.few ? 32 : kCrossRows;
  d.tiles = static_cast<int32_t>((rows + d.rows - 1) / d.rows);
  const int64_t units = B * Hkv * d.tiles;
  d.target = d.least = 0;
  if (d.few) {
    // Cut by the lengths on the device into as many chunks as workgroups run at a time (one
    // of 128 values per CU, two of 64; 16 sequences of 0 to 16384 keys: 45 us, 62 in chunks of
    // 2048), never into fewer than two per head, nor into ones of fewer keys than pay for a
    // chunk.  Up to 1024 keys, or 4096 where heads alone fill the chip, none are cut: the join
    // and what it reads cost more (four heads over 1000 keys: 13 us, 14 cut; 512 over 577
    // of 64 values: 16 and 24; 256 over 4000: 95 and 102; but 64 over 2000 of uneven lengths:
    // 20 and 17).
    const int64_t slots = D == 128 ? 256 : 512, least = 512;
    const int64_t whole = std::min<int64_t>(std::max<int64_t>(16 * units, 1024), 4096);
    const int64_t most = Nk <= whole ? 1 : (Nk + least - 1) / least;
    d.chunks = most > 1 && B <= kMaxDealt ? 2 : 1;   // or more
    d.chunk = 0;
    d.items = units;
    if (d.chunks > 1) {
      d.target = static_cast<int32_t>(std::max(slots, 2 * units));
      d.least = static_cast<int32_t>(least / kFewKeys);
      d.items = std::min<int64_t>(d.target, units * most);
    }
    return d;
  }
  // Many rows: parts and their join cost about as much as 512 keys, so the keys are cut only
  // where row tiles leave half of the CUs without one (8 tiles over 16384 keys: 24 us in 32
  // chunks, 324 in one), or, of many keys, where CUs have very different numbers of them: in
  // three up to one each (130 tiles over 4096 keys: 60 us, 84 in one; 256 over 16384: 351 and
  // 412; but 200 over 4096: 94 and 90), in four up to three for every two CUs (288 over 8192:
  // 170 and 230, 384: 208 and 224; 448: 241 and 239).
  const int64_t balanced = units <= 256 ? 3 : units <= 384 ? 4 : 1;
  const int64_t chunks = units <= 128       ? std::max<int64_t>(1, std::min(Nk / 512, 512 / units))
                         : Nk >= 24 * units ? balanced
                                            : 1;
  d.chunk = static_cast<int32_t>(((Nk + chunks - 1) / chunks + 127) / 128 * 128);
  d.chunks = static_cast<int32_t>((Nk + d.chunk - 1) / d.chunk);
  d.items = units * d.chunks;
  return d;
}

}  // namespace

size_t cross_attn_workspace_bytes(int64_t B, int64_t Hq, int64_t Hkv, int64_t Nq, int64_t Nk,
                                  int64_t D) {
  const Deal d = deal(B, Hq, Hkv, Nq, Nk, D);
  return d.chunks > 1 ? static_cast<size_t>(d.items) * d.rows * (D + 2) * sizeof(float) +
                            (d.few ? static_cast<size_t>(B) * 2 * sizeof(int32_t) : 0)
                      : 0;
}

bool cross_attn_grid_ok(int64_t B, int64_t Hq, int64_t Hkv, int64_t Nq, int64_t Nk, int64_t D) {
  if (Nq * (Hq / Hkv) > (int64_t(1) << 30) || B * Hkv > (int64_t(1) << 24)) return false;
  return deal(B, Hq, Hkv, Nq, Nk, D).items <= (int64_t(1) << 23);
}

hipError_t launch_cross_attn(const CrossArgs& x, hipStream_t stream) {
  const Deal d = deal(x.q.B, x.q.H, x.k.H, x.q.N, x.k.N, x.q.D);
  CrossParams a;
  a.q = static_cast<const uint16_t*>(x.q.ptr);
  a.k = static_cast<const uint16_t*>(x.k.ptr);
  a.v = static_cast<const uint16_t*>(x.v.ptr);
  a.q_sB = x.q.sB, a.q_sH = x.q.sH, a.q_sN = x.q.sN;
  a.k_sB = x.k.sB, a.k_sH = x.k.sH, a.k_sN = x.k.sN;
  a.v_sB = x.v.sB, a.v_sH = x.v.sH, a.v_sN = x.v.sN;
  a.o = static_cast<uint16_t*>(x.o);
  a.o_sB = x.o_sB, a.o_sH = x.o_sH, a.o_sN = x.o_sN;
  a.lse = x.lse;
  a.lens = x.lens;
  a.mask = x.mask, a.mask_sB = x.mask_sB;
  a.n_q = x.n_q;
  a.clear = x.clear && x.n_q;
  a.part = static_cast<float*>(x.workspace);
  a.Hkv = static_cast<int32_t>(x.k.H);
  a.group = static_cast<int32_t>(x.q.H / x.k.H);
  a.Nq = static_cast<int32_t>(x.q.N), a.Nk = static_cast<int32_t>(x.k.N);
  a.row_tiles = d.tiles, a.chunks = d.chunks, a.chunk = d.chunk;
  a.batch = static_cast<int32_t>(x.q.B), a.target = d.target, a.least = d.least;
  a.items = static_cast<uint32_t>(d.items);
  const float scale = x.scale != 0.0f ? x.scale : 1.0f / sqrtf(static_cast<float>(x.q.D));
  a.scale_log2 = std::max(scale * 1.4426950408889634f, 0x1p-126f);   // -inf * 0 is no mask
  const dim3 grid(a.items);
  auto pick = [&](auto dim) {
    constexpr int D = decltype(dim)::value;
    if (d.few && a.Nq * a.group <= 16)
      hipLaunchKernelGGL((k_cross_few<D, true>), grid, dim3(256), 0, stream, a);
    else if (d.few) hipLaunchKernelGGL((k_cross_few<D, false>), grid, dim3(256), 0, stream, a);
    else if (a.mask) hipLaunchKernelGGL((k_cross_many<D, true>), grid, dim3(256), 0, stream, a);
    else hipLaunchKernelGGL((k_cross_many<D, false>), grid, dim3(256), 0, stream, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || d.chunks == 1) return e;
    const int64_t total = x.q.B * x.q.H * x.q.N;
    const dim3 joins(static_cast<unsigned>((total + 3) / 4));
    if (d.few) hipLaunchKernelGGL((k_cross_merge<D, true>), joins, dim3(256), 0, stream, a, d.rows, total);
    else hipLaunchKernelGGL((k_cross_merge<D, false>), joins, dim3(256), 0, stream, a, d.rows, total);
    return hipGetLastError();
  };
  return x.q.D == 128 ? pick(std::integral_constant<int, 128>{})
                      : pick(std::integral_constant<int, 64>{});
}

}  // namespace vecattn
