// Attention over an encoder's states: every row of q sees the same keys of its
// sequence, those below its length that the mask leaves.
//
// The query heads that share a key/value head are rows beside each other (row = token *
// group + head), so that one token's heads read K and V once.  The matrix products are
// v_mfma_f32_32x32x16_bf16, S^T = K Q^T and O^T += V^T P^T, with a row's softmax state in
// its two lanes; K and V go from memory straight to LDS with the swizzle of
// device_common.h, and V is read back transposed.  Rows of masked keys of V are fetched
// from past the buffer's end, which reads 0: what such a key holds never meets a
// product, and its score is set to -inf.  The weights are rounded to bf16 (half a step,
// 2^-9) before they meet V, as the operands are; their sum is of what was not rounded.
//
// Two kernels.  Of more than 32 rows, a workgroup owns 128 of them (a wave 32) and its
// waves share tiles of 64 keys.  Of up to 32, each of four waves takes tiles of 32 keys
// of its own, without barriers, and the waves' sums are joined at the end.  Where the
// rows alone do not fill the chip, the keys are cut into chunks, and a second kernel
// joins the chunks of a row.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "device_common.h"
#include "launch.h"

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
  float* part;         // [item][rows of a tile][D] sums, then [item][rows of a tile] (m, l)
  int32_t Hkv, group, Nq, Nk, row_tiles, chunks, chunk, run;
  int64_t items;
  float scale_log2;
};

struct Item {
  int64_t b, index;
  int hk, rt, c, len, rows, count;   // keys and rows that exist, chunks of the sequence
};

__device__ __forceinline__ int chunks_of(const CrossParams& a, int len) {
  return max(1, (len + a.chunk - 1) / a.chunk);
}
__device__ __forceinline__ int keys_of(const CrossParams& a, int64_t b) {
  return a.lens ? min(max(a.lens[b], 0), a.Nk) : a.Nk;
}
__device__ __forceinline__ int rows_of(const CrossParams& a, int64_t b) {
  return (a.n_q ? min(max(a.n_q[b], 0), a.Nq) : a.Nq) * a.group;
}

// Sequence and key/value head, then row tile, then chunk.  The hardware deals workgroup x
// to XCD x % 8; an XCD takes `run` consecutive items at a time, which share keys, so that
// it finds them in its own L2.
__device__ __forceinline__ bool find_item(const CrossParams& a, int tile_rows, Item& s) {
  const int64_t slot = blockIdx.x >> 3;
  int64_t i = (slot / a.run * 8 + (blockIdx.x & 7)) * a.run + slot % a.run;
  if (i >= a.items) return false;
  s.index = i;
  s.c = static_cast<int>(i % a.chunks);
  i /= a.chunks;
  s.rt = static_cast<int>(i % a.row_tiles);
  i /= a.row_tiles;
  s.hk = static_cast<int>(i % a.Hkv);
  s.b = i / a.Hkv;
  s.len = keys_of(a, s.b);
  s.rows = rows_of(a, s.b);
  s.count = chunks_of(a, s.len);
  return s.rt * tile_rows < s.rows && s.c < s.count;
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

// Bit r: key j0 + r exists and the mask leaves it.
template <int KEYS>
__device__ __forceinline__ uint64_t visible(const CrossParams& a, const Item& s, int j0, int lane) {
  bool see = lane < KEYS && j0 + lane < s.len;
  if (a.mask && see) see = a.mask[s.b * a.mask_sB + j0 + lane] != 0;
  return __ballot(see);
}

// Direct-to-LDS instruction u of a tile of KEYS rows (16 bytes a lane).  HIDE: rows that
// are not visible read 0; rows at or past len do so always.
template <int D, int KEYS, bool HIDE>
__device__ __forceinline__ void gather(const uint16_t* base, int64_t sN, int j0, int len, int u,
                                       int lane, uint64_t see, uint16_t* dst) {
  constexpr int CH = D / 8;
  const uint32_t rowb = static_cast<uint32_t>(sN) * 2u;
  const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(
      const_cast<uint16_t*>(base + j0 * sN), 0, max(min(KEYS, len - j0) - 1, 0) * rowb + 2 * D,
      0x00020000);
  const int i = u * 64 + lane, r = i / CH;
  uint32_t at = r * rowb + 16u * ((i % CH) ^ swz<D>(r));
  if constexpr (HIDE) at = see >> r & 1 ? at : 0x80000000u;
  gather16_to_lds(rs, at, dst + u * 64 * 8);
}

// One wave's 32 rows against tiles of keys.  KEYS: of a tile, 32 or 64.
template <int D, int KEYS>
struct Wave {
  static constexpr int DS = D / 16, DB = D / 32, RB = 2 * D, HF = KEYS / 32;
  bf16x8 qf[DS];
  f32x16 oacc[DB];
  float m_run, l_run;
  uint32_t koff[DS], voff[DB][2];
  int g, ln;

  __device__ __forceinline__ void start(int lane) {
    g = lane >> 5, ln = lane & 31;
    m_run = kUnseen;
    l_run = 0.0f;
#pragma unroll
    for (int db = 0; db < DB; ++db) oacc[db] = f32x16{};
#pragma unroll
    for (int s = 0; s < DS; ++s) koff[s] = ln * RB + 16 * ((2 * s + g) ^ swz<D>(ln));
    const int j16 = lane & 15, tq = j16 >> 2, tp = j16 & 3, vhalf = (lane >> 4) & 1;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int hi = 0; hi < 2; ++hi) {
        const int d = 32 * db + 16 * vhalf + 4 * tp;
        const int k0 = 4 * g + tq + 8 * hi;
        voff[db][hi] = k0 * RB + 16 * ((d >> 3) ^ swz<D>(k0)) + 8 * ((d >> 2) & 1);
      }
  }
  __device__ __forceinline__ void load(const uint16_t* row, bool have) {
#pragma unroll
    for (int s = 0; s < DS; ++s) {
      u32x4 t = {0, 0, 0, 0};
      if (have) t = reinterpret_cast<const u32x4*>(row)[2 * s + g];
      qf[s] = __builtin_bit_cast(bf16x8, t);
    }
  }
  __device__ __forceinline__ void score(f32x16 (&s)[HF], const uint16_t* k) {
    const char* kb = reinterpret_cast<const char*>(k);
#pragma unroll
    for (int hf = 0; hf < HF; ++hf) {
      s[hf] = f32x16{};
#pragma unroll
      for (int i = 0; i < DS; ++i)
        s[hf] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
            __builtin_bit_cast(bf16x8,
                               *reinterpret_cast<const u32x4*>(kb + hf * 32 * RB + koff[i])),
            qf[i], s[hf], 0, 0, 0);
    }
  }
  __device__ __forceinline__ void hide(f32x16 (&s)[HF], uint64_t see) {
#pragma unroll
    for (int hf = 0; hf < HF; ++hf) {
      const uint32_t bits = static_cast<uint32_t>(see >> (32 * hf)) >> (4 * g);
#pragma unroll
      for (int e = 0; e < 16; ++e) s[hf][e] = bits >> (8 * (e / 4) + e % 4) & 1u ? s[hf][e] : kNegInf;
    }
  }
  // The weights against the reference as it is; a row whose sum is past 256 on one of its
  // lanes (one that had none among them) moves its reference to its maximum first.
  __device__ __forceinline__ void weigh(const f32x16 (&s)[HF], float scale_log2,
                                        bf16x8 (&pb)[2 * HF]) {
    float p[HF][16], sum;
    auto weights = [&]() __attribute__((always_inline)) {
      float part[2 * HF];
#pragma unroll
      for (int hf = 0; hf < HF; ++hf) {
#pragma unroll
        for (int e = 0; e < 16; ++e)
          p[hf][e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[hf][e], scale_log2, -m_run));
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const float* y = p[hf] + 8 * x;
          part[2 * hf + x] = ((y[0] + y[1]) + (y[2] + y[3])) + ((y[4] + y[5]) + (y[6] + y[7]));
        }
      }
      sum = part[0] + part[1];
      if constexpr (HF == 2) sum += part[2] + part[3];
    };
    weights();
    if (__any(sum > 256.0f)) {
      float top = kNegInf;
#pragma unroll
      for (int hf = 0; hf < HF; ++hf)
#pragma unroll
        for (int e = 0; e < 16; ++e) top = fmaxf(top, s[hf][e]);
      const bool up = wave_max_xor32(sum) > 256.0f;   // no row depends on its neighbours
      const float m_new = up ? fmaxf(m_run, wave_max_xor32(top) * scale_log2) : m_run;
      const float alpha = __builtin_amdgcn_exp2f(m_run - m_new);
      m_run = m_new;
      l_run *= alpha;
#pragma unroll
      for (int db = 0; db < DB; ++db) oacc[db] *= alpha;
      weights();
    }
    l_run += sum;
#pragma unroll
    for (int hf = 0; hf < HF; ++hf)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        f32x8 y;
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = p[hf][8 * x + e];
        pb[2 * hf + x] = __builtin_convertvector(y, bf16x8);
      }
  }
  __device__ __forceinline__ void add(const bf16x8 (&pb)[2 * HF], const uint16_t* v) {
    const char* vb = reinterpret_cast<const char*>(v);
#pragma unroll
    for (int ks = 0; ks < 2 * HF; ++ks)
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        // The swizzle repeats every 16 rows.
        const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            LDS_PTR(i16x4, vb + voff[db][0] + 16 * ks * RB));
        const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            LDS_PTR(i16x4, vb + voff[db][1] + 16 * ks * RB));
        const i16x8 x = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        oacc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, x), pb[ks],
                                                           oacc[db], 0, 0, 0);
      }
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
  return a.part + a.items * tile_rows * D + (index * tile_rows + r) * 2;
}

template <int D>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2))) void k_cross_many(
    const CrossParams a) {
  constexpr int KEYS = 64, U = KEYS * (D / 8) / 256;
  using W = Wave<D, KEYS>;
  __shared__ __align__(16) uint16_t k_s0[KEYS * D];
  __shared__ __align__(16) uint16_t k_s1[KEYS * D];
  __shared__ __align__(16) uint16_t v_s0[KEYS * D];
  __shared__ __align__(16) uint16_t v_s1[KEYS * D];
  Item s;
  if (!find_item(a, kCrossRows, s)) return;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint16_t* kh = a.k + s.b * a.k_sB + s.hk * a.k_sH;
  const uint16_t* vh = a.v + s.b * a.v_sB + s.hk * a.v_sH;
  const int first = s.c * a.chunk, last = min(s.len, first + a.chunk);
  const int ntiles = (last - first + KEYS - 1) / KEYS;
  const int row = s.rt * kCrossRows + 32 * wave + (lane & 31);
  const bool have = row < s.rows;
  W w;
  w.start(lane);
  w.load(q_row(a, s, have ? row : 0), have);

  auto fetch = [&](int t, uint64_t see, uint16_t* k, uint16_t* v) __attribute__((always_inline)) {
    const int j0 = first + t * KEYS;
#pragma unroll
    for (int u = 0; u < U; ++u)
      gather<D, KEYS, false>(kh, a.k_sN, j0, s.len, wave * U + u, lane, see, k);
    if (a.mask) {
#pragma unroll
      for (int u = 0; u < U; ++u)
        gather<D, KEYS, true>(vh, a.v_sN, j0, s.len, wave * U + u, lane, see, v);
    } else {
#pragma unroll
      for (int u = 0; u < U; ++u)
        gather<D, KEYS, false>(vh, a.v_sN, j0, s.len, wave * U + u, lane, see, v);
    }
  };
  uint64_t see = 0, see_next = 0;
  if (ntiles > 0) {
    see = visible<KEYS>(a, s, first, lane);
    fetch(0, see, k_s0, v_s0);
  }
  auto turn = [&](int t, const uint16_t* k, const uint16_t* v, uint16_t* k1, uint16_t* v1)
                  __attribute__((always_inline)) {
    if (t + 1 < ntiles) see_next = visible<KEYS>(a, s, first + (t + 1) * KEYS, lane);
    wait_all();
    __builtin_amdgcn_s_barrier();
    if (t + 1 < ntiles) fetch(t + 1, see_next, k1, v1);
    f32x16 x[2];
    bf16x8 pb[4];
    w.score(x, k);
    if (see != ~uint64_t(0)) w.hide(x, see);
    w.weigh(x, a.scale_log2, pb);
    w.add(pb, v);
    see = see_next;
  };
  for (int t = 0; t < ntiles; t += 2) {
    turn(t, k_s0, v_s0, k_s1, v_s1);
    if (t + 1 < ntiles) turn(t + 1, k_s1, v_s1, k_s0, v_s0);
  }

  float l = w.l_run;
  l += __shfl_xor(l, 32);
  if (!have) return;
  if (s.count > 1) {
    const int r = 32 * wave + w.ln;
#pragma unroll
    for (int db = 0; db < W::DB; ++db)
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
  if (w.g == 0) put_lse(a, s.b, s.hk, row, w.m_run, l);
  uint16_t* orow = o_row(a, s.b, s.hk, row);
#pragma unroll
  for (int db = 0; db < W::DB; ++db)
#pragma unroll
    for (int vq = 0; vq < 4; ++vq) {
      f32x4 y;
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = w.oacc[db][4 * vq + e] * inv;
      *reinterpret_cast<bf16x4*>(orow + 32 * db + 8 * vq + 4 * w.g) =
          __builtin_convertvector(y, bf16x4);
    }
}

template <int D>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(1))) void k_cross_few(
    const CrossParams a) {
  constexpr int KEYS = 32, U = KEYS * (D / 8) / 64, ROWS = 32;
  using W = Wave<D, KEYS>;
  __shared__ __align__(16) uint16_t k_s0[4][KEYS * D];
  __shared__ __align__(16) uint16_t k_s1[4][KEYS * D];
  __shared__ __align__(16) uint16_t v_s0[4][KEYS * D];
  __shared__ __align__(16) uint16_t v_s1[4][KEYS * D];
  __shared__ float s_m[4][ROWS], s_l[4][ROWS];
  Item s;
  if (!find_item(a, ROWS, s)) return;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint16_t* kh = a.k + s.b * a.k_sB + s.hk * a.k_sH;
  const uint16_t* vh = a.v + s.b * a.v_sB + s.hk * a.v_sH;
  const int first = s.c * a.chunk, last = min(s.len, first + a.chunk);
  const int ntiles = (last - first + KEYS - 1) / KEYS;
  const int row = s.rt * ROWS + (lane & 31);
  const bool have = row < s.rows;
  W w;
  w.start(lane);
  w.load(q_row(a, s, have ? row : 0), have);

  auto fetch = [&](int t, uint64_t see, uint16_t* k, uint16_t* v) __attribute__((always_inline)) {
    const int j0 = first + t * KEYS;
#pragma unroll
    for (int u = 0; u < U; ++u) gather<D, KEYS, false>(kh, a.k_sN, j0, s.len, u, lane, see, k);
#pragma unroll
    for (int u = 0; u < U; ++u) gather<D, KEYS, true>(vh, a.v_sN, j0, s.len, u, lane, see, v);
  };
  // A tile is worked on while the wave's next is fetched; past the last one the fetch
  // goes to the last again (into a buffer that nothing reads).
  auto tile = [&](int t) __attribute__((always_inline)) { return min(t, ntiles - 1); };
  int t = wave;
  uint64_t see = 0, see1 = 0;
  if (t < ntiles) {
    see = visible<KEYS>(a, s, first + t * KEYS, lane);
    fetch(t, see, k_s0[wave], v_s0[wave]);
    see1 = visible<KEYS>(a, s, first + tile(t + 4) * KEYS, lane);
  }
  auto turn = [&](const uint16_t* k, const uint16_t* v, uint16_t* k1, uint16_t* v1)
                  __attribute__((always_inline)) {
    fetch(tile(t + 4), see1, k1, v1);
    wait_vmcnt<2 * U>();
    f32x16 x[1];
    bf16x8 pb[2];
    w.score(x, k);
    if (see != 0xFFFFFFFFu) w.hide(x, see);
    w.weigh(x, a.scale_log2, pb);
    w.add(pb, v);
    see = see1;
    t += 4;
    see1 = visible<KEYS>(a, s, first + tile(t + 4) * KEYS, lane);
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
  const int r = threadIdx.x >> 3, sr = s.rt * ROWS + r;
  if (sr >= s.rows) return;
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
    if (s.count > 1) {
      put_part<D>(a, s, ROWS, r, d, y);
    } else {
      y *= inv;
      *reinterpret_cast<bf16x4*>(o_row(a, s.b, s.hk, sr) + d) = __builtin_convertvector(y, bf16x4);
    }
  }
  if ((threadIdx.x & 7) == 0) {
    if (s.count > 1) {
      float* ml = part_ml<D>(a, s.index, ROWS, r);
      ml[0] = mr, ml[1] = lr;
    } else {
      put_lse(a, s.b, s.hk, sr, mr, lr);
    }
  }
}

// Joins the chunks of a row, a wave per row, a lane D / 64 values.
template <int D>
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
  const int count = chunks_of(a, keys_of(a, b));
  if (count <= 1 || row >= rows_of(a, b)) return;
  const int64_t at = (bh * a.row_tiles + row / tile_rows) * a.chunks;
  const int r = row % tile_rows;
  const float* ml = part_ml<D>(a, at, tile_rows, r);
  const float* src = a.part + (at * tile_rows + r) * D + V * lane;
  const int64_t step = static_cast<int64_t>(tile_rows);
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
  int32_t rows, tiles, chunks, chunk;
  int64_t items;
};

Deal deal(int64_t B, int64_t Hq, int64_t Hkv, int64_t Nq, int64_t Nk, int64_t D) {
  Deal d;
  const int64_t rows = Nq * (Hq / Hkv);
  d.few = rows <= 32;
  d.rows = d.few ? 32 : kCrossRows;
  d.tiles = static_cast<int32_t>((rows + d.rows - 1) / d.rows);
  const int64_t units = B * Hkv * d.tiles;
  // Workgroups that run at a time, and the fewest keys that pay for a chunk.
  const int64_t slots = d.few && D == 128 ? 256 : 512;
  const int64_t least = 256;
  int64_t chunks = std::min((Nk + least - 1) / least, std::max<int64_t>(1, 2 * slots / units));
  d.chunk = static_cast<int32_t>(((Nk + chunks - 1) / chunks + 127) / 128 * 128);
  d.chunks = static_cast<int32_t>((Nk + d.chunk - 1) / d.chunk);
  d.items = units * d.chunks;
  return d;
}

}  // namespace

size_t cross_attn_workspace_bytes(int64_t B, int64_t Hq, int64_t Hkv, int64_t Nq, int64_t Nk,
                                  int64_t D) {
  const Deal d = deal(B, Hq, Hkv, Nq, Nk, D);
  return d.chunks > 1 ? static_cast<size_t>(d.items) * d.rows * (D + 2) * sizeof(float) : 0;
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
  a.part = static_cast<float*>(x.workspace);
  a.Hkv = static_cast<int32_t>(x.k.H);
  a.group = static_cast<int32_t>(x.q.H / x.k.H);
  a.Nq = static_cast<int32_t>(x.q.N), a.Nk = static_cast<int32_t>(x.k.N);
  a.row_tiles = d.tiles, a.chunks = d.chunks, a.chunk = d.chunk;
  a.items = d.items;
  const float scale = x.scale != 0.0f ? x.scale : 1.0f / sqrtf(static_cast<float>(x.q.D));
  a.scale_log2 = std::max(scale * 1.4426950408889634f, 0x1p-126f);   // -inf * 0 is no mask
  a.run = static_cast<int32_t>(std::min<int64_t>(64, std::max<int64_t>(1, a.items / 32)));
  const int64_t rounds = (a.items + 8 * a.run - 1) / (8 * a.run);
  const dim3 grid(static_cast<unsigned>(rounds * 8 * a.run));
  auto pick = [&](auto dim) {
    constexpr int D = decltype(dim)::value;
    if (d.few) hipLaunchKernelGGL(k_cross_few<D>, grid, dim3(256), 0, stream, a);
    else hipLaunchKernelGGL(k_cross_many<D>, grid, dim3(256), 0, stream, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || d.chunks == 1) return e;
    const int64_t total = x.q.B * x.q.H * x.q.N;
    hipLaunchKernelGGL(k_cross_merge<D>, dim3(static_cast<unsigned>((total + 3) / 4)), dim3(256), 0,
                       stream, a, d.rows, total);
    return hipGetLastError();
  };
  return x.q.D == 128 ? pick(std::integral_constant<int, 128>{})
                      : pick(std::integral_constant<int, 64>{});
}

}  // namespace vecattn
