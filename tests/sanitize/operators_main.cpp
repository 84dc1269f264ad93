// Rotary positions, eviction from the cache and cross attention through the C ABI's host code
// under AddressSanitizer and UndefinedBehaviorSanitizer, without a GPU: ladders, workspace sizes
// over a range of shapes up to the limits, refusals (with addresses that are never dereferenced), and
// calls with valid arguments, which reach the launch code and must fail with
// VECATTN_ERR_DEVICE.  Prints "ok" at the end.
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <limits>
#include <vector>

#include "vecattn.h"

static int failures = 0;
static void expect(bool ok, const char* what) {
  if (!ok) {
    std::printf("FAILED: %s\n", what);
    ++failures;
  }
}

static vecattn_tdesc desc(int64_t B, int64_t H, int64_t N, int64_t D) {
  return vecattn_tdesc{B, H, N, D, H * N * D, N * D, D};
}

static void* const fake = reinterpret_cast<void*>(uintptr_t(0x100000));
static void* const fake2 = reinterpret_cast<void*>(uintptr_t(0x40000000));
static int32_t* const ifake = static_cast<int32_t*>(fake);
static float* const ffake = static_cast<float*>(fake);
static uint8_t* const bfake = static_cast<uint8_t*>(fake);
constexpr int64_t kMost = int64_t(1) << 30;
constexpr size_t kBig = size_t(1) << 40;

static void ladders() {
  for (int32_t rot : {2, 4, 6, 48, 126, 128})
    for (int32_t scaling = VECATTN_ROPE_NONE; scaling <= VECATTN_ROPE_BANDS; ++scaling)
      for (double base : {1.0000001, 1e4, 1e300})
        for (double context : {1e-300, 3.0, 8192.0, 1e18, 1e300}) {
          std::vector<double> freq(rot / 2, std::nan(""));   // no entry behind the last
          double m = 0.0;
          expect(vecattn_rope_ladder(rot, base, scaling, 16.0, context, 32.0, 1.0, freq.data(), &m) ==
                     VECATTN_OK, "ladder");
          for (double f : freq) expect(f >= 0.0 && f <= 1.0, "frequency");
          expect(m >= 1.0, "factor of the ladder");
        }
  double f[64], m;
  const double inf = std::numeric_limits<double>::infinity();
  expect(vecattn_rope_ladder(130, 1e4, 0, 1.0, 1.0, 2.0, 1.0, f, &m) == VECATTN_ERR_INVALID_ARG, "rot");
  expect(vecattn_rope_ladder(8, inf, 0, 1.0, 1.0, 2.0, 1.0, f, &m) == VECATTN_ERR_INVALID_ARG, "base");
  expect(vecattn_rope_ladder(8, 1e4, 3, 1.0, inf, 2.0, 1.0, f, &m) == VECATTN_ERR_INVALID_ARG, "context");
}

static void rope() {
  for (int64_t D : {int64_t(64), int64_t(128)})
    for (int32_t layout : {VECATTN_ROPE_HALF, VECATTN_ROPE_INTERLEAVED})
      for (int32_t rot : {int32_t(2), int32_t(20), int32_t(D)}) {
        const std::vector<double> freq(rot / 2, 1.0);   // host memory that the launch reads
        std::vector<int32_t> axis(rot / 2, 1);
        vecattn_rope_spec s{rot, layout, 2, VECATTN_CLEAR_PADDING, 1.0, freq.data(), axis.data()};
        for (int64_t N : {int64_t(1), int64_t(1000), int64_t(1) << 26, kMost}) {
          const vecattn_tdesc q = desc(1, 4, N, D), k = desc(1, 1, N, D);
          expect(vecattn_rope(fake, &q, fake, &k, &s, ifake, N, 0, nullptr, nullptr, 0, fake2, &q, fake2,
                              &k, nullptr) == VECATTN_ERR_DEVICE, "rope launch");
          expect(vecattn_rope(fake, &q, nullptr, nullptr, &s, nullptr, 0, 0, ifake, ifake, 0, fake, &q,
                              nullptr, nullptr, nullptr) == VECATTN_ERR_DEVICE, "rope in place");
        }
        s.axis = nullptr;
        const vecattn_tdesc q = desc(1 << 20, 2, 1, D), many = desc(2, 1, kMost, D);
        expect(vecattn_rope(fake, &q, nullptr, nullptr, &s, nullptr, 0, 0, nullptr, nullptr, kMost, fake2,
                            &q, nullptr, nullptr, nullptr) == VECATTN_ERR_DEVICE, "rope of tokens");
        expect(vecattn_rope(fake, &many, nullptr, nullptr, &s, nullptr, 0, 0, nullptr, nullptr, 0, fake2,
                            &many, nullptr, nullptr, nullptr) == VECATTN_ERR_UNSUPPORTED, "rope size");
        axis.back() = 2;
        s.axis = axis.data();
        expect(vecattn_rope(fake, &q, nullptr, nullptr, &s, nullptr, 0, 0, nullptr, nullptr, 0, fake2, &q,
                            nullptr, nullptr, nullptr) == VECATTN_ERR_INVALID_ARG, "rope axis");
      }
}

static void eviction() {
  for (int32_t D : {64, 128})
    for (int32_t bits : {4, 8}) {
      const vecattn_cache c{fake, 100, 4, D, 64, bits};
      for (int64_t group : {int64_t(1), int64_t(7)})
        for (int64_t n : {int64_t(1), int64_t(4), int64_t(40), int64_t(1000), int64_t(1) << 20})
          for (int64_t M : {int64_t(1), int64_t(131072), kMost}) {
            const vecattn_tdesc q = desc(2, 4 * group, n, D);
            size_t bytes = 1;
            const vecattn_status st = vecattn_cache_mass_workspace_size(&q, &c, &bytes);
            const bool fits = 2 * 4 * group * n < (int64_t(1) << 24);
            expect(st == (fits ? VECATTN_OK : VECATTN_ERR_UNSUPPORTED), "mass size");
            expect(vecattn_cache_mass(fake, &q, ffake, &c, ifake, 4, ifake, ifake, kMost, 0, 0.0f, 0.5f,
                                      ffake, static_cast<float*>(fake2), M, VECATTN_CLEAR_PADDING, fake,
                                      kBig, nullptr) == (fits ? VECATTN_ERR_DEVICE
                                                              : VECATTN_ERR_UNSUPPORTED), "mass launch");
            if (fits && bytes > 0)
              expect(vecattn_cache_mass(fake, &q, ffake, &c, ifake, 4, ifake, nullptr, 9, 3, 1.0f, 1.0f,
                                        nullptr, ffake, M, 0, fake, bytes - 1, nullptr) ==
                         VECATTN_ERR_CAPACITY, "mass workspace");
          }
      for (int64_t M : {int64_t(1), int64_t(8192), int64_t(32768), int64_t(32769), kMost})
        for (int64_t cols : {int64_t(1), int64_t(513), kMost / 64}) {
          size_t bytes = 1;
          expect(vecattn_cache_keep_workspace_size(&c, cols, 3, M, &bytes) == VECATTN_OK, "keep size");
          expect((bytes > 0) == (M > 32768 && cols * 64 > 32768), "keep workspace");
          expect(vecattn_cache_keep(ffake, M, 3, &c, ifake, cols, ifake, kMost, 9, kMost - 9, ifake, ifake,
                                    fake, kBig, nullptr) == VECATTN_ERR_DEVICE, "keep launch");
        }
      for (int64_t budget : {int64_t(1), int64_t(4097), kMost / 2}) {
        expect(vecattn_cache_gather(&c, ifake, 9, 3, ifake, ifake, budget, &c, ifake, 9, ffake, 77, ffake,
                                    VECATTN_CLEAR_PADDING, nullptr) == VECATTN_ERR_DEVICE, "gather launch");
        expect(vecattn_cache_gather_wide(&c, ifake, 9, 3, ifake, ifake, budget, &c, ifake, 9, ffake, 77,
                                         ffake, kMost, 0, nullptr) == VECATTN_ERR_DEVICE, "wide launch");
        expect(vecattn_cache_gather_wide(&c, ifake, 9, 3, ifake, ifake, budget, &c, ifake, 9, ffake, 77,
                                         ffake, budget - 1, 0, nullptr) == VECATTN_ERR_INVALID_ARG, "wide");
      }
      const vecattn_tdesc k = desc(3, 4, 100, D);
      expect(vecattn_cache_read_whole(&c, ifake, 9, ifake, kMost, fake, &k, fake2, &k, nullptr) ==
                 VECATTN_ERR_DEVICE, "read launch");
      expect(vecattn_cache_read_whole(&c, ifake, 9, ifake, -1, fake, &k, fake2, &k, nullptr) ==
                 VECATTN_ERR_INVALID_ARG, "read start");
    }
}

static void cross() {
  for (int64_t D : {int64_t(64), int64_t(128)})
    for (int64_t B : {int64_t(1), int64_t(256), int64_t(300), int64_t(1) << 20})
      for (int64_t Hkv : {int64_t(1), int64_t(12)})
        for (int64_t group : {int64_t(1), int64_t(7)})
          for (int64_t Nq : {int64_t(1), int64_t(5), int64_t(300), int64_t(75600), kMost})
            for (int64_t Nk : {int64_t(1), int64_t(577), int64_t(4097), int64_t(131072), kMost}) {
              const vecattn_tdesc q = desc(B, Hkv * group, Nq, D);
              vecattn_tdesc k = desc(B, Hkv, Nk, D);
              size_t bytes = 0;
              const vecattn_status st = vecattn_cross_attn_workspace_size(&q, &k, &bytes);
              expect(st == VECATTN_OK || st == VECATTN_ERR_UNSUPPORTED, "cross size");
              if (q.sB > (int64_t(1) << 60) / B || k.sB > (int64_t(1) << 60) / B) continue;
              expect(vecattn_cross_attn(fake, &q, fake, &k, fake, &k, ifake, bfake, Nk, ifake,
                                        VECATTN_CLEAR_PADDING, 0.0f, fake2, &q, ffake, fake,
                                        size_t(1) << 50, nullptr) ==
                         (st == VECATTN_OK ? VECATTN_ERR_DEVICE : st), "cross launch");
              if (st == VECATTN_OK && bytes > 0)
                expect(vecattn_cross_attn(fake, &q, fake, &k, fake, &k, nullptr, nullptr, 0, nullptr, 0,
                                          1.0f, fake2, &q, nullptr, fake, bytes - 1, nullptr) ==
                           VECATTN_ERR_CAPACITY, "cross workspace");
              k.sN = int64_t(1) << 24;
              if (st == VECATTN_OK && Nk > 1)
                expect(vecattn_cross_attn(fake, &q, fake, &k, fake, &k, nullptr, nullptr, 0, nullptr, 0,
                                          1.0f, fake2, &q, nullptr, fake, bytes, nullptr) ==
                           VECATTN_ERR_UNSUPPORTED, "cross stride");
            }
}

int main() {
  ladders();
  rope();
  eviction();
  cross();
  std::printf(failures ? "failures: %d\n" : "ok\n", failures);
  return failures ? 1 : 0;
}
