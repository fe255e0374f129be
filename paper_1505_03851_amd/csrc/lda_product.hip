// Host side and C ABI of the products of 8-bit rows and weights (gfx950): argument
// checks, launch shapes and launches.  Device code: product.hpp, elements.hpp.
#include <hip/hip_runtime.h>

#include <stdint.h>

#include "lda_draw.h"
#include "status.hpp"
#include "arguments.hpp"
#include "product.hpp"

namespace lda {
namespace {

constexpr int64_t kMaxTiles = 1 << 20;  // of a launch; workgroups stride over the rest

constexpr int64_t kUnits = 256, kLdsBytes = 160 << 10;

template <typename T>
void launch_direct(const ProductArgs<T> &a, hipStream_t s) {
  const int64_t rows = (a.M + 15) / 16, cols = ((int64_t)a.N + 15) / 16, tiles = rows * cols;
  const int steps = (a.K + kStep - 1) / kStep;
  int waves = 4;
  while (waves > 1 && waves * 2 > steps) waves /= 2;
  direct_product_kernel<T><<<(unsigned)(tiles < kMaxTiles ? tiles : kMaxTiles), 64 * waves, 0, s>>>(
      a, (uint32_t)cols, tiles);
}

int64_t tiles_of(int64_t M, int64_t N, int BM, int BN) {
  return (M + BM - 1) / BM * ((N + BN - 1) / BN);
}

// As many workgroups as the GPU holds at once, each with its tiles.
template <int BM, int BN, int WM, int WN, int GROUPS, bool ANY, typename T>
void launch_tiled(const ProductArgs<T> &a, hipStream_t s) {
  constexpr int kWaves = WM * WN * GROUPS;
  constexpr int64_t lds = (int64_t)(BM + BN) * GROUPS * 2 * kStage;
  constexpr int64_t per = kLdsBytes / lds < 32 / kWaves ? kLdsBytes / lds : 32 / kWaves;
  const int64_t tiles = tiles_of(a.M, a.N, BM, BN);
  tiled_product_kernel<T, BM, BN, WM, WN, GROUPS, ANY>
      <<<(unsigned)(tiles < kUnits * per ? tiles : kUnits * per), 64 * kWaves, 0, s>>>(
          a, (uint32_t)((a.M + BM - 1) / BM), (uint32_t)tiles);
}

// Which kernel, by the number of tiles (times in us on one MI355X, aligned lines, K = 4,096
// unless named):
//   * up to 16 rows and 16,384 channels, the direct one: 1 x 8,192 8.9 against 11.3 for the
//     best tile, 16,384 14.7 against 17.2, 32,768 25.6 against 24.9;
//   * tiles of 256 x 256 run one to a compute unit, of 128 x 128 two; a round of the first
//     takes 1.8 times a round of the second (4,096 x 4,096: 65 and 2 x 36; through registers
//     97 and 2 x 68, but short lines by the second alone: 616 x 66,816 x 70 45 against 54);
//   * from 160 tiles of 128 x 128 and more than 64 rows those two: 1,000 x 5,000 x 1,024 12.6
//     against 16.4 for 64 x 64, but 512 x 4,096 (128 tiles) 26 against 22;
//   * below, the fewer tiles the more groups share K: 32 x 32 by eight where all run at once
//     (32 x 4,096 8.2 against 11.3 for 64 x 64 by four, 512 x 512 8.6 against 12.0; 128 x 4,096,
//     512 tiles, 16 against 12), 64 x 64 by two from 384 tiles (256 x 8,192 22; by four 27, by one
//     26), by one from 1,024 and for short lines (64 x 100,000 92, by two 96, by four 113; 1 x
//     100,000 x 128 7.6, 9.9, 19.5), else by four;
//   * lines through registers the same, and 32 x 64 by four where those all run at once
//     (128 x 4,096 x 4,095 17.5 against 21.6).
template <typename T>
int launch_product(const ProductArgs<T> &a, hipStream_t s) {
  const bool lines = a.K % 16 == 0 && aligned(a.q, 16) && aligned(a.w, 16) &&
                     (a.M == 1 || a.ldq % 16 == 0) && (a.N == 1 || a.ldw % 16 == 0);
  // the tiled kernels address a tile's lines in 32 bits
  const bool near = a.ldq <= 1 << 23 && a.ldw <= 1 << 23 && tiles_of(a.M, a.N, 32, 32) < 1LL << 31;
  if (!near || a.K < 16 || (lines && a.M <= 16 && a.N <= 16384)) {
    launch_direct(a, s);
    return launch_status();
  }
  const int64_t t256 = tiles_of(a.M, a.N, 256, 256), t128 = tiles_of(a.M, a.N, 128, 128);
  const int64_t t64 = tiles_of(a.M, a.N, 64, 64);
#define LDA_TILES(BM, BN, WM, WN, GROUPS)              \
  do {                                                 \
    if (lines)                                         \
      launch_tiled<BM, BN, WM, WN, GROUPS, false>(a, s); \
    else                                               \
      launch_tiled<BM, BN, WM, WN, GROUPS, true>(a, s);  \
  } while (0)
  if (a.M > 64 && t128 >= 160) {
    const int64_t rounds = (t256 + kUnits - 1) / kUnits, halves = (t128 + 2 * kUnits - 1) / (2 * kUnits);
    if (lines ? 9 * rounds <= 5 * halves : a.K >= 512 && 3 * rounds <= 2 * halves)
      LDA_TILES(256, 256, 2, 4, 1);
    else
      LDA_TILES(128, 128, 2, 4, 1);
  } else if (a.K >= 1024 && tiles_of(a.M, a.N, 32, 32) <= kUnits) {
    LDA_TILES(32, 32, 1, 1, 8);
  } else if (a.K <= 512 || t64 >= 1024) {
    LDA_TILES(64, 64, 2, 2, 1);
  } else if (t64 >= 384) {
    LDA_TILES(64, 64, 2, 2, 2);
  } else if (!lines && tiles_of(a.M, a.N, 32, 64) <= kUnits) {
    launch_tiled<32, 64, 1, 2, 4, true>(a, s);
  } else {
    LDA_TILES(64, 64, 2, 2, 4);
  }
#undef LDA_TILES
  return launch_status();
}

template <typename T>
int run_product(const int8_t *q, int64_t ldq, const float *scale, const int8_t *w, int64_t ldw,
                const float *weight_scale, const float *bias, void *out, int64_t ldo, int64_t M,
                int32_t N, int32_t K, hipStream_t s) {
  return launch_product(ProductArgs<T>{q, w, scale, weight_scale, bias, (typename T::store *)out,
                                       ldq, ldw, ldo, M, N, K},
                        s);
}

}  // namespace
}  // namespace lda

using namespace lda;

extern "C" int lda_project_int8(const int8_t *q, int64_t ld_q, const float *scale,
                                const int8_t *weight, int64_t ld_weight,
                                const float *weight_scale, const float *bias, void *out,
                                int64_t ld_out, int64_t M, int32_t N, int32_t K, int32_t dtype,
                                void *stream) {
  if (M < 0 || N <= 0 || K <= 0) return LDA_ERR_SHAPE;
  if (M > LDA_MAX_N || K > LDA_PROJECT_MAX_K) return LDA_ERR_UNSUPPORTED;
  const int size = dtype_size(dtype);
  if (!size || ld_q < 0 || ld_weight < 0 || ld_out < N) return LDA_ERR_VALUE;
  if (M == 0) return LDA_OK;
  if (!q || !scale || !weight || !weight_scale || !out) return LDA_ERR_NULL;
  if (!aligned(scale, 4) || !aligned(weight_scale, 4) || !aligned(bias, 4) || !aligned(out, size))
    return LDA_ERR_ALIGN;
  hipStream_t s = static_cast<hipStream_t>(stream);
#define LDA_RUN(T) \
  run_product<T>(q, ld_q, scale, weight, ld_weight, weight_scale, bias, out, ld_out, M, N, K, s)
  switch (dtype) {
    case LDA_F32: return LDA_RUN(F32);
    case LDA_BF16: return LDA_RUN(Bf16);
    default: return LDA_RUN(F16);
  }
#undef LDA_RUN
}
