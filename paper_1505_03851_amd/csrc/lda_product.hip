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
  int waves = 8;
  while (waves > 1 && waves * 2 > steps) waves /= 2;
  direct_product_kernel<T><<<(unsigned)(tiles < kMaxTiles ? tiles : kMaxTiles), 64 * waves, 0, s>>>(
      a, (uint32_t)cols, tiles);
}

int64_t tiles_of(int64_t M, int64_t N, int BM, int BN) {
  return (M + BM - 1) / BM * ((N + BN - 1) / BN);
}

// As many workgroups as the GPU holds at once, each with its tiles.
template <int BM, int BN, int WM, int WN, int GROUPS, int STAGES, bool ANY, typename T>
void launch_tiled(const ProductArgs<T> &a, hipStream_t s) {
  constexpr int kWaves = WM * WN * GROUPS;
  constexpr int64_t lds = (int64_t)(BM + BN) * GROUPS * STAGES * kStage;
  constexpr int64_t per = kLdsBytes / lds < 32 / kWaves ? kLdsBytes / lds : 32 / kWaves;
  const int64_t tiles = tiles_of(a.M, a.N, BM, BN);
  tiled_product_kernel<T, BM, BN, WM, WN, GROUPS, STAGES, ANY>
      <<<(unsigned)(tiles < kUnits * per ? tiles : kUnits * per), 64 * kWaves, 0, s>>>(
          a, (uint32_t)((a.M + BM - 1) / BM), (uint32_t)tiles);
}

// Which kernel, by the number of tiles (times in us on one MI355X, K = 4,096 unless named):
//   * up to 16 rows and 16,384 channels, the direct one: 1 x 4,096 7.5 against 9.3 for 32 x 64
//     tiles and 13 for 64 x 64; at 100,000 channels 64 x 64 tiles 77 against 87;
//   * tiles of 256 x 256 run one to a compute unit, of 128 x 128 two; a round of the first
//     takes 1.8 times a round of the second (4,096 x 4,096: 65 and 2 x 36);
//   * from 160 tiles of 128 x 128 and more than 64 rows those two: 1,000 x 5,000 x 1,024 12.6
//     against 16.4 for 64 x 64, but 512 x 4,096 (128 tiles) 26 against 22;
//   * below, 64 x 64: one group where there are many (64 x 100,000: 92; two groups 96, four
//     113), two groups from 384 tiles (256 x 8,192: 22; one 26, four 27), else four (128 x
//     4,096: 12; two 14, one 19); up to 32 rows 32 x 64 by four (32 x 4,096: 9.6 against 11.2).
// Lines that are not aligned pass registers: 128 x 128 tiles (4,000 x 4,001 x 4,001 135; 256 x
// 256 would spill), and 64 x 64 by two and four groups (333 x 1,003 x 1,001 13.1 and 12.5).
template <typename T>
int launch_product(const ProductArgs<T> &a, hipStream_t s) {
  // the tiled kernels address a tile's lines in 32 bits
  const bool near = a.ldq <= 1 << 23 && a.ldw <= 1 << 23 && tiles_of(a.M, a.N, 32, 64) < 1LL << 31;
  if (!near || (a.M <= 16 && a.N <= 16384)) {
    launch_direct(a, s);
    return launch_status();
  }
  const bool lines = a.K % 16 == 0 && aligned(a.q, 16) && aligned(a.w, 16) &&
                     (a.M == 1 || a.ldq % 16 == 0) && (a.N == 1 || a.ldw % 16 == 0);
  const int64_t t256 = tiles_of(a.M, a.N, 256, 256), t128 = tiles_of(a.M, a.N, 128, 128);
  const int64_t t64 = tiles_of(a.M, a.N, 64, 64);
  if (a.M > 64 && t128 >= 160) {
    const int64_t rounds = (t256 + kUnits - 1) / kUnits, halves = (t128 + 2 * kUnits - 1) / (2 * kUnits);
    if (!lines)
      launch_tiled<128, 128, 2, 4, 1, 2, true>(a, s);
    else if (9 * rounds <= 5 * halves)
      launch_tiled<256, 256, 2, 4, 1, 2, false>(a, s);
    else
      launch_tiled<128, 128, 2, 4, 1, 2, false>(a, s);
  } else if (!lines) {
    if (t64 >= 384)
      launch_tiled<64, 64, 2, 2, 2, 2, true>(a, s);
    else
      launch_tiled<64, 64, 2, 2, 4, 2, true>(a, s);
  } else if (t64 >= 1024) {
    launch_tiled<64, 64, 2, 2, 1, 2, false>(a, s);
  } else if (t64 >= 384) {
    launch_tiled<64, 64, 2, 2, 2, 2, false>(a, s);
  } else if (a.M <= 32) {
    launch_tiled<32, 64, 1, 2, 4, 2, false>(a, s);
  } else {
    launch_tiled<64, 64, 2, 2, 4, 2, false>(a, s);
  }
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
