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

template <typename T, int MT, int NT>
void launch_direct(const ProductArgs<T> &a, int waves, hipStream_t s) {
  const int64_t rows = (a.M + 16 * MT - 1) / (16 * MT);
  const int64_t cols = ((int64_t)a.N + 16 * NT - 1) / (16 * NT);
  const int64_t tiles = rows * cols;
  direct_product_kernel<T, MT, NT>
      <<<(unsigned)(tiles < kMaxTiles ? tiles : kMaxTiles), 64 * waves, 0, s>>>(a, (uint32_t)cols,
                                                                               tiles);
}

template <typename T>
int launch_product(const ProductArgs<T> &a, hipStream_t s) {
  const int steps = (a.K + kStep - 1) / kStep;
  int waves = 8;
  while (waves > 1 && waves * 2 > steps) waves /= 2;
  if (a.M <= 16)
    launch_direct<T, 1, 1>(a, waves, s);
  else if (a.M <= 32)
    launch_direct<T, 2, 2>(a, waves, s);
  else
    launch_direct<T, 4, 4>(a, waves, s);
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
