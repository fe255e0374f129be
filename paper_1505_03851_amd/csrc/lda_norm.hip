// Host side and C ABI of the rows' norm, its gradient, and rows in 8 bits
// (gfx950): argument checks, launch shapes and launches.
//
// lda_add_norm       the residual added, rows divided by their root mean square;
//                    in the rows' type or in 8 bits with a scale for each row.
// lda_norm_grad      the gradients of the rows and of the weight.
// lda_quantise_rows  rows in 8 bits with a scale for each.
//
// Device code: norm_rows.hpp, elements.hpp, wave_ops.hpp.
#include <hip/hip_runtime.h>

#include <stdint.h>

#include "lda_draw.h"
#include "status.hpp"
#include "arguments.hpp"
#include "norm_rows.hpp"

namespace lda {
namespace {

// Rows of a launch: fewer than 2^32 work-items.
constexpr int64_t kSlice = 1 << 22;
// Rows that stay in registers, a lane's 8 columns loaded together; others go to the
// kernels that take rows of any length.
bool in_registers(int32_t D) { return D >= 8 && D <= 16384; }
constexpr int64_t kLongBlocks = 512;

// f(WAVES, UNITS) of the shape that holds rows of D columns.  Up to 2,048 columns a row
// is one wavefront's, without a barrier.
#define LDA_ROW_SHAPE(D, F) \
  do {                      \
    if ((D) <= 512) {       \
      F(1, 1);              \
    } else if ((D) <= 1024) { \
      F(1, 2);              \
    } else if ((D) <= 2048) { \
      F(1, 4);              \
    } else if ((D) <= 4096) { \
      F(4, 2);              \
    } else if ((D) <= 6144) { \
      F(4, 3);              \
    } else if ((D) <= 8192) { \
      F(4, 4);              \
    } else {                \
      F(4, 8);              \
    }                       \
  } while (0)

// Rows of 16 bits pass the caches by where a call reads and writes more than they hold (times
// of a call among others): 16,384 x 4,096 bfloat16 with a residual (537 MB) 87.6 us against 94,
// its gradient 109 against 118, without one (403 MB) 84 against 88; below, what the launch before
// wrote may still be there: the norm of 16,384 x 4,096 without a residual (268 MB) 46 against 39,
// of 8,192 x 4,096 with one (268 MB) 45 against 40.  A lane's 32 bytes of floats are two accesses
// to one line: 16,384 x 4,096 with a residual 202 against 189, its gradient 209 against 207.
template <typename T>
bool past_caches(int64_t rows, int64_t columns, int arrays) {
  const int64_t size = (int64_t)sizeof(typename T::store);
  return size == 2 && rows * columns * arrays * size > (int64_t)320 << 20;
}

unsigned long_grid(int64_t N) { return (unsigned)(N < kLongBlocks ? N : kLongBlocks); }

template <typename T, bool BITS8>
int launch_norm(NormArgs<T> a, hipStream_t s) {
  if (!in_registers(a.D)) {
    norm_long_kernel<T, BITS8><<<long_grid(a.N), kLongThreads, 0, s>>>(a);
    return launch_status();
  }
  constexpr bool kMayStream = sizeof(typename T::store) == 2;
  const int64_t N = a.N;
  const bool stream = past_caches<T>(N, a.D, 2 + (a.residual != nullptr) + (a.sum != nullptr));
  for (int64_t at = 0; at < N; at += kSlice) {
    a.N = N - at < kSlice ? N - at : kSlice;
#define LDA_NORM_BY(WAVES, UNITS, STREAM)                                             \
  norm_kernel<T, WAVES, UNITS, BITS8, STREAM>                                         \
      <<<(unsigned)(WAVES == 1 ? (a.N + 3) / 4 : a.N), WAVES == 1 ? 256 : 64 * WAVES, \
         0, s>>>(a)
#define LDA_NORM(WAVES, UNITS)               \
  if (stream)                                \
    LDA_NORM_BY(WAVES, UNITS, kMayStream);   \
  else                                       \
    LDA_NORM_BY(WAVES, UNITS, false)
    LDA_ROW_SHAPE(a.D, LDA_NORM);
#undef LDA_NORM
#undef LDA_NORM_BY
    a.x += a.N * a.ldx;
    if (a.residual) a.residual += a.N * a.ldr;
    if (a.sum) a.sum += a.N * a.lds;
    a.out = (char *)a.out + a.N * a.ldo * (int64_t)(BITS8 ? 1 : sizeof(typename T::store));
    if (BITS8) a.scale += a.N;
  }
  return launch_status();
}

template <typename T>
int run_norm(const void *x, int64_t ldx, const void *residual, int64_t ldr, const void *weight,
             void *out, int64_t ldo, void *sum, int64_t lds, float *scale, int64_t N, int32_t D,
             bool weight_float, bool bits8, double eps, hipStream_t s) {
  using S = typename T::store;
  const NormArgs<T> a{(const S *)x, (const S *)residual, weight, out, (S *)sum, scale,
                      ldx,          ldr,                 ldo,    lds, N,        D,
                      (float)eps,   weight_float};
  return bits8 ? launch_norm<T, true>(a, s) : launch_norm<T, false>(a, s);
}

template <typename T>
int launch_quantise(const void *x, int64_t ldx, int8_t *q, int64_t ldq, float *scale, int64_t N,
                    int32_t D, hipStream_t s) {
  QuantArgs<T> a{(const typename T::store *)x, q, scale, ldx, ldq, N, D};
  if (!in_registers(D)) {
    quantise_long_kernel<T><<<long_grid(N), kLongThreads, 0, s>>>(a);
    return launch_status();
  }
  for (int64_t at = 0; at < N; at += kSlice) {
    a.N = N - at < kSlice ? N - at : kSlice;
#define LDA_QUANTISE(WAVES, UNITS)                                                    \
  quantise_kernel<T, WAVES, UNITS>                                                    \
      <<<(unsigned)(WAVES == 1 ? (a.N + 3) / 4 : a.N), WAVES == 1 ? 256 : 64 * WAVES, \
         0, s>>>(a)
    LDA_ROW_SHAPE(D, LDA_QUANTISE);
#undef LDA_QUANTISE
    a.x += a.N * ldx;
    a.q += a.N * ldq;
    a.scale += a.N;
  }
  return launch_status();
}

// The workgroups that share the rows of a gradient, each with a strip's sums of D: as
// many as the GPU holds at 16 wavefronts to a compute unit.  One, which needs no second
// launch (3 us of a small call's 14), for up to eight turns of its rows.
int32_t strips_of(int64_t N, int32_t D) {
  if (N == 0) return 0;  // nothing is read: there is no workspace either
  if (!in_registers(D)) return (int32_t)(N < 256 ? N : 256);
  const int64_t rows = D <= 1024 ? 4 : D <= 2048 ? 2 : 1;  // at a time
  if (N <= 8 * rows) return 1;
  const int64_t most = D <= 4096 ? 1024 : D <= 8192 ? 512 : 256, all = (N + rows - 1) / rows;
  return (int32_t)(all < most ? all : most);
}

// Whether the strips' sums are added up by a launch of their own, in a workspace.
bool joins_strips(int64_t N, int32_t D) {
  return N == 0 || !in_registers(D) || strips_of(N, D) > 1;
}

template <typename T>
int launch_norm_grad(const void *grad, int64_t ldg, const void *h, int64_t ldh,
                     const void *residual, int64_t ldr, const void *weight, void *dx, int64_t ldx,
                     float *dw, int64_t N, int32_t D, bool weight_float, double eps,
                     bool accumulate, float *part, hipStream_t s) {
  using S = typename T::store;
  const int32_t strips = strips_of(N, D);
  const bool joins = joins_strips(N, D);
  const NormGradArgs<T> a{(const S *)grad, (const S *)h, (const S *)residual, weight, (S *)dx,
                          joins ? part : dw, !joins && accumulate, ldg, ldh, ldr, ldx, N, D,
                          (float)eps, weight_float};
  if (N > 0 && !in_registers(D))
    norm_grad_long_kernel<T><<<(unsigned)strips, kLongThreads, 0, s>>>(a);
  else if (N > 0) {
    constexpr bool kMayStream = sizeof(S) == 2;
    const bool stream = past_caches<T>(N, D, 3 + (residual != nullptr));
#define LDA_NORM_GRAD_BY(WAVES, STREAM) \
  norm_grad_kernel<T, WAVES, STREAM>    \
      <<<(unsigned)strips, WAVES <= 4 ? kNormThreads : 64 * WAVES, 0, s>>>(a)
#define LDA_NORM_GRAD(WAVES)             \
  if (stream)                            \
    LDA_NORM_GRAD_BY(WAVES, kMayStream); \
  else                                   \
    LDA_NORM_GRAD_BY(WAVES, false)
    if (D <= 1024) {
      LDA_NORM_GRAD(1);
    } else if (D <= 2048) {
      LDA_NORM_GRAD(2);
    } else if (D <= 4096) {
      LDA_NORM_GRAD(4);
    } else if (D <= 8192) {
      LDA_NORM_GRAD(8);
    } else {
      LDA_NORM_GRAD(16);
    }
#undef LDA_NORM_GRAD
#undef LDA_NORM_GRAD_BY
  }
  if (!joins) return launch_status();
  const int64_t tiles = ((int64_t)D + 63) / 64;
  join_strips_kernel<<<(unsigned)(tiles < (1 << 16) ? tiles : 1 << 16), 1024, 0, s>>>(
      part, strips, D, dw, accumulate);
  return launch_status();
}

}  // namespace
}  // namespace lda

using namespace lda;

extern "C" int lda_add_norm(const void *x, int64_t ld_x, const void *residual,
                            int64_t ld_residual, const void *weight, void *out, int64_t ld_out,
                            void *sum, int64_t ld_sum, float *scale, int64_t N, int32_t D,
                            int32_t dtype, int32_t weight_dtype, int32_t out_dtype, double eps,
                            void *stream) {
  if (N < 0 || D <= 0) return LDA_ERR_SHAPE;
  if (N > LDA_MAX_N) return LDA_ERR_UNSUPPORTED;
  const int size = dtype_size(dtype), weight_size = dtype_size(weight_dtype);
  if (!size || !weight_size || (out_dtype != LDA_I8 && !dtype_size(out_dtype)) ||
      !positive_finite(eps))
    return LDA_ERR_VALUE;
  if (ld_x < 0 || ld_out < D || (residual && ld_residual < 0) || (sum && ld_sum < D))
    return LDA_ERR_VALUE;
  if (sum && sum == out) return LDA_ERR_VALUE;
  const bool bits8 = out_dtype == LDA_I8;
  if ((weight_dtype != dtype && weight_dtype != LDA_F32) || (!bits8 && out_dtype != dtype))
    return LDA_ERR_UNSUPPORTED;
  if (N == 0) return LDA_OK;
  if (!x || !weight || !out || (bits8 && !scale)) return LDA_ERR_NULL;
  if (!aligned(x, size) || !aligned(residual, size) || !aligned(weight, weight_size) ||
      !aligned(out, bits8 ? 1 : size) || !aligned(sum, size) || (bits8 && !aligned(scale, 4)))
    return LDA_ERR_ALIGN;
  hipStream_t s = static_cast<hipStream_t>(stream);
#define LDA_RUN(T)                                                                             \
  run_norm<T>(x, ld_x, residual, ld_residual, weight, out, ld_out, sum, ld_sum, scale, N, D,   \
              weight_dtype == LDA_F32, bits8, eps, s)
  switch (dtype) {
    case LDA_F32: return LDA_RUN(F32);
    case LDA_BF16: return LDA_RUN(Bf16);
    default: return LDA_RUN(F16);
  }
#undef LDA_RUN
}

extern "C" size_t lda_norm_grad_workspace_bytes(int64_t N, int32_t D) {
  if (N <= 0 || D <= 0 || N > LDA_MAX_N) return 0;
  return joins_strips(N, D) ? 4 * (size_t)strips_of(N, D) * (size_t)D : 0;
}

extern "C" int lda_norm_grad(const void *grad, int64_t ld_grad, const void *h, int64_t ld_h,
                             const void *residual_grad, int64_t ld_residual, const void *weight,
                             void *dx, int64_t ld_dx, float *dweight, int64_t N, int32_t D,
                             int32_t dtype, int32_t weight_dtype, double eps, int32_t accumulate,
                             void *workspace, size_t workspace_bytes, void *stream) {
  if (N < 0 || D <= 0) return LDA_ERR_SHAPE;
  if (N > LDA_MAX_N) return LDA_ERR_UNSUPPORTED;
  const int size = dtype_size(dtype), weight_size = dtype_size(weight_dtype);
  if (!size || !weight_size || !positive_finite(eps)) return LDA_ERR_VALUE;
  if (ld_grad < 0 || ld_h < 0 || (residual_grad && ld_residual < 0) || ld_dx < D)
    return LDA_ERR_VALUE;
  if (weight_dtype != dtype && weight_dtype != LDA_F32) return LDA_ERR_UNSUPPORTED;
  const size_t need = lda_norm_grad_workspace_bytes(N, D);
  if (!dweight || (N > 0 && (!grad || !h || !weight || !dx)) || (need > 0 && !workspace))
    return LDA_ERR_NULL;
  if (!aligned(grad, size) || !aligned(h, size) || !aligned(residual_grad, size) ||
      !aligned(weight, weight_size) || !aligned(dx, size) || !aligned(dweight, 4) ||
      !aligned(workspace, 8))
    return LDA_ERR_ALIGN;
  if (workspace_bytes < need) return LDA_ERR_WORKSPACE;
  hipStream_t s = static_cast<hipStream_t>(stream);
#define LDA_RUN(T)                                                                              \
  launch_norm_grad<T>(grad, ld_grad, h, ld_h, residual_grad, ld_residual, weight, dx, ld_dx,    \
                      dweight, N, D, weight_dtype == LDA_F32, eps, accumulate != 0,             \
                      (float *)workspace, s)
  switch (dtype) {
    case LDA_F32: return LDA_RUN(F32);
    case LDA_BF16: return LDA_RUN(Bf16);
    default: return LDA_RUN(F16);
  }
#undef LDA_RUN
}

extern "C" int lda_quantise_rows(const void *x, int64_t ld_x, int8_t *q, int64_t ld_q,
                                 float *scale, int64_t N, int32_t D, int32_t dtype,
                                 void *stream) {
  if (N < 0 || D <= 0) return LDA_ERR_SHAPE;
  if (N > LDA_MAX_N) return LDA_ERR_UNSUPPORTED;
  const int size = dtype_size(dtype);
  if (!size || ld_x < 0 || ld_q < D) return LDA_ERR_VALUE;
  if (N == 0) return LDA_OK;
  if (!x || !q || !scale) return LDA_ERR_NULL;
  if (!aligned(x, size) || !aligned(scale, 4)) return LDA_ERR_ALIGN;
  hipStream_t s = static_cast<hipStream_t>(stream);
  switch (dtype) {
    case LDA_F32: return launch_quantise<F32>(x, ld_x, q, ld_q, scale, N, D, s);
    case LDA_BF16: return launch_quantise<Bf16>(x, ld_x, q, ld_q, scale, N, D, s);
    default: return launch_quantise<F16>(x, ld_x, q, ld_q, scale, N, D, s);
  }
}
