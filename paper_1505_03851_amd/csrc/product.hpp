// Products of 8-bit rows with 8-bit weights:
//
//   out[m][n] = (sum over k of q[m][k] w[n][k]) scale[m] weight_scale[n] + bias[n]
//
// The sums are whole numbers in 32 bits, exact (K is at most 131,071); they become
// float once, take the two scales and the bias there, and are rounded to the output's
// type.  Both operands have k contiguous, as v_mfma_i32_16x16x64_i8 takes them: lane l
// holds 16 bytes of row l % 16 from k = 16 (l / 16) on.  The weights are its first
// operand, so that a lane's four sums are those of four channels next to each other:
// row l % 16 of q, channels 4 (l / 16) + 0 .. 3.
//
// direct_product_kernel: a tile of 16 MT rows and 16 NT channels to a workgroup, whose
// wavefronts share the length of K and read what they multiply straight into
// registers; their sums meet in LDS (whole numbers: in any order the same).
#pragma once

#include "elements.hpp"

namespace lda {

typedef int32_t ints4 __attribute__((ext_vector_type(4)));
typedef ints4 ints4_any __attribute__((aligned(1), may_alias));

constexpr int kStep = 64;  // bytes of K that one matrix instruction takes

template <typename T>
struct ProductArgs {
  const int8_t *q, *w;
  const float *scale, *weight_scale, *bias;
  typename T::store *out;
  int64_t ldq, ldw, ldo, M;
  int32_t N, K;
};

// 16 bytes at p, of which only the first n are read where n < 16 (the rest: 0).
__device__ __forceinline__ ints4 load_bytes(const int8_t *p, int n) {
  if (n >= 16) return *reinterpret_cast<const ints4_any *>(p);
  ints4 v = {0, 0, 0, 0};
#pragma unroll
  for (int j = 0; j < 16; ++j)
    if (j < n) v[j / 4] |= (int)((uint32_t)(uint8_t)p[j] << (8 * (j % 4)));
  return v;
}

template <typename T, int MT, int NT>
__global__ __launch_bounds__(512) void direct_product_kernel(ProductArgs<T> a, uint32_t col_tiles, int64_t tiles) {
  constexpr int kRows = 16 * MT, kCols = 16 * NT, kPitch = kCols + 4;
  __shared__ int32_t joined[kRows * kPitch];
  const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int waves = (int)blockDim.x >> 6;
  const int line = lane & 15, part = lane >> 4;
  // this wavefront's share of K, in steps; the last may be a piece of one
  const int steps = (a.K + kStep - 1) / kStep;
  const int from = (int)((int64_t)steps * wave / waves), to = (int)((int64_t)steps * (wave + 1) / waves);
  const int whole = to * kStep <= a.K ? to : to - 1;
  for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
    const int64_t row_tile = tile / col_tiles;
    const int64_t m0 = row_tile * kRows, n0 = (tile - row_tile * col_tiles) * kCols;
    for (int i = (int)threadIdx.x; i < kRows * kPitch; i += (int)blockDim.x) joined[i] = 0;
    const int8_t *q[MT], *w[NT];
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const int64_t m = m0 + 16 * i + line;
      q[i] = a.q + (m < a.M ? m : a.M - 1) * a.ldq + 16 * part;
    }
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      const int64_t n = n0 + 16 * j + line;
      w[j] = a.w + (n < a.N ? n : a.N - 1) * a.ldw + 16 * part;
    }
    ints4 sum[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < NT; ++j) sum[i][j] = ints4{0, 0, 0, 0};
#pragma unroll(MT * NT >= 8 ? 2 : 4)
    for (int s = from; s < whole; ++s) {
      ints4 x[MT], y[NT];
#pragma unroll
      for (int j = 0; j < NT; ++j) y[j] = *reinterpret_cast<const ints4_any *>(w[j] + s * kStep);
#pragma unroll
      for (int i = 0; i < MT; ++i) x[i] = *reinterpret_cast<const ints4_any *>(q[i] + s * kStep);
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j)
          sum[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(y[j], x[i], sum[i][j], 0, 0, 0);
    }
    if (from < to && whole < to) {
      const int n = a.K - whole * kStep - 16 * part;
      ints4 x[MT], y[NT];
#pragma unroll
      for (int j = 0; j < NT; ++j) y[j] = load_bytes(w[j] + whole * kStep, n);
#pragma unroll
      for (int i = 0; i < MT; ++i) x[i] = load_bytes(q[i] + whole * kStep, n);
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j)
          sum[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(y[j], x[i], sum[i][j], 0, 0, 0);
    }
    __syncthreads();  // cleared
    if (from < to) {
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            atomicAdd(&joined[(16 * i + line) * kPitch + 16 * j + 4 * part + r], sum[i][j][r]);
    }
    __syncthreads();
    for (int i = (int)threadIdx.x; i < kRows * kCols; i += (int)blockDim.x) {
      const int64_t m = m0 + i / kCols, n = n0 + i % kCols;
      if (m >= a.M || n >= a.N) continue;
      float v = (float)joined[(i / kCols) * kPitch + i % kCols] * a.scale[m] * a.weight_scale[n];
      if (a.bias) v += a.bias[n];
      a.out[m * a.ldo + n] = T::down(v);
    }
    __syncthreads();  // read before the next tile clears it
  }
}

}  // namespace lda
