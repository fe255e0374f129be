// Rows normed by their root mean square, the gradient of that, and rows in 8 bits.
//
//   norm      h = x + residual,  s = 1 / sqrt(mean(h^2) + eps),  y = h s w
//   gradient  u = h s, d = dy w:  dx = s (d - u mean(d u)) [+ residual_grad],
//             dw = the sum over the rows of dy u
//   8 bits    q = y 127 / max |y| to the nearest whole number (halves to the even
//             one), scale = max |y| / 127
//
// A row is read once and stays in registers as float: UNITS units of 8 columns a
// lane, in one wavefront (four rows to a workgroup) or in one workgroup of WAVES.
// Longer rows are read again from the caches (the *_long kernels).
//
// The gradient of w is summed by workgroup over a strip of rows, in registers, and
// the strips' sums by a second launch, each in an order fixed by the sizes alone:
// the same call gives the same bits.
#pragma once

#include "elements.hpp"
#include "wave_ops.hpp"

namespace lda {

typedef words2 words2_byte __attribute__((aligned(1), may_alias));

constexpr int kNormThreads = 256;
constexpr int kLongThreads = 1024;

// Sums (or, of float bits, the largest) over the WAVES wavefronts of a workgroup.
// `turn` alternates between calls, so that one barrier a call will do.
template <int WAVES>
__device__ __forceinline__ float row_sum(float v, float (&shared)[2][16], int turn) {
  v = wave_sum(v);
  if (WAVES == 1) return v;
  if ((threadIdx.x & 63) == 0) shared[turn][threadIdx.x >> 6] = v;
  __syncthreads();
  float all = 0.0f;
#pragma unroll
  for (int i = 0; i < WAVES; ++i) all += shared[turn][i];
  return all;
}

__device__ __forceinline__ uint32_t wave_largest(uint32_t v) {
  return wave_reduce(v, 0u, [](uint32_t a, uint32_t b) { return a > b ? a : b; });
}

template <int WAVES>
__device__ __forceinline__ uint32_t row_largest(uint32_t v, uint32_t (&shared)[16]) {
  v = wave_largest(v);
  if (WAVES == 1) return v;
  if ((threadIdx.x & 63) == 0) shared[threadIdx.x >> 6] = v;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < WAVES; ++i) v = shared[i] > v ? shared[i] : v;
  return v;
}

__device__ __forceinline__ uint32_t magnitude(float v) {
  return __builtin_bit_cast(uint32_t, v) & 0x7FFFFFFFu;
}

// How a row is put into 8 bits, from the bits of its largest magnitude (those of an
// infinity or NaN are above all others).
struct Steps {
  float shift;    // a power of two that keeps 127 / top and 127 x in range
  float top;      // the largest magnitude, shifted
  float inverse;  // 1 / top (0: every q is 0)
  float scale;    // what a step stands for: top / 127; NaN if the row holds a NaN or infinity
};

__device__ __forceinline__ Steps steps_of(uint32_t top_bits) {
  const float top = __builtin_bit_cast(float, top_bits);
  Steps s;
  s.shift = top_bits < 0x0D800000u ? 0x1p100f : top_bits > 0x71800000u ? 0x1p-60f : 1.0f;
  const bool finite = top_bits < 0x7F800000u;
  s.top = finite ? top * s.shift : 0.0f;
  s.inverse = s.top > 0.0f ? 1.0f / s.top : 0.0f;
  s.scale = finite ? top / 127.0f : __builtin_nanf("");
  return s;
}

// The nearest step of a value.  127 x / top is half a step above a whole number for every
// x = top / 2, and for many x where top's digits have a factor 127, so the side of
// the half is decided exactly.  16-bit x: 127 x is exact, and one correction of the
// quotient by its remainder (exact too) rounds it rightly; the nearest half is then
// either met or 2^-12 away.  Float: the sign of 127 x - (floor + 1/2) top, of which
// fma gives every digit.
template <typename T>
__device__ __forceinline__ int exact_step_of(float x, const Steps &s) {
  x *= s.shift;
  const float p = 127.0f * x, t = p * s.inverse;
  if constexpr (sizeof(typename T::store) == 2) {
    return (int)rintf(__builtin_fmaf(__builtin_fmaf(-t, s.top, p), s.inverse, t));
  } else {
    const float low = __builtin_fmaf(127.0f, x, -p);
    const float f = floorf(t);
    const float above = __builtin_fmaf(-(f + 0.5f), s.top, p) + low;
    const int q = (int)f;
    return s.inverse > 0.0f ? q + ((above > 0.0f || (above == 0.0f && (q & 1))) ? 1 : 0) : 0;
  }
}

// The same of 8 floats (the norm's, which were rounded on their way and are seldom next to a
// half), in the low bytes of q.  Two roundings leave the quotient off by 127 * 2 * 2^-24 at
// most, so only within 2^-16 of a half is the side decided exactly: about one in 64 times of a
// wavefront's 512 columns.
__device__ __forceinline__ void exact_steps_of(const float (&x)[8], const Steps &s, int (&q)[8]) {
  constexpr float kWhole = 0x1.8p23f;  // what rounds to whole numbers, in the last bits
  const float per = 127.0f * s.inverse;
  float furthest = 0.0f;  // from a whole number
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float v = x[j] * s.shift, t = __builtin_fmaf(v, per, kWhole);
    furthest = fmaxf(furthest, fabsf(__builtin_fmaf(v, per, -(t - kWhole))));
    q[j] = __builtin_bit_cast(int, t);
  }
  if (furthest > 0.5f - 0x1p-16f || !(s.inverse > 0.0f)) {
#pragma unroll
    for (int j = 0; j < 8; ++j) q[j] = exact_step_of<F32>(x[j], s);
  }
}

// q[0 .. n) of 8 steps
__device__ __forceinline__ void store_steps(int8_t *p, int n, const int (&q)[8]) {
  if (n >= 8) {
    words2 w;
#pragma unroll
    for (int j = 0; j < 2; ++j)
      w[j] = ((uint32_t)q[4 * j] & 0xFFu) | ((uint32_t)q[4 * j + 1] & 0xFFu) << 8 |
             ((uint32_t)q[4 * j + 2] & 0xFFu) << 16 | (uint32_t)q[4 * j + 3] << 24;
    *reinterpret_cast<words2_byte *>(p) = w;
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < n) p[j] = (int8_t)q[j];
  }
}

template <typename I>
__device__ __forceinline__ int columns_left(I D, I col) {
  return D - col < 0 ? 0 : D - col < 8 ? (int)(D - col) : 8;
}

// The weight may be of the rows' type or float.
template <typename T>
__device__ __forceinline__ void load_weight(const void *w, bool w_float, int64_t col, int n,
                                            float (&v)[8]) {
  if (sizeof(typename T::store) == 4 || w_float)
    load_elements<F32, 8>((const float *)w + (n > 0 ? col : 0), n, v);
  else
    load_elements<T, 8>((const typename T::store *)w + (n > 0 ? col : 0), n, v);
}

// The 8 columns of a lane's unit in a row of D >= 8: those from `at` on, of which the first
// `skip` are not its own.  The last unit of a row whose length is no multiple of 8 starts
// where its 8 columns end with the row's, and a unit past the end has none of its own: so
// every lane loads 16 bytes at once, without a branch that loads would have to wait in.
struct Columns {
  int at, skip;
  __device__ __forceinline__ Columns() {}
  __device__ __forceinline__ Columns(int D, int unit)
      : at(unit * 8 <= D - 8 ? unit * 8 : D - 8),
        skip(unit * 8 <= D - 8 ? 0 : unit * 8 < D ? 8 - (D - unit * 8) : 8) {}
};

// Zero in the columns that are not the unit's own.
__device__ __forceinline__ void own_columns(const Columns &c, float (&x)[8]) {
#pragma unroll
  for (int j = 0; j < 8; ++j) x[j] = j >= c.skip ? x[j] : 0.0f;
}

template <typename T, bool STREAM = false>
__device__ __forceinline__ void load_columns(const typename T::store *row, const Columns &c,
                                             float (&x)[8]) {
  load_elements<T, 8, STREAM>(row + c.at, 8, x);
  own_columns(c, x);
}

template <typename T>
__device__ __forceinline__ void load_weight_columns(const void *w, bool w_float, const Columns &c,
                                                    float (&v)[8]) {
  load_weight<T>(w, w_float, c.at, 8, v);
  own_columns(c, v);
}

template <typename T, bool STREAM = false>
__device__ __forceinline__ void store_columns(typename T::store *row, const Columns &c,
                                              const float (&x)[8]) {
  if (c.skip == 0) {
    store_elements<T, 8, STREAM>(row + c.at, 8, x);
  } else {
#pragma unroll
    for (int j = 1; j < 8; ++j)
      if (j >= c.skip) row[c.at + j] = T::down(x[j]);
  }
}

__device__ __forceinline__ void store_step_columns(int8_t *row, const Columns &c, const int (&q)[8]) {
  if (c.skip == 0) {
    store_steps(row + c.at, 8, q);
  } else {
#pragma unroll
    for (int j = 1; j < 8; ++j)
      if (j >= c.skip) row[c.at + j] = (int8_t)q[j];
  }
}

// What a launch of the norm works on.  `residual` and `sum` (where h goes) may be NULL.
template <typename T>
struct NormArgs {
  const typename T::store *x, *residual;
  const void *weight;
  void *out;
  typename T::store *sum;
  float *scale;
  int64_t ldx, ldr, ldo, lds, N;
  int32_t D;
  float eps;
  bool weight_float;
};

// BITS8: out is int8, with a scale for each row.  STREAM: rows pass the caches by.
template <typename T, int WAVES, int UNITS, bool BITS8, bool STREAM>
__global__ __launch_bounds__(WAVES == 1 ? kNormThreads : 64 * WAVES) void norm_kernel(
    NormArgs<T> a) {
  using S = typename T::store;
  __shared__ float sums[2][16];
  __shared__ uint32_t tops[16];
  constexpr int kLanes = 64 * WAVES;
  const int lane = (int)threadIdx.x & (kLanes - 1);
  const int64_t row =
      WAVES == 1 ? (int64_t)blockIdx.x * (kNormThreads / 64) +
                       __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6)
                 : (int64_t)blockIdx.x;
  if (row >= a.N) return;  // (a whole wavefront; workgroups of one row are never here)
  const S *x = a.x + row * a.ldx;
  float h[UNITS][8];
  Columns c[UNITS];
#pragma unroll
  for (int u = 0; u < UNITS; ++u) {
    c[u] = Columns(a.D, u * kLanes + lane);
    load_columns<T, STREAM>(x, c[u], h[u]);
  }
  if (a.residual) {
    const S *r = a.residual + row * a.ldr;
#pragma unroll
    for (int u = 0; u < UNITS; ++u) {
      float v[8];
      load_columns<T, STREAM>(r, c[u], v);
#pragma unroll
      for (int j = 0; j < 8; ++j) h[u][j] += v[j];
    }
  }
  float square = 0.0f;
#pragma unroll
  for (int u = 0; u < UNITS; ++u)
#pragma unroll
    for (int j = 0; j < 8; ++j) square = __builtin_fmaf(h[u][j], h[u][j], square);
  const float s = 1.0f / sqrtf(row_sum<WAVES>(square, sums, 0) / (float)a.D + a.eps);
  if (a.sum) {
#pragma unroll
    for (int u = 0; u < UNITS; ++u) store_columns<T, STREAM>(a.sum + row * a.lds, c[u], h[u]);
  }
  uint32_t top = 0;
#pragma unroll
  for (int u = 0; u < UNITS; ++u) {
    float w[8];
    load_weight_columns<T>(a.weight, a.weight_float, c[u], w);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      h[u][j] = h[u][j] * s * w[j];
      if (BITS8 && j >= c[u].skip) top = magnitude(h[u][j]) > top ? magnitude(h[u][j]) : top;
    }
    if (!BITS8) store_columns<T, STREAM>((S *)a.out + row * a.ldo, c[u], h[u]);
  }
  if (BITS8) {
    const Steps steps = steps_of(row_largest<WAVES>(top, tops));
    if (lane == 0) a.scale[row] = steps.scale;
#pragma unroll
    for (int u = 0; u < UNITS; ++u) {
      int q[8];
      exact_steps_of(h[u], steps, q);
      store_step_columns((int8_t *)a.out + row * a.ldo, c[u], q);
    }
  }
}

// A row of any length, one workgroup to a row: h is made again in each pass.
template <typename T, bool BITS8>
__global__ __launch_bounds__(kLongThreads) void norm_long_kernel(NormArgs<T> a) {
  using S = typename T::store;
  __shared__ float sums[2][16];
  __shared__ uint32_t tops[16];
  constexpr int kWaves = kLongThreads / 64;
  const int64_t D = a.D;
  int turn = 0;
  for (int64_t row = blockIdx.x; row < a.N; row += gridDim.x) {
    const S *x = a.x + row * a.ldx, *r = a.residual + (a.residual ? row * a.ldr : 0);
    const auto load = [&](int64_t col, int n, float (&h)[8]) {
      load_elements<T, 8>(x + col, n, h);
      if (a.residual) {
        float v[8];
        load_elements<T, 8>(r + col, n, v);
#pragma unroll
        for (int j = 0; j < 8; ++j) h[j] += v[j];
      }
    };
    float square = 0.0f;
    for (int64_t col = (int64_t)threadIdx.x * 8; col < D; col += kLongThreads * 8) {
      float h[8];
      load(col, columns_left(D, col), h);
#pragma unroll
      for (int j = 0; j < 8; ++j) square = __builtin_fmaf(h[j], h[j], square);
    }
    const float s = 1.0f / sqrtf(row_sum<kWaves>(square, sums, turn) / (float)D + a.eps);
    turn ^= 1;
    Steps steps{};
    if (BITS8) {
      uint32_t top = 0;
      for (int64_t col = (int64_t)threadIdx.x * 8; col < D; col += kLongThreads * 8) {
        const int n = columns_left(D, col);
        float h[8], w[8];
        load(col, n, h);
        load_weight<T>(a.weight, a.weight_float, col, n, w);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const uint32_t m = magnitude(h[j] * s * w[j]);
          if (j < n) top = m > top ? m : top;
        }
      }
      steps = steps_of(row_largest<kWaves>(top, tops));
      if (threadIdx.x == 0) a.scale[row] = steps.scale;
      __syncthreads();  // `tops` is read before the next row writes it
    }
    for (int64_t col = (int64_t)threadIdx.x * 8; col < D; col += kLongThreads * 8) {
      const int n = columns_left(D, col);
      float h[8], w[8];
      load(col, n, h);
      load_weight<T>(a.weight, a.weight_float, col, n, w);
      if (a.sum) store_elements<T, 8>(a.sum + row * a.lds + col, n, h);
#pragma unroll
      for (int j = 0; j < 8; ++j) h[j] = h[j] * s * w[j];
      if (BITS8) {
        int q[8];
        exact_steps_of(h, steps, q);
        store_steps((int8_t *)a.out + row * a.ldo + col, n, q);
      } else {
        store_elements<T, 8>((S *)a.out + row * a.ldo + col, n, h);
      }
    }
  }
}

// ---- the gradient

template <typename T>
struct NormGradArgs {
  const typename T::store *grad, *h, *residual;
  const void *weight;
  typename T::store *dx;
  float *part;  // [workgroups][D]: the strips' sums of dw, or dw itself where there is one
  bool add;     // to what is there (one strip)
  int64_t ldg, ldh, ldr, ldx, N;
  int32_t D;
  float eps;
  bool weight_float;
};

// WAVES wavefronts to a row, two units of 8 columns a lane; the rows of a workgroup go
// together.  The next row is on its way while this one is worked on.
template <typename T, int WAVES, bool STREAM>
__global__ __launch_bounds__(WAVES <= 4 ? kNormThreads : 64 * WAVES) void norm_grad_kernel(
    NormGradArgs<T> a) {
  constexpr int kUnits = 2, kLanes = 64 * WAVES;
  constexpr int kThreads = WAVES <= 4 ? kNormThreads : 64 * WAVES, kRows = kThreads / kLanes;
  constexpr int kColumns = kLanes * kUnits * 8;
  __shared__ float sums[2][2][16];
  __shared__ float joined[kRows > 1 ? kColumns : 1];
  const int lane = kRows > 1 ? (int)threadIdx.x & (kLanes - 1) : (int)threadIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), slot = kRows > 1 ? wave / WAVES : 0;
  Columns c[kUnits];
  float w[kUnits][8], dw[kUnits][8];
#pragma unroll
  for (int u = 0; u < kUnits; ++u) {
    c[u] = Columns(a.D, u * kLanes + lane);
    load_weight_columns<T>(a.weight, a.weight_float, c[u], w[u]);
#pragma unroll
    for (int j = 0; j < 8; ++j) dw[u][j] = 0.0f;
  }
  struct Row {
    Packed<T, 8> d[kUnits], h[kUnits], r[kUnits];
  };
  const auto load = [&](int64_t row) {
    const int64_t at = row < a.N ? row : a.N - 1;  // (the last one again: its results are not used)
    Row v;
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
      v.d[u] = load_packed<T, 8, STREAM>(a.grad + at * a.ldg + c[u].at, 8);
      v.h[u] = load_packed<T, 8, STREAM>(a.h + at * a.ldh + c[u].at, 8);
      if (a.residual) v.r[u] = load_packed<T, 8, STREAM>(a.residual + at * a.ldr + c[u].at, 8);
    }
    return v;
  };
  const int64_t step = (int64_t)gridDim.x * kRows;
  int64_t row = (int64_t)blockIdx.x * kRows + slot;
  Row next = load(row);
  int turn = 0;
  for (int64_t base = (int64_t)blockIdx.x * kRows; base < a.N; base += step, row += step) {
    const Row now = next;
    next = load(row + step);
    float d[kUnits][8], h[kUnits][8];
    float square = 0.0f, along = 0.0f;
    const bool there = row < a.N;
#pragma unroll
    for (int u = 0; u < kUnits; ++u)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        // (h too where there is no row: what was loaded in its place, the last row again, another
        // wavefront may just be writing over with an infinite dx)
        const bool own = there && j >= c[u].skip;
        d[u][j] = own ? T::up(now.d[u].v[j]) : 0.0f;
        h[u][j] = own ? T::up(now.h[u].v[j]) : 0.0f;
        square = __builtin_fmaf(h[u][j], h[u][j], square);
        along = __builtin_fmaf(d[u][j] * w[u][j], h[u][j], along);
      }
    square = wave_sum(square);
    along = wave_sum(along);
    if (WAVES > 1) {
      if ((threadIdx.x & 63) == 0) {
        sums[turn][0][wave] = square;
        sums[turn][1][wave] = along;
      }
      __syncthreads();
      square = along = 0.0f;
#pragma unroll
      for (int i = 0; i < WAVES; ++i) {
        square += sums[turn][0][slot * WAVES + i];
        along += sums[turn][1][slot * WAVES + i];
      }
      turn ^= 1;  // (one barrier a row: the other half is read before this one is written again)
    }
    const float s = 1.0f / sqrtf(square / (float)a.D + a.eps);
    const float pull = along * s / (float)a.D;  // mean(d u)
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
      float dx[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float unit = h[u][j] * s;
        dw[u][j] = __builtin_fmaf(d[u][j], unit, dw[u][j]);
        dx[j] = s * __builtin_fmaf(-unit, pull, d[u][j] * w[u][j]);
        if (a.residual) dx[j] += T::up(now.r[u].v[j]);
      }
      if (there) store_columns<T, STREAM>(a.dx + row * a.ldx, c[u], dx);
    }
  }
  // the workgroup's strip: its rows' wavefronts one after another
  float *part = a.part + (int64_t)blockIdx.x * a.D;
  if (kRows > 1) {
    for (int r = 0; r < kRows; ++r) {
      if (slot == r) {
#pragma unroll
        for (int u = 0; u < kUnits; ++u)
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            if (j < c[u].skip) continue;
            float &to = joined[c[u].at + j];
            to = r == 0 ? dw[u][j] : to + dw[u][j];
          }
      }
      __syncthreads();
    }
    for (int c = (int)threadIdx.x; c < a.D; c += kThreads) part[c] = a.add ? part[c] + joined[c] : joined[c];
  } else {
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
      if (a.add) {
        float before[8];
        load_columns<F32>(part, c[u], before);
#pragma unroll
        for (int j = 0; j < 8; ++j) dw[u][j] += before[j];
      }
      store_columns<F32>(part, c[u], dw[u]);
    }
  }
}

// A row of any length: read twice, the strip's sums in the workspace.
template <typename T>
__global__ __launch_bounds__(kLongThreads) void norm_grad_long_kernel(NormGradArgs<T> a) {
  __shared__ float sums[2][2][16];
  constexpr int kWaves = kLongThreads / 64;
  const int64_t D = a.D;
  float *part = a.part + (int64_t)blockIdx.x * D;
  int turn = 0;
  for (int64_t row = blockIdx.x; row < a.N; row += gridDim.x) {
    const auto *g = a.grad + row * a.ldg, *x = a.h + row * a.ldh;
    float square = 0.0f, along = 0.0f;
    for (int64_t col = (int64_t)threadIdx.x * 8; col < D; col += kLongThreads * 8) {
      const int n = columns_left(D, col);
      float d[8], h[8], w[8];
      load_elements<T, 8>(g + col, n, d);
      load_elements<T, 8>(x + col, n, h);
      load_weight<T>(a.weight, a.weight_float, col, n, w);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        square = __builtin_fmaf(h[j], h[j], square);
        along = __builtin_fmaf(d[j] * w[j], h[j], along);
      }
    }
    square = row_sum<kWaves>(square, sums[0], turn);
    along = row_sum<kWaves>(along, sums[1], turn);
    turn ^= 1;
    const float s = 1.0f / sqrtf(square / (float)D + a.eps);
    const float pull = along * s / (float)D;
    for (int64_t col = (int64_t)threadIdx.x * 8; col < D; col += kLongThreads * 8) {
      const int n = columns_left(D, col);
      float d[8], h[8], w[8], r[8] = {}, dw[8] = {};
      load_elements<T, 8>(g + col, n, d);
      load_elements<T, 8>(x + col, n, h);
      load_weight<T>(a.weight, a.weight_float, col, n, w);
      if (a.residual) load_elements<T, 8>(a.residual + row * a.ldr + col, n, r);
      if (row != (int64_t)blockIdx.x) load_elements<F32, 8>(part + col, n, dw);
      float dx[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float unit = h[j] * s;
        dw[j] = __builtin_fmaf(d[j], unit, dw[j]);
        dx[j] = s * __builtin_fmaf(-unit, pull, d[j] * w[j]) + r[j];
      }
      store_elements<F32, 8>(part + col, n, dw);
      store_elements<T, 8>(a.dx + row * a.ldx + col, n, dx);
    }
  }
}

// dw of 64 columns: the strips' sums, 16 wavefronts each taking every 16th in order,
// then those 16.
__global__ __launch_bounds__(1024) void join_strips_kernel(const float *__restrict__ part,
                                                           int32_t strips, int32_t D, float *dw,
                                                           bool accumulate) {
  __shared__ float sums[16][64];
  const int lane = (int)threadIdx.x & 63, wave = (int)threadIdx.x >> 6;
  for (int64_t first = (int64_t)blockIdx.x * 64; first < D; first += (int64_t)gridDim.x * 64) {
    const int64_t col = first + lane;
    float v = 0.0f;
    if (col < D)
#pragma unroll 8
      for (int i = wave; i < strips; i += 16) v += part[(int64_t)i * D + col];
    sums[wave][lane] = v;
    __syncthreads();
    if (wave == 0 && col < D) {
      float all = 0.0f;
#pragma unroll
      for (int i = 0; i < 16; ++i) all += sums[i][lane];
      dw[col] = accumulate ? dw[col] + all : all;
    }
    __syncthreads();
  }
}

// ---- rows in 8 bits

template <typename T>
struct QuantArgs {
  const typename T::store *x;
  int8_t *q;
  float *scale;
  int64_t ldx, ldq, N;
  int32_t D;
};

template <typename T, int WAVES, int UNITS>
__global__ __launch_bounds__(WAVES == 1 ? kNormThreads : 64 * WAVES) void quantise_kernel(
    QuantArgs<T> a) {
  __shared__ uint32_t tops[16];
  constexpr int kLanes = 64 * WAVES;
  const int lane = (int)threadIdx.x & (kLanes - 1);
  const int64_t row =
      WAVES == 1 ? (int64_t)blockIdx.x * (kNormThreads / 64) +
                       __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6)
                 : (int64_t)blockIdx.x;
  if (row >= a.N) return;  // (a whole wavefront; workgroups of one row are never here)
  float x[UNITS][8];
  Columns c[UNITS];
  uint32_t top = 0;
#pragma unroll
  for (int u = 0; u < UNITS; ++u) {
    c[u] = Columns(a.D, u * kLanes + lane);
    load_columns<T>(a.x + row * a.ldx, c[u], x[u]);
  }
#pragma unroll
  for (int u = 0; u < UNITS; ++u)
#pragma unroll
    for (int j = 0; j < 8; ++j) top = magnitude(x[u][j]) > top ? magnitude(x[u][j]) : top;
  const Steps steps = steps_of(row_largest<WAVES>(top, tops));
  if (lane == 0) a.scale[row] = steps.scale;
#pragma unroll
  for (int u = 0; u < UNITS; ++u) {
    int q[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) q[j] = steps.inverse > 0.0f ? exact_step_of<T>(x[u][j], steps) : 0;
    store_step_columns(a.q + row * a.ldq, c[u], q);
  }
}

template <typename T>
__global__ __launch_bounds__(kLongThreads) void quantise_long_kernel(QuantArgs<T> a) {
  __shared__ uint32_t tops[16];
  const int64_t D = a.D;
  for (int64_t row = blockIdx.x; row < a.N; row += gridDim.x) {
    const auto *p = a.x + row * a.ldx;
    uint32_t top = 0;
    for (int64_t col = (int64_t)threadIdx.x * 8; col < D; col += kLongThreads * 8) {
      float x[8];
      load_elements<T, 8>(p + col, columns_left(D, col), x);
#pragma unroll
      for (int j = 0; j < 8; ++j) top = magnitude(x[j]) > top ? magnitude(x[j]) : top;
    }
    const Steps steps = steps_of(row_largest<kLongThreads / 64>(top, tops));
    if (threadIdx.x == 0) a.scale[row] = steps.scale;
    for (int64_t col = (int64_t)threadIdx.x * 8; col < D; col += kLongThreads * 8) {
      const int n = columns_left(D, col);
      float x[8];
      int q[8];
      load_elements<T, 8>(p + col, n, x);
#pragma unroll
      for (int j = 0; j < 8; ++j) q[j] = steps.inverse > 0.0f ? exact_step_of<T>(x[j], steps) : 0;
      store_steps(a.q + row * a.ldq + col, n, q);
    }
    __syncthreads();  // `tops` is read before the next row writes it
  }
}

}  // namespace lda
