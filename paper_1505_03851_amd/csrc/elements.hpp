// Elements of the token operators' tensors: float, bfloat16 and half in
// memory, float in registers.
//
// A lane reads and writes W consecutive elements of a row (W a power of two up
// to 8: 16 bytes of a 16-bit type).  Rows start at any element (odd widths, row
// strides), so the vector types are declared at the element's alignment: the
// hardware takes such loads and stores in one instruction.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace lda {

struct F32 {
  using store = float;
  static __device__ __forceinline__ float up(float v) { return v; }
  static __device__ __forceinline__ float down(float v) { return v; }
};

struct Bf16 {
  using store = uint16_t;
  static __device__ __forceinline__ float up(uint16_t v) {
    return __builtin_bit_cast(float, (uint32_t)v << 16);
  }
  // round to nearest even (the hardware's conversion; NaN stays NaN)
  static __device__ __forceinline__ uint16_t down(float v) {
    return __builtin_bit_cast(uint16_t, (__bf16)v);
  }
};

struct F16 {
  using store = uint16_t;
  static __device__ __forceinline__ float up(uint16_t v) {
    return (float)__builtin_bit_cast(_Float16, v);
  }
  static __device__ __forceinline__ uint16_t down(float v) {
    return __builtin_bit_cast(uint16_t, (_Float16)v);
  }
};

// W elements of a row as one value of BYTES, which may lie at any element: the
// types are declared at 2 bytes' alignment.
typedef uint32_t words2 __attribute__((ext_vector_type(2)));
typedef uint32_t words4 __attribute__((ext_vector_type(4)));
typedef uint32_t words8 __attribute__((ext_vector_type(8)));
typedef uint32_t words1_any __attribute__((aligned(2), may_alias));
typedef words2 words2_any __attribute__((aligned(2), may_alias));
typedef words4 words4_any __attribute__((aligned(2), may_alias));
typedef words8 words8_any __attribute__((aligned(2), may_alias));
typedef uint16_t half_any __attribute__((may_alias));

template <int BYTES>
struct Raw;
template <>
struct Raw<2> {
  using type = uint16_t;
  using memory = half_any;
};
template <>
struct Raw<4> {
  using type = uint32_t;
  using memory = words1_any;
};
template <>
struct Raw<8> {
  using type = words2;
  using memory = words2_any;
};
template <>
struct Raw<16> {
  using type = words4;
  using memory = words4_any;
};
template <>
struct Raw<32> {
  using type = words8;
  using memory = words8_any;
};

template <typename T, int W>
struct Packed {
  typename T::store v[W];
};

// p[0 .. W) as it is in memory; only the first `n` are read (the rest: 0)
// where n < W.  STREAM: what is read or written passes the caches by, so that it
// does not put out what they hold, nor wait for what they have to write back; meant
// for what is larger than they are and touched once.
template <typename T, int W, bool STREAM = false>
__device__ __forceinline__ Packed<T, W> load_packed(const typename T::store *p, int n) {
  using R = Raw<W * (int)sizeof(typename T::store)>;
  Packed<T, W> a;
  if (n >= W) {
    const auto *memory = reinterpret_cast<const typename R::memory *>(p);
    const typename R::type raw = STREAM ? __builtin_nontemporal_load(memory) : *memory;
    a = __builtin_bit_cast(Packed<T, W>, raw);
  } else {
#pragma unroll
    for (int j = 0; j < W; ++j) a.v[j] = j < n ? p[j] : typename T::store(0);
  }
  return a;
}

// p[0 .. W) -> x in float
template <typename T, int W, bool STREAM = false>
__device__ __forceinline__ void load_elements(const typename T::store *p, int n, float (&x)[W]) {
  const Packed<T, W> a = load_packed<T, W, STREAM>(p, n);
#pragma unroll
  for (int j = 0; j < W; ++j) x[j] = T::up(a.v[j]);
}

template <typename T, int W, bool STREAM = false>
__device__ __forceinline__ void store_elements(typename T::store *p, int n, const float (&x)[W]) {
  using R = Raw<W * (int)sizeof(typename T::store)>;
  if (n >= W) {
    Packed<T, W> a;
#pragma unroll
    for (int j = 0; j < W; ++j) a.v[j] = T::down(x[j]);
    auto *memory = reinterpret_cast<typename R::memory *>(p);
    if (STREAM)
      __builtin_nontemporal_store(__builtin_bit_cast(typename R::type, a), memory);
    else
      *memory = __builtin_bit_cast(typename R::type, a);
  } else {
#pragma unroll
    for (int j = 0; j < W; ++j)
      if (j < n) p[j] = T::down(x[j]);
  }
}

}  // namespace lda
