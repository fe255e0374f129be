// Host side and C ABI of the sampling from logits by uniform numbers (gfx950): argument
// checks and the launch.  Device code: sampling.hpp, elements.hpp, wave_ops.hpp.
#include <hip/hip_runtime.h>

#include <stdint.h>

#include "lda_draw.h"
#include "status.hpp"
#include "arguments.hpp"
#include "sampling.hpp"

namespace lda {
namespace {

constexpr int64_t kSlice = 1 << 20;  // rows of a launch: fewer than 2^32 work-items

// The digits of a weight: V of them, each at most 2^digits, add up in 64 bits.
int weight_digits(int32_t V) {
  int bits = 0;
  while (bits < 31 && ((int64_t)1 << bits) < V) ++bits;
  return bits > 17 ? 63 - bits : 46;
}

template <typename T>
int launch_sample(const void *logits, int64_t ld, int64_t B, int32_t V, const float *u,
                  const float *temperature, const int32_t *top_k, const float *top_p,
                  const float *min_p, int32_t *z, float *prob, hipStream_t s) {
  // chunks of a lane that stay in registers: 4 or as many as fit in 64
  constexpr int kMost = 64 / (2 * (int)sizeof(typename T::store));
  const int64_t chunks = ((int64_t)V + 8 * kSampleThreads - 1) / (8 * kSampleThreads);
  for (int64_t at = 0; at < B; at += kSlice) {
    const auto from = [&](const auto *p) { return p ? p + at : p; };
#define LDA_SAMPLE(CHUNKS)                                                                      \
  sample_kernel<T, CHUNKS><<<(unsigned)(B - at < kSlice ? B - at : kSlice), kSampleThreads, 0,  \
                             s>>>((const typename T::store *)logits + at * ld, ld, V,           \
                                  weight_digits(V), u + at, from(temperature), from(top_k),     \
                                  from(top_p), from(min_p), z + at, prob + at)
    if (chunks <= 4)
      LDA_SAMPLE(4);
    else if (chunks <= kMost)
      LDA_SAMPLE(kMost);
    else
      LDA_SAMPLE(0);
#undef LDA_SAMPLE
  }
  return launch_status();
}

}  // namespace
}  // namespace lda

using namespace lda;

extern "C" int lda_sample_logits(const void *logits, int64_t ld_logits, int64_t B, int32_t V,
                                 int32_t dtype, const float *u, const float *temperature,
                                 const int32_t *top_k, const float *top_p, const float *min_p,
                                 int32_t *z, float *prob, void *stream) {
  if (B < 0 || V <= 0) return LDA_ERR_SHAPE;
  if (B > LDA_LOGITS_MAX_ROWS) return LDA_ERR_UNSUPPORTED;
  const int size = dtype_size(dtype);
  if (!size || ld_logits < 0) return LDA_ERR_VALUE;
  if (B == 0) return LDA_OK;
  if (!logits || !u || !z || !prob) return LDA_ERR_NULL;
  if (!aligned(logits, size) || !aligned(u, 4) || !aligned(temperature, 4) || !aligned(top_k, 4) ||
      !aligned(top_p, 4) || !aligned(min_p, 4) || !aligned(z, 4) || !aligned(prob, 4))
    return LDA_ERR_ALIGN;
  hipStream_t s = static_cast<hipStream_t>(stream);
#define LDA_RUN(T) \
  launch_sample<T>(logits, ld_logits, B, V, u, temperature, top_k, top_p, min_p, z, prob, s)
  switch (dtype) {
    case LDA_F32: return LDA_RUN(F32);
    case LDA_BF16: return LDA_RUN(Bf16);
    default: return LDA_RUN(F16);
  }
#undef LDA_RUN
}
