// Checks of arguments that the host sides share.
#pragma once

#include <math.h>
#include <stdint.h>

#include "lda_draw.h"

namespace lda {

inline bool aligned(const void *p, int bytes) {
  return !(reinterpret_cast<uintptr_t>(p) & (uintptr_t)(bytes - 1));
}

// Bytes of an element of rows (0: no such type, or not one of rows' own).
inline int dtype_size(int32_t dtype) {
  switch (dtype) {
    case LDA_F32: return 4;
    case LDA_BF16:
    case LDA_F16: return 2;
    default: return 0;
  }
}

// (as the kernels take it, in float)
inline bool positive_finite(double v) { return (float)v > 0.0f && isfinite((float)v); }

}  // namespace lda
