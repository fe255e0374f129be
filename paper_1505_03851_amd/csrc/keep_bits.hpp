// The dropout mask, made where it is used and never stored.
//
// Eight neighbouring columns of a row share one Philox4x32-10 call (Salmon,
// Moraes, Dror and Shaw, SC 2011; philox.hpp has the rounds): counter
// (col / 8, row, step, 1), key (seed mod 2^32, seed >> 32).  Column c takes
// half c % 2 (low half first) of output word (c % 8) / 2 and is kept if that
// 16-bit number is at least q = round(65536 p), so the probability of keeping
// it is exactly (65536 - q) / 65536, and the factor of what is kept is the
// reciprocal of that: the expectation is exact for the p in use, which is at
// most 2^-17 away from the p asked for.  (With 32 bits to an element the ten
// rounds of integer products, not memory, would bound a 16-bit tensor.)
// The counter's last word, 1, keeps these numbers apart from the topic draws'
// (0) and the token draws' (2 and 3).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace lda {

struct Dropout {
  uint32_t q;     // kept where the 16-bit number >= q
  uint32_t step;  // the counter's third word
  uint32_t k0, k1;
};

// The four words of columns 8 group .. 8 group + 7 of `row`.  Where `row` is
// the same for a wavefront (in scalar registers) and `group` the same for
// several rows, the compiler keeps two and a half of the ten rounds out of the
// loop or in scalar registers: the counter's other words are uniform, and a
// round mixes only two of the four.
struct KeepWords {
  uint32_t w[4];

  // whether column 8 group + j is kept; j is known at compile time (an odd
  // column's number is the word's upper half, which the whole word's comparison
  // with q << 16 decides)
  __device__ __forceinline__ bool kept(int j, uint32_t q) const {
    return j & 1 ? w[j >> 1] >= q << 16 : (uint16_t)w[j >> 1] >= (uint16_t)q;
  }

  // bit j: whether column 8 group + j is kept
  __device__ __forceinline__ uint32_t bits(uint32_t q) const {
    uint32_t b = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) b |= (uint32_t)kept(j, q) << j;
    return b;
  }
};

__device__ __forceinline__ KeepWords keep_words(uint32_t group, uint32_t row, const Dropout &d) {
  uint32_t x0 = group, x1 = row, x2 = d.step, x3 = 1u, k0 = d.k0, k1 = d.k1;
#pragma unroll
  for (int round = 0; round < 10; ++round) {
    const uint64_t p0 = (uint64_t)0xD2511F53u * x0;
    const uint64_t p1 = (uint64_t)0xCD9E8D57u * x2;
    const uint32_t y0 = (uint32_t)(p1 >> 32) ^ x1 ^ k0;
    const uint32_t y2 = (uint32_t)(p0 >> 32) ^ x3 ^ k1;
    x1 = (uint32_t)p1;
    x3 = (uint32_t)p0;
    x0 = y0;
    x2 = y2;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return KeepWords{{x0, x1, x2, x3}};
}

}  // namespace lda
