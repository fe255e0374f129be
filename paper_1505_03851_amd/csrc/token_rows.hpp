// Rows of activations: the embedding lookup (gathered, scaled, dropped out)
// and the dropout of any rows.
//
//   embed    out[n][c] = table[word_id[n]][c] * f * kept(n, c)
//   dropout  out[n][c] = x[n][c] * f * kept(n, c)
//
// with f = scale / P(kept) in float, one rounding to the tensor's type; what is
// not kept is 0 whatever it was (an infinity or NaN too), and a word outside
// [0, V) gives a row of zeros.  Both are bound by memory: each lane takes 8
// columns of kRowsEach rows, all loads before the first store.  (Philox's products
// take 25 us of vector instructions on 67M elements, under the 33 us of memory.)
//
// Measured on MI355X: 16,384 rows of 4,096 bfloat16 out of 100,000, dropped out,
// 32.5 us (5.8 TB/s of the 187 MB that have to move); 32,768 rows of 4,096 dropped
// out 85 us (6.3 TB/s of 537 MB); 64 rows of 1,024, 3.4 us on the GPU and 8 a call.
#pragma once

#include "elements.hpp"
#include "keep_bits.hpp"

namespace lda {

constexpr int kRowThreads = 256;
constexpr int kRowsEach = 4;  // rows of one lane, loaded together

// A workgroup covers (256 >> lanes_log2) * kRowsEach rows and
// 8 << lanes_log2 columns; `col_tiles` such tiles cover a row.  WIDE: lanes_log2
// is 6 or more, so a wavefront's rows are known to scalar registers.
template <typename T, bool GATHER, bool DROP, bool WIDE>
__global__ __launch_bounds__(kRowThreads) void rows_kernel(
    const typename T::store *x, int64_t ldx, const int32_t *__restrict__ word_id,
    typename T::store *out, int64_t ldo, int64_t N, int32_t V, int64_t D, float factor,
    Dropout drop, int lanes_log2, uint32_t col_tiles, int64_t tiles) {
  // What passes the caches by, whatever its size: rows looked up are stored so, and
  // 16-bit rows dropped out are read and stored so.  Alone, 16,384 rows of 4,096
  // bfloat16 looked up take 35 us against 45, 32,768 dropped out 86 against 94, 2,048
  // 7.0 against 9.2; 8,192 float rows looked up 43 against 49 where few words are
  // frequent but 54 against 47 where all are alike; float rows dropped out 105
  // against 98, since a lane's 32 bytes are two accesses to one line.  With a kernel
  // after it that reads what was written: 64 rows of 1,024 bfloat16 looked up 4.9
  // against 4.7, 2,048 of 4,096 16.7 against 16.3, 32,768 170 against 176; dropped
  // out 5.4 against 5.2, 17.1 against 18.1, 178 against 181; 2,048 of 4,096 floats
  // looked up 27 against 24.
  constexpr bool kStreamStore = GATHER || sizeof(typename T::store) == 2;
  constexpr bool kStreamLoad = !GATHER && sizeof(typename T::store) == 2;
  const int lane = (int)threadIdx.x & ((1 << lanes_log2) - 1);
  const int own_slot = (int)threadIdx.x >> lanes_log2;
  const int slot = WIDE ? __builtin_amdgcn_readfirstlane(own_slot) : own_slot;
  const int slots = kRowThreads >> lanes_log2;
  for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
    const int64_t row_tile = tile / col_tiles;
    const int64_t col = (((tile - row_tile * col_tiles) << lanes_log2) + lane) * 8;
    if (col >= D) continue;
    const int n = D - col < 8 ? (int)(D - col) : 8;
    const int64_t first = row_tile * slots * kRowsEach + slot;
    float v[kRowsEach][8];
#pragma unroll
    for (int r = 0; r < kRowsEach; ++r) {
      const int64_t row = first + (int64_t)r * slots;
      int64_t from = row;
      bool there = row < N;
      if (GATHER && there) {
        const int32_t w = word_id[row];
        there = (uint32_t)w < (uint32_t)V;
        from = w;
      }
      load_elements<T, 8, kStreamLoad>(x + (there ? from * ldx + col : 0), there ? n : 0, v[r]);
    }
#pragma unroll
    for (int r = 0; r < kRowsEach; ++r) {
      const int64_t row = first + (int64_t)r * slots;
      if (row >= N) break;
      if (DROP) {
        const KeepWords k = keep_words((uint32_t)(col >> 3), (uint32_t)row, drop);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[r][j] = k.kept(j, drop.q) ? v[r][j] * factor : 0.0f;
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[r][j] *= factor;
      }
      store_elements<T, 8, kStreamStore>(out + row * ldo + col, n, v[r]);
    }
  }
}

}  // namespace lda
