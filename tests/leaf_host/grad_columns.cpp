// The columns of the embedding gradient's lanes (grad_columns.hpp) on the CPU.
//
//   grad_columns D   every lane of the first and last tiles of rows of D columns:
//                    what it reads lies in the row, at most a tile from the
//                    wavefront's first column, and the columns it writes are the
//                    row's, each once
#include "hip/hip_runtime.h"

#include "grad_columns.hpp"

template <int W>
int check(int64_t D) {
  using namespace lda;
  const int64_t tiles = column_tiles<W>(D);
  int64_t next = 0;  // the first column that no lane has written
  for (int64_t t = 0; t < tiles; ++t) {
    if (t == 2 && tiles > 6) {
      t = tiles - 3;
      next = t * 64 * W;
    }
    for (unsigned lane = 0; lane < 64; ++lane) {
      emu::thread_idx.x = 64 + lane;  // (of the workgroup's second wavefront)
      const Columns<W> c((uint32_t)t, (int32_t)D);
      const int64_t at = (int64_t)c.first + c.offset;
      if (c.col < 0 || c.col + (int64_t)W > D || at != c.col || c.offset >= 64 * W) {
        printf("W %d, tile %lld, lane %u reads from %d (%lld)\n", W, (long long)t, lane, c.col,
               (long long)at);
        return 1;
      }
      const int64_t own = c.own;
      if (c.n < 0 || c.n > W || (c.n > 0 && (own != next || own + c.n > D))) {
        printf("W %d, tile %lld, lane %u writes %d from %lld\n", W, (long long)t, lane, c.n,
               (long long)own);
        return 1;
      }
      // (a lane with a part of its columns has them at the end of those it reads)
      if (c.n > 0 && own + c.n != (c.n == W ? c.col + (int64_t)W : D)) return 1;
      next += c.n;
    }
  }
  if (next != D) printf("W %d: %lld of %lld columns written\n", W, (long long)next, (long long)D);
  return next != D;
}

int main(int argc, char **argv) {
  const int64_t D = atoll(argv[1]);
  return check<1>(D) || (D >= 2 && check<2>(D)) || (D >= 4 && check<4>(D)) ||
         (D >= 8 && check<8>(D));
}
