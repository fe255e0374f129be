// The embedding's gradient by sorted tokens:
//
//   G[v][c] = f * sum over the tokens n with word_id[n] = v, in order, of
//             grad[n][c] where (n, c) was kept,             f = scale / P(kept)
//
// summed in float and rounded once (added to what G holds where the caller
// accumulates).  The tokens are first sorted by word, stably (digits from the
// lowest, each pass a histogram and a scatter over chunks of kSortChunk), so a
// word's tokens are neighbours in token order.  Then a wavefront takes `chunk`
// sorted positions and a tile of 64 W columns, adds the rows of one word in
// registers and writes a word's row when it ends.  A word that crosses a chunk
// leaves its part in `part` (slot 2 c: the head of chunk c, a word that began
// before; 2 c + 1: its tail, a word that goes on), and join_kernel adds those in
// order.  No sum depends on the order in which workgroups run.
#pragma once

#include "elements.hpp"
#include "keep_bits.hpp"

namespace lda {

constexpr int kSortThreads = 1024;
constexpr int kSortWaves = kSortThreads / 64;
constexpr int kSortEach = 4;
constexpr int kSortChunk = kSortThreads * kSortEach;  // tokens of one workgroup
constexpr int kSortMaxBits = 10;                      // bits of a digit
constexpr int kSortMaxBins = 1 << kSortMaxBits;

// a token's key: its word, or V (sorted last, given no gradient) outside [0, V)
__device__ __forceinline__ uint32_t sort_key(const int32_t *word_id, const uint32_t *key,
                                             int64_t i, int32_t V) {
  if (key) return key[i];
  const int32_t w = word_id[i];
  return (uint32_t)w < (uint32_t)V ? (uint32_t)w : (uint32_t)V;
}

// hist[chunk][digit]: the tokens of each chunk with each digit
__global__ __launch_bounds__(kSortThreads) void sort_hist_kernel(
    const int32_t *__restrict__ word_id, const uint32_t *__restrict__ key, int64_t N, int32_t V,
    int shift, int bits, uint32_t *__restrict__ hist, uint32_t *crossing) {
  __shared__ uint32_t count[kSortMaxBins];
  const int bins = 1 << bits;
  if (crossing && blockIdx.x == 0 && threadIdx.x == 0) *crossing = 0;
  for (int b = threadIdx.x; b < bins; b += kSortThreads) count[b] = 0;
  __syncthreads();
  const int64_t first = (int64_t)blockIdx.x * kSortChunk;
#pragma unroll
  for (int r = 0; r < kSortEach; ++r) {
    const int64_t i = first + r * kSortThreads + threadIdx.x;
    if (i < N) atomicAdd(&count[sort_key(word_id, key, i, V) >> shift & (bins - 1)], 1u);
  }
  __syncthreads();
  for (int b = threadIdx.x; b < bins; b += kSortThreads)
    hist[(int64_t)blockIdx.x * bins + b] = count[b];
}

// Exclusive sum of one value per thread over the workgroup, by thread index.
__device__ __forceinline__ uint32_t block_exclusive_sum(uint32_t v, uint32_t *wave_sums) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint32_t s = v;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t o = __shfl_up(s, d);
    if (lane >= d) s += o;
  }
  if (lane == 63) wave_sums[wave] = s;
  __syncthreads();
  uint32_t before = 0;
  for (int w = 0; w < wave; ++w) before += wave_sums[w];
  __syncthreads();
  return before + s - v;
}

// Many chunks: hist[c][b] becomes the tokens of digit b in the chunks before c,
// total[b] those of all.  A workgroup takes 64 digits, each wavefront a run of
// chunks.
__global__ __launch_bounds__(kSortThreads) void sort_scan_kernel(uint32_t *hist, uint32_t *total,
                                                                 uint32_t chunks, int bins) {
  __shared__ uint32_t sums[kSortWaves][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int b = (int)blockIdx.x * 64 + lane;
  const uint32_t each = (chunks + kSortWaves - 1) / kSortWaves;
  const uint32_t from = wave * each < chunks ? wave * each : chunks;
  const uint32_t to = from + each < chunks ? from + each : chunks;
  uint32_t s = 0;
  if (b < bins)
    for (uint32_t c = from; c < to; ++c) s += hist[(int64_t)c * bins + b];
  sums[wave][lane] = s;
  __syncthreads();
  uint32_t before = 0, all = 0;
  for (int w = 0; w < kSortWaves; ++w) {
    before += w < wave ? sums[w][lane] : 0;
    all += sums[w][lane];
  }
  if (b >= bins) return;
  if (wave == 0) total[b] = all;
  for (uint32_t c = from; c < to; ++c) {
    const uint32_t h = hist[(int64_t)c * bins + b];
    hist[(int64_t)c * bins + b] = before;
    before += h;
  }
}

// The tokens of one chunk to their places by one digit: the chunk's base for
// the digit, and the token's rank among the chunk's tokens of that digit, by
// wavefront (a wavefront holds 64 kSortEach neighbours), round and lane.
__global__ __launch_bounds__(kSortThreads) void sort_scatter_kernel(
    const int32_t *__restrict__ word_id, const uint32_t *__restrict__ key,
    const uint32_t *__restrict__ index, int64_t N, int32_t V, int shift, int bits,
    const uint32_t *__restrict__ hist, const uint32_t *__restrict__ total,
    uint32_t *__restrict__ key_out,
    uint32_t *__restrict__ index_out) {
  __shared__ uint32_t base[kSortMaxBins];
  __shared__ uint16_t count[kSortWaves][kSortMaxBins];
  __shared__ uint32_t wave_sums[kSortWaves];
  const int bins = 1 << bits;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int b = lane; b < bins; b += 64) count[wave][b] = 0;
  // this digit's tokens of all chunks (to place the digit) and of earlier
  // chunks: from sort_scan_kernel, or (few chunks) summed here
  uint32_t all = 0, before = 0;
  if ((int)threadIdx.x < bins && total) {
    all = total[threadIdx.x];
    before = hist[(int64_t)blockIdx.x * bins + threadIdx.x];
  } else if ((int)threadIdx.x < bins) {
    for (uint32_t c = 0; c < gridDim.x; ++c) {
      const uint32_t h = hist[(int64_t)c * bins + threadIdx.x];
      all += h;
      before += c < blockIdx.x ? h : 0;
    }
  }
  const uint32_t place = block_exclusive_sum(all, wave_sums);
  if ((int)threadIdx.x < bins) base[threadIdx.x] = place + before;
  const int64_t first = (int64_t)blockIdx.x * kSortChunk + wave * 64 * kSortEach + lane;
  uint32_t k[kSortEach], rank[kSortEach];
#pragma unroll
  for (int r = 0; r < kSortEach; ++r) {
    const int64_t i = first + 64 * r;
    k[r] = i < N ? sort_key(word_id, key, i, V) : 0;
    const uint32_t digit = k[r] >> shift & (bins - 1);
    uint64_t same = __ballot(i < N);
    for (int b = 0; b < bits; ++b) {
      const uint64_t set = __ballot(digit >> b & 1);
      same &= digit >> b & 1 ? set : ~set;
    }
    const uint64_t below = same & ((1ull << lane) - 1);
    const uint32_t prior = count[wave][digit];
    rank[r] = prior + __popcll(below);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    if (i < N && below == 0) count[wave][digit] = (uint16_t)(prior + __popcll(same));
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
  __syncthreads();
  for (int b = threadIdx.x; b < bins; b += kSortThreads) {
    uint32_t s = 0;
    for (int w = 0; w < kSortWaves; ++w) {
      const uint32_t c = count[w][b];
      count[w][b] = (uint16_t)s;
      s += c;
    }
  }
  __syncthreads();
#pragma unroll
  for (int r = 0; r < kSortEach; ++r) {
    const int64_t i = first + 64 * r;
    if (i >= N) break;
    const uint32_t digit = k[r] >> shift & (bins - 1);
    const uint32_t at = base[digit] + count[wave][digit] + rank[r];
    key_out[at] = k[r];
    index_out[at] = index ? index[i] : (uint32_t)i;
  }
}

// rows [0, V) of `out` to zero, D elements each
template <typename T>
__global__ __launch_bounds__(256) void clear_rows_kernel(typename T::store *out, int64_t ldo,
                                                         int32_t V, int32_t D) {
  const int64_t cols = (D + 7) / 8, units = cols * V;
  const float zero[8] = {};
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < units;
       i += (int64_t)gridDim.x * 256) {
    const int64_t row = i / cols;
    const int32_t col = (int32_t)(i - row * cols) * 8;
    store_elements<T, 8>(out + row * ldo + col, D - col, zero);
  }
}

// The sorted tokens and what is left of them.
struct GradPlan {
  const uint32_t *key, *index;  // [N], by word and then by token
  uint32_t N;
  uint32_t V;
  uint32_t chunk, chunks;  // sorted positions of a wavefront, and how many
  float *part;             // [2 chunks][ld_part]
  int64_t ld_part;
  uint32_t *crossing;  // [0]: how many, then the chunks in which a word that
                       // goes past the chunk's end begins
};

template <typename TO, int W>
__device__ __forceinline__ void write_row(typename TO::store *out, int64_t ldo, uint32_t word,
                                          int32_t col, int n, float factor, bool accumulate,
                                          float (&sum)[W]) {
  typename TO::store *p = out + (int64_t)word * ldo + col;
  float old[W] = {};
  if (accumulate) load_elements<TO, W>(p, n, old);
#pragma unroll
  for (int j = 0; j < W; ++j) sum[j] = accumulate ? fmaf(sum[j], factor, old[j]) : sum[j] * factor;
  store_elements<TO, W>(p, n, sum);
}

// One wavefront: `chunk` sorted positions, 64 W columns.
template <typename TG, typename TO, int W, bool DROP>
__global__ __launch_bounds__(256) void reduce_kernel(const typename TG::store *__restrict__ grad,
                                                     int64_t ldg, typename TO::store *out,
                                                     int64_t ldo, int32_t D, float factor,
                                                     Dropout drop, bool accumulate,
                                                     uint32_t col_tiles, GradPlan g) {
  constexpr int U = 8;  // rows loaded together
  const int lane = threadIdx.x & 63;
  const uint32_t item = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
  const uint32_t c = item / col_tiles;
  if (c >= g.chunks) return;
  const uint32_t tile = item - c * col_tiles;
  const int32_t col = (int32_t)(tile * 64 + lane) * W;
  const int n = D - col < W ? (D - col > 0 ? D - col : 0) : W;
  const uint32_t begin = c * g.chunk;
  const uint32_t end = g.N - begin < g.chunk ? g.N : begin + g.chunk;
  bool began_here = begin == 0 || g.key[begin - 1] != g.key[begin];
  float sum[W] = {};
  for (uint32_t p = begin; p < end; p += U) {
    float v[U][W];
    uint32_t row[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const uint32_t at = p + u < end ? p + u : end - 1;
      row[u] = g.index[at];
      load_elements<TG, W>(grad + (int64_t)row[u] * ldg + (n ? col : 0), n, v[u]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (p + u >= end) break;
      const uint32_t word = g.key[p + u];
      if (word >= g.V) return;  // from here on only tokens without a word
      uint32_t kept = 0;
      if (DROP) kept = keep_bits((uint32_t)col >> 3, row[u], drop) >> (col & 7);
#pragma unroll
      for (int j = 0; j < W; ++j) sum[j] += !DROP || (kept >> j & 1) ? v[u][j] : 0.0f;
      const bool goes_on = p + u + 1 < g.N && g.key[p + u + 1] == word;
      if (goes_on && p + u + 1 < end) continue;
      if (began_here && !goes_on) {
        if (n) write_row<TO, W>(out, ldo, word, col, n, factor, accumulate, sum);
      } else {
        float *slot = g.part + (int64_t)(2 * c + (began_here ? 1 : 0)) * g.ld_part + col;
        if (n) store_elements<F32, W>(slot, W, sum);
        if (began_here && tile == 0 && lane == 0)
          g.crossing[1 + atomicAdd(g.crossing, 1u)] = c;
      }
      began_here = true;
#pragma unroll
      for (int j = 0; j < W; ++j) sum[j] = 0.0f;
    }
  }
}

// The words that cross chunks: each one's parts added in order.  The four
// wavefronts of a workgroup take a quarter of the parts each.
template <typename TO, int W>
__global__ __launch_bounds__(256) void join_kernel(typename TO::store *out, int64_t ldo, int32_t D,
                                                   float factor, bool accumulate,
                                                   uint32_t col_tiles, GradPlan g) {
  __shared__ float quarter[3][64 * W];
  const int lane = threadIdx.x & 63;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t items = g.crossing[0] * col_tiles;
  for (uint32_t item = blockIdx.x; item < items; item += gridDim.x) {
    const uint32_t i = item / col_tiles;
    const int32_t col = (int32_t)((item - i * col_tiles) * 64 + lane) * W;
    const int n = D - col < W ? (D - col > 0 ? D - col : 0) : W;
    const uint32_t c0 = g.crossing[1 + i];
    const uint32_t word = g.key[(c0 + 1) * g.chunk - 1];
    uint32_t lo = (c0 + 1) * g.chunk, hi = g.N;  // the first position past the word
    while (lo < hi) {
      const uint32_t mid = lo + (hi - lo) / 2;
      if (g.key[mid] == word)
        lo = mid + 1;
      else
        hi = mid;
    }
    const uint32_t parts = (lo - 1) / g.chunk - c0 + 1;
    const uint32_t each = (parts + 3) / 4;
    const uint32_t from = wave * each, to = from + each < parts ? from + each : parts;
    float sum[W] = {};
    for (uint32_t k = from; k < to; ++k) {
      float v[W];
      const uint32_t slot = 2 * (c0 + k) + (k == 0 ? 1 : 0);
      load_elements<F32, W>(g.part + (int64_t)slot * g.ld_part + (n ? col : 0), n ? W : 0, v);
#pragma unroll
      for (int j = 0; j < W; ++j) sum[j] += v[j];
    }
    if (wave > 0) {
#pragma unroll
      for (int j = 0; j < W; ++j) quarter[wave - 1][j * 64 + lane] = sum[j];
    }
    __syncthreads();
    if (wave == 0 && n) {
#pragma unroll
      for (int j = 0; j < W; ++j)
        for (int q = 0; q < 3; ++q) sum[j] += quarter[q][j * 64 + lane];
      write_row<TO, W>(out, ldo, word, col, n, factor, accumulate, sum);
    }
    __syncthreads();
  }
}

}  // namespace lda
