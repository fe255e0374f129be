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
//
// Measured on MI355X: 1M tokens of 256 bfloat16 over 32,768 Zipf words 167 us (3.3
// TB/s of the 558 MB that have to move): the sums 115 us at 4.7 TB/s, bound by
// memory, the sort 42, a chain of six launches, and the joins 11; 32,768 tokens
// of 2,048 bfloat16 into 50,000 float rows, dropped out, 130 us (4.2 TB/s): clearing
// at 4.9 TB/s with the sort under it, then 47 of sums (added to what is there: 89 us,
// the rows that occur alone); 4,096 tokens of 1,000
// floats 23 us, three launches of 4 to 10 us, each a few round trips; up to 128
// tokens of 512 columns into 10,000 rows 6 us, one into 400 MB 64 (6.3 TB/s).
#pragma once

#include "elements.hpp"
#include "grad_columns.hpp"
#include "keep_bits.hpp"
#include "wave_ops.hpp"

namespace lda {

constexpr int kSortThreads = 1024;
constexpr int kSortWaves = kSortThreads / 64;
constexpr int kSortEach = 4;
constexpr int kSortChunk = kSortThreads * kSortEach;  // tokens of one workgroup
constexpr int kSortMaxBits = 10;                      // bits of a digit
constexpr int kSortMaxBins = 1 << kSortMaxBits;

// The share of the gradient's rows that a sorting launch sets to zero, in its
// workgroups past those that sort: the sort is a chain of short launches bound
// by latency, the clearing one long store, and the two do not touch the same
// memory, so each launch of the chain carries a part of it.
struct ClearShare {
  char *out;
  int64_t ld, width, rows;  // in bytes; dense rows are given as one
  uint32_t part, parts;
  uint32_t blocks;  // workgroups that sort
};

// 16 bytes from p on, or n if there are fewer, to zero.  STREAM: past the caches,
// so that the gradient's reads do not wait for them to write zeros back (32,768
// tokens of 2,048 columns into 50,000 float rows: 127 us against 140; the rows of
// few_kernel, one by one and with little to read, 94 against 79).
template <bool STREAM>
__device__ __forceinline__ void clear_bytes(char *p, int64_t n) {
  auto *memory = reinterpret_cast<words4_any *>(p);
  if (n >= 16 && STREAM) {
    __builtin_nontemporal_store(words4{}, memory);
  } else if (n >= 16) {
    *memory = words4{};
  } else {
    for (int64_t j = 0; j < n; j += 2) *reinterpret_cast<half_any *>(p + j) = 0;
  }
}

__device__ __forceinline__ void clear_share(const ClearShare &c) {
  const int64_t units = (c.width + 15) >> 4, all = units * c.rows;
  const int64_t end = all * (c.part + 1) / c.parts;
  for (int64_t i = all * c.part / c.parts + (int64_t)(blockIdx.x - c.blocks) * kSortThreads +
                   threadIdx.x;
       i < end; i += (int64_t)(gridDim.x - c.blocks) * kSortThreads) {
    const int64_t row = c.rows == 1 ? 0 : i / units;
    const int64_t at = (i - row * units) << 4;
    clear_bytes<true>(c.out + row * c.ld + at, c.width - at);
  }
}

// A token to be sorted, kept and moved as one value of 8 bytes: its word, or V
// (sorted last, given no gradient) outside [0, V), and its number.
struct alignas(8) Token {
  uint32_t word, number;
};

// token i as the pass before left it, or (the first pass) from word_id
__device__ __forceinline__ Token load_token(const int32_t *word_id, const Token *sorted, int64_t i,
                                            int32_t V) {
  if (sorted) return sorted[i];
  const int32_t w = word_id[i];
  return Token{(uint32_t)w < (uint32_t)V ? (uint32_t)w : (uint32_t)V, (uint32_t)i};
}

// hist[chunk][digit]: the tokens of each chunk with each digit
__global__ __launch_bounds__(kSortThreads) void sort_hist_kernel(
    const int32_t *__restrict__ word_id, const Token *__restrict__ sorted, int64_t N, int32_t V,
    int shift, int bits, uint32_t *__restrict__ hist, uint32_t *crossing, ClearShare clear) {
  __shared__ uint32_t count[kSortMaxBins];
  if (blockIdx.x >= clear.blocks) {
    clear_share(clear);
    return;
  }
  const int bins = 1 << bits;
  if (crossing && blockIdx.x == 0 && threadIdx.x == 0) *crossing = 0;
  const int64_t first = (int64_t)blockIdx.x * kSortChunk;
  uint32_t k[kSortEach];
#pragma unroll
  for (int r = 0; r < kSortEach; ++r) {
    const int64_t i = first + r * kSortThreads + threadIdx.x;
    k[r] = i < N ? load_token(word_id, sorted, i, V).word : 0;
  }
  for (int b = threadIdx.x; b < bins; b += kSortThreads) count[b] = 0;
  __syncthreads();
#pragma unroll
  for (int r = 0; r < kSortEach; ++r)
    if (first + r * kSortThreads + threadIdx.x < N) atomicAdd(&count[k[r] >> shift & (bins - 1)], 1u);
  __syncthreads();
  for (int b = threadIdx.x; b < bins; b += kSortThreads)
    hist[(int64_t)blockIdx.x * bins + b] = count[b];
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
  if (b < bins) {
#pragma unroll 8
    for (uint32_t c = from; c < to; ++c) s += hist[(int64_t)c * bins + b];
  }
  sums[wave][lane] = s;
  __syncthreads();
  uint32_t before = 0, all = 0;
  for (int w = 0; w < kSortWaves; ++w) {
    before += w < wave ? sums[w][lane] : 0;
    all += sums[w][lane];
  }
  if (b >= bins) return;
  if (wave == 0) total[b] = all;
  constexpr int U = 8;
  for (uint32_t c = from; c < to; c += U) {
    uint32_t h[U];
#pragma unroll
    for (int u = 0; u < U; ++u) h[u] = c + u < to ? hist[(int64_t)(c + u) * bins + b] : 0;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (c + u < to) hist[(int64_t)(c + u) * bins + b] = before;
      before += h[u];
    }
  }
}

// Exclusive sum of one value per thread over the workgroup, by thread index.
__device__ __forceinline__ uint32_t block_exclusive_sum(uint32_t v, uint32_t *wave_sums) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint32_t s = wave_inclusive_sum(v);
  if (lane == 63) wave_sums[wave] = s;
  __syncthreads();
  uint32_t before = 0;
#pragma unroll
  for (int w = 0; w < kSortWaves; ++w) before += w < wave ? wave_sums[w] : 0;
  __syncthreads();
  return before + s - v;
}

struct SortLds {
  uint32_t base[kSortMaxBins];
  uint16_t count[kSortWaves][kSortMaxBins];
  uint32_t wave_sums[kSortWaves];
};

// A chunk's `n` tokens among the workgroup's threads: a wavefront holds 64
// rounds(n) neighbours, 64 to a round; token 64 r + the place of its first in the
// chunk is the lane's of round r.
__device__ __forceinline__ int rounds_of(int n) { return (n + kSortThreads - 1) / kSortThreads; }

__device__ __forceinline__ int first_of(int rounds) {
  return (int)(threadIdx.x >> 6) * 64 * rounds + (int)(threadIdx.x & 63);
}

// Ranks by one digit of a chunk's tokens: rank[r] is the number of tokens of the
// same digit before the token in its wavefront, and count[wave][digit] becomes
// the number in the wavefronts before it.  Returns thread b's tokens of digit b in
// the whole chunk.
__device__ __forceinline__ uint32_t rank_chunk(SortLds &s, const Token (&k)[kSortEach], int n,
                                               int rounds, int shift, int bits,
                                               uint32_t (&rank)[kSortEach]) {
  const int bins = 1 << bits, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int first = first_of(rounds);
  for (int b = lane; b < bins; b += 64) s.count[wave][b] = 0;
  // the lanes of a round with the lane's digit, a ballot for each bit
  uint64_t same[kSortEach];
#pragma unroll
  for (int r = 0; r < kSortEach; ++r) {
    if (r >= rounds) break;
    const uint32_t digit = k[r].word >> shift;
    const uint64_t there = __ballot(first + 64 * r < n);
    uint32_t low = (uint32_t)there, high = (uint32_t)(there >> 32);
    for (int b = 0; b < bits; ++b) {
      const uint32_t set = (uint32_t)((int32_t)(digit << (31 - b)) >> 31);  // all ones: bit b is 1
      const uint64_t with = __ballot(set != 0);
      low &= ~((uint32_t)with ^ set);
      high &= ~((uint32_t)(with >> 32) ^ set);
    }
    same[r] = (uint64_t)high << 32 | low;
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
#pragma unroll
  for (int r = 0; r < kSortEach; ++r) {
    if (r >= rounds) break;
    const uint32_t digit = k[r].word >> shift & (bins - 1);
    const uint64_t below = same[r] & ((1ull << lane) - 1);
    const uint32_t prior = s.count[wave][digit];
    rank[r] = prior + __popcll(below);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    if (first + 64 * r < n && below == 0)
      s.count[wave][digit] = (uint16_t)(prior + __popcll(same[r]));
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
  __syncthreads();
  uint32_t all = 0;
  if ((int)threadIdx.x < bins) {
    uint32_t c[kSortWaves];
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) c[w] = s.count[w][threadIdx.x];
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) {
      s.count[w][threadIdx.x] = (uint16_t)all;
      all += c[w];
    }
  }
  return all;
}

// The tokens of one chunk to their places by one digit: the chunk's base for
// the digit, the wavefront's and the token's rank in it.
__global__ __launch_bounds__(kSortThreads) void sort_scatter_kernel(
    const int32_t *__restrict__ word_id, const Token *__restrict__ sorted, int64_t N, int32_t V,
    int shift, int bits, const uint32_t *__restrict__ hist, const uint32_t *__restrict__ total,
    Token *__restrict__ out, ClearShare clear) {
  __shared__ SortLds s;
  if (blockIdx.x >= clear.blocks) {
    clear_share(clear);
    return;
  }
  const int bins = 1 << bits, wave = threadIdx.x >> 6;
  const int64_t start = (int64_t)blockIdx.x * kSortChunk;
  const int n = N - start < kSortChunk ? (int)(N - start) : kSortChunk;
  const int rounds = rounds_of(n), first = first_of(rounds);
  Token k[kSortEach];
  uint32_t rank[kSortEach];
#pragma unroll
  for (int r = 0; r < kSortEach; ++r) {
    const int i = first + 64 * r;
    k[r] = r < rounds && i < n ? load_token(word_id, sorted, start + i, V) : Token{0, 0};
  }
  // this digit's tokens of all chunks (to place the digit) and of earlier
  // chunks: from sort_scan_kernel, or (few chunks) summed here
  uint32_t all = 0, before = 0;
  if ((int)threadIdx.x < bins && total) {
    all = total[threadIdx.x];
    before = hist[(int64_t)blockIdx.x * bins + threadIdx.x];
  } else if ((int)threadIdx.x < bins) {
#pragma unroll 8
    for (uint32_t c = 0; c < clear.blocks; ++c) {
      const uint32_t h = hist[(int64_t)c * bins + threadIdx.x];
      all += h;
      before += c < blockIdx.x ? h : 0;
    }
  }
  rank_chunk(s, k, n, rounds, shift, bits, rank);
  const uint32_t place = block_exclusive_sum(all, s.wave_sums);
  if ((int)threadIdx.x < bins) s.base[threadIdx.x] = place + before;
  __syncthreads();
#pragma unroll
  for (int r = 0; r < kSortEach; ++r) {
    if (r >= rounds || first + 64 * r >= n) break;
    const uint32_t digit = k[r].word >> shift & (bins - 1);
    out[s.base[digit] + s.count[wave][digit] + rank[r]] = k[r];
  }
}

// One chunk: every pass in one workgroup, through LDS.
__global__ __launch_bounds__(kSortThreads) void sort_chunk_kernel(
    const int32_t *__restrict__ word_id, int32_t N, int32_t V, int passes, int bits,
    Token *__restrict__ out, uint32_t *crossing, ClearShare clear) {
  __shared__ SortLds s;
  __shared__ Token tokens[kSortChunk];
  if (blockIdx.x >= clear.blocks) {
    clear_share(clear);
    return;
  }
  if (threadIdx.x == 0) *crossing = 0;
  const int wave = threadIdx.x >> 6;
  const int rounds = rounds_of(N), first = first_of(rounds);
  Token k[kSortEach];
  uint32_t rank[kSortEach];
#pragma unroll
  for (int r = 0; r < kSortEach; ++r) {
    const int i = first + 64 * r;
    k[r] = r < rounds && i < N ? load_token(word_id, nullptr, i, V) : Token{0, 0};
  }
  for (int pass = 0; pass < passes; ++pass) {
    const int shift = pass * bits;
    const uint32_t all = rank_chunk(s, k, N, rounds, shift, bits, rank);
    const uint32_t place = block_exclusive_sum(all, s.wave_sums);
    if ((int)threadIdx.x < 1 << bits) s.base[threadIdx.x] = place;
    __syncthreads();
    const bool last = pass + 1 == passes;
    Token *to = last ? out : tokens;
#pragma unroll
    for (int r = 0; r < kSortEach; ++r) {
      if (r >= rounds || first + 64 * r >= N) break;
      const uint32_t digit = k[r].word >> shift & ((1 << bits) - 1);
      to[s.base[digit] + s.count[wave][digit] + rank[r]] = k[r];
    }
    __syncthreads();
    if (last) break;
#pragma unroll
    for (int r = 0; r < kSortEach; ++r)
      if (r < rounds && first + 64 * r < N) k[r] = tokens[first + 64 * r];
    __syncthreads();
  }
}

// Nothing to sort: clearing alone.
__global__ __launch_bounds__(kSortThreads) void clear_kernel(ClearShare clear) {
  clear_share(clear);
}

// How the sorted positions are cut, and where the words that cross a cut are
// kept.
struct GradPlan {
  uint32_t N, V;
  uint32_t chunk, chunks;  // sorted positions of a wavefront, and how many
  int64_t ld_part;
};

// The last n of a lane's W sums to its n columns of the word's row, which
// begin at `own`.
template <typename TO, int W>
__device__ __forceinline__ void write_row(typename TO::store *out, int64_t ldo, uint32_t word,
                                          uint32_t own, int n, float factor, bool accumulate,
                                          float (&sum)[W]) {
  typename TO::store *p = out + (int64_t)word * ldo + own;
  if (n == W) {
    float old[W] = {};
    if (accumulate) load_elements<TO, W>(p, W, old);
#pragma unroll
    for (int j = 0; j < W; ++j) sum[j] = accumulate ? fmaf(sum[j], factor, old[j]) : sum[j] * factor;
    store_elements<TO, W>(p, W, sum);
  } else {
    p -= W - n;
#pragma unroll
    for (int j = 0; j < W; ++j)
      if (j >= W - n)
        p[j] = TO::down(accumulate ? fmaf(sum[j], factor, TO::up(p[j])) : sum[j] * factor);
  }
}

// What dropout kept of a row's W columns from `col` on, added to `sum`.
// `straddles`: some lane's columns lie in two of the mask's groups of eight.
template <typename TG, int W, bool DROP>
__device__ __forceinline__ void add_row(const Packed<TG, W> &v, uint32_t row, int32_t col,
                                        bool straddles, const Dropout &drop, float (&sum)[W]) {
  float x[W];
#pragma unroll
  for (int j = 0; j < W; ++j) x[j] = TG::up(v.v[j]);
  if (DROP) {
    const uint32_t group = (uint32_t)col >> 3;
    const KeepWords k = keep_words(group, row, drop);
    if (W == 8 && !straddles) {
#pragma unroll
      for (int j = 0; j < W; ++j) x[j] = k.kept(j, drop.q) ? x[j] : 0.0f;
    } else {
      uint32_t bits = k.bits(drop.q);
      if (straddles) bits |= keep_words(group + 1, row, drop).bits(drop.q) << 8;
      bits >>= col & 7;
#pragma unroll
      for (int j = 0; j < W; ++j) x[j] = bits >> j & 1 ? x[j] : 0.0f;
    }
  }
#pragma unroll
  for (int j = 0; j < W; ++j) sum[j] += x[j];
}

// W columns of a row, `offset` bytes into what `grad` has of it; the row's address
// stays in scalar registers.
template <typename TG, int W, bool STREAM>
__device__ __forceinline__ Packed<TG, W> load_row(const typename TG::store *grad, int64_t ldg,
                                                  uint32_t row, uint32_t offset) {
  uint64_t base = reinterpret_cast<uint64_t>(grad + (int64_t)row * ldg);
  asm("" : "+s"(base));
  const auto *p = reinterpret_cast<const __attribute__((address_space(1))) char *>(base);
  return load_packed<TG, W, STREAM>((const typename TG::store *)(p + offset), W);
}

// One wavefront: `chunk` sorted positions, 64 W columns.  It reads the words and
// row numbers of 64 positions at a time, one to a lane; the ends of the words'
// runs are then a mask in scalar registers, and a row's number a lane read.  U
// rows are on their way together.  crossing[0] counts the chunks in which a word that
// goes past the chunk's end begins, listed after it.
template <typename TG, typename TO, int W, bool DROP, bool STREAM>
__global__ __launch_bounds__(256) void reduce_kernel(
    const typename TG::store *__restrict__ grad, int64_t ldg, typename TO::store *__restrict__ out,
    int64_t ldo, int32_t D, float factor, Dropout drop, bool accumulate, uint32_t col_tiles,
    GradPlan g, const Token *__restrict__ token, float *__restrict__ part,
    uint32_t *__restrict__ crossing) {
  // rows of a lane in flight: 32 registers of them
  constexpr int U = sizeof(Packed<TG, W>) <= 8 ? 16 : 128 / (int)sizeof(Packed<TG, W>);
  static_assert(64 % U == 0, "a batch lies within 64 positions");
  const int lane = threadIdx.x & 63;
  const uint32_t item = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
  const uint32_t c = item / col_tiles;
  if (c >= g.chunks) return;
  const uint32_t tile = item - c * col_tiles;
  const Columns<W> columns(tile, D);
  const uint32_t own = columns.own;
  const int32_t n = columns.n, col = columns.col;
  const bool straddles = DROP && D % W != 0 && tile == col_tiles - 1;
  grad += columns.first;
  const uint32_t offset = columns.offset * (uint32_t)sizeof(typename TG::store);
  const uint32_t begin = c * g.chunk;
  const uint32_t end = g.N - begin < g.chunk ? g.N : begin + g.chunk;
  bool began_here = begin == 0 || token[begin - 1].word != token[begin].word;
  float sum[W] = {};
  for (uint32_t p = begin; p < end; p += 64) {
    const uint32_t at = p + lane < end ? p + lane : end - 1;
    const Token own_token = token[at];
    const uint32_t word = own_token.word, row = own_token.number;
    const uint32_t next = at + 1 < g.N ? token[at + 1].word : g.V;  // the word after
    const bool live = p + lane < end && word < g.V;
    // (tokens without a word are the last)
    const int count = __popcll(__ballot(live));
    const uint64_t ends = __ballot(live && (next != word || at + 1 == end));

    if (count == 0) return;
    for (int t = 0; t < count; t += U) {
      Packed<TG, W> v[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        v[u] = load_row<TG, W, STREAM>(grad, ldg, (uint32_t)__builtin_amdgcn_readlane(row, t + u),
                                       offset);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (t + u >= count) break;
        add_row<TG, W, DROP>(v[u], (uint32_t)__builtin_amdgcn_readlane(row, t + u), col, straddles,
                             drop, sum);
        if (!(ends >> (t + u) & 1)) continue;
        const uint32_t w = __builtin_amdgcn_readlane(word, t + u);
        const bool goes_on = __builtin_amdgcn_readlane(next, t + u) == w;
        if (began_here && !goes_on) {
          write_row<TO, W>(out, ldo, w, own, n, factor, accumulate, sum);
        } else {
          float *slot = part + (int64_t)(2 * c + (began_here ? 1 : 0)) * g.ld_part + col;
          if (n) store_elements<F32, W>(slot, W, sum);
          if (began_here && tile == 0 && lane == 0) crossing[1 + atomicAdd(crossing, 1u)] = c;
        }
        began_here = true;
#pragma unroll
        for (int j = 0; j < W; ++j) sum[j] = 0.0f;
      }
    }
  }
}

constexpr int kJoinWaves = 8;

// The words that cross chunks: each one's parts added in order, a run of them
// by each wavefront of the workgroup.
template <typename TO, int W>
__global__ __launch_bounds__(kJoinWaves * 64) void join_kernel(
    typename TO::store *__restrict__ out, int64_t ldo, int32_t D, float factor, bool accumulate,
    uint32_t col_tiles, GradPlan g, const Token *__restrict__ token,
    const float *__restrict__ part, const uint32_t *__restrict__ crossing) {
  constexpr int U = 8;
  __shared__ float sums[kJoinWaves - 1][64 * W];
  const int lane = threadIdx.x & 63;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t items = crossing[0] * col_tiles;
  for (uint32_t item = blockIdx.x; item < items; item += gridDim.x) {
    const uint32_t i = item / col_tiles;
    const Columns<W> columns(item - i * col_tiles, D);
    const uint32_t own = columns.own;
    const int32_t n = columns.n, col = columns.col;
    const uint32_t c0 = crossing[1 + i];
    const uint32_t word = token[(c0 + 1) * g.chunk - 1].word;
    // the chunk in which the word ends: the last whose first token is one of it,
    // sought 64 at a time
    uint32_t lo = c0 + 1, hi = g.chunks;
    while (hi - lo > 1) {
      const uint32_t step = (hi - lo + 62) / 64, probe = lo + (lane + 1) * step;
      const uint64_t yes = __ballot(probe < hi && token[probe * g.chunk].word == word);
      lo += __popcll(yes) * step;
      hi = hi - lo > step ? lo + step : hi;
    }
    const uint32_t parts = lo - c0 + 1;
    const uint32_t each = (parts + kJoinWaves - 1) / kJoinWaves;
    const uint32_t from = wave * each < parts ? wave * each : parts;
    const uint32_t to = from + each < parts ? from + each : parts;
    float sum[W] = {};
    for (uint32_t k = from; k < to; k += U) {
      float v[U][W];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const uint32_t slot = 2 * (c0 + k + u) + (k + u == 0 ? 1 : 0);
        load_elements<F32, W>(part + (int64_t)slot * g.ld_part + col, k + u < to ? W : 0, v[u]);
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int j = 0; j < W; ++j) sum[j] += v[u][j];
    }
    if (wave > 0) {
#pragma unroll
      for (int j = 0; j < W; ++j) sums[wave - 1][j * 64 + lane] = sum[j];
    }
    __syncthreads();
    if (wave == 0) {
#pragma unroll
      for (int j = 0; j < W; ++j)
        for (int q = 0; q < kJoinWaves - 1; ++q) sum[j] += sums[q][j * 64 + lane];
      write_row<TO, W>(out, ldo, word, own, n, factor, accumulate, sum);
    }
    __syncthreads();
  }
}

// A few tokens, without a sort: each wavefront has one token and a tile of
// columns, finds the tokens of the same word by comparing all of them (two to a
// lane), and, if its own is the first of them, adds them up.  The workgroups
// before those clear the rows without tokens, `rows` to a wavefront.
constexpr int kFewTokens = 128;

template <typename TG, typename TO, int W, bool DROP>
__global__ __launch_bounds__(256) void few_kernel(
    const typename TG::store *__restrict__ grad, int64_t ldg, const int32_t *__restrict__ word_id,
    int32_t N, typename TO::store *__restrict__ out, int64_t ldo, int32_t V, int32_t D, float factor,
    Dropout drop, bool accumulate, uint32_t col_tiles, uint32_t clear_blocks, int32_t rows) {
  constexpr int U = 8;
  const int lane = threadIdx.x & 63;
  const int32_t low = lane < N ? word_id[lane] : -1;
  const int32_t high = lane + 64 < N ? word_id[lane + 64] : -1;
  if (blockIdx.x < clear_blocks) {
    const int64_t width = (int64_t)D * (int64_t)sizeof(typename TO::store);
    const uint32_t unit = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
    for (int64_t first = (int64_t)unit * rows; first < V; first += (int64_t)clear_blocks * 4 * rows) {
      for (int64_t row = first; row < first + rows && row < V; ++row) {
        if (__ballot(low == row) | __ballot(high == row)) continue;
        char *p = reinterpret_cast<char *>(out + row * ldo);
        for (int64_t at = lane * 16; at < width; at += 1024) clear_bytes<false>(p + at, width - at);
      }
    }
    return;
  }
  const uint32_t items = (uint32_t)N * col_tiles;
  uint32_t item = __builtin_amdgcn_readfirstlane((blockIdx.x - clear_blocks) * 4 + (threadIdx.x >> 6));
  for (; item < items; item += (gridDim.x - clear_blocks) * 4) {
    const uint32_t t = item / col_tiles, tile = item - t * col_tiles;
    const int32_t word = t < 64 ? __builtin_amdgcn_readlane(low, t)
                                : __builtin_amdgcn_readlane(high, t - 64);
    if ((uint32_t)word >= (uint32_t)V) continue;
    uint64_t a = __ballot(low == word), b = __ballot(high == word);
    if ((a ? (uint32_t)__builtin_ctzll(a) : 64 + (uint32_t)__builtin_ctzll(b)) != t) continue;
    const Columns<W> columns(tile, D);
    const bool straddles = DROP && D % W != 0 && tile == col_tiles - 1;
    const uint32_t offset = columns.offset * (uint32_t)sizeof(typename TG::store);
    float sum[W] = {};
    while (a | b) {
      Packed<TG, W> v[U];
      uint32_t row[U];
      int n = 0;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (a | b) {
          row[u] = a ? (uint32_t)__builtin_ctzll(a) : 64 + (uint32_t)__builtin_ctzll(b);
          if (a)
            a &= a - 1;
          else
            b &= b - 1;
          n = u + 1;
        } else {
          row[u] = t;
        }
        v[u] = load_row<TG, W, false>(grad + columns.first, ldg, row[u], offset);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (u < n) add_row<TG, W, DROP>(v[u], row[u], columns.col, straddles, drop, sum);
      }
    }
    write_row<TO, W>(out, ldo, (uint32_t)word, columns.own, columns.n, factor, accumulate, sum);
  }
}

}  // namespace lda
