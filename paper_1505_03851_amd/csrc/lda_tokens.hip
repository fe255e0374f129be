// Host side and C ABI of the operators around a language model's tokens
// (gfx950): argument checks, launch shapes and launches.
//
// lda_embed            rows of a table by word, scaled and dropped out.
// lda_dropout          dropout of any rows, and of their gradient.
// lda_embed_grad       the table's gradient by sorted tokens.
// lda_penalise_logits  penalties for repeated tokens, biases, masks.
// lda_draw_logits      one token per row of logits under those rules.
//
// Device code: elements.hpp (element types), wave_ops.hpp, keep_bits.hpp (the dropout
// mask), token_rows.hpp, token_grad.hpp with grad_columns.hpp, logits.hpp.
#include <hip/hip_runtime.h>

#include <math.h>
#include <stdint.h>

#include "lda_draw.h"
#include "status.hpp"
#include "token_rows.hpp"
#include "token_grad.hpp"
#include "logits.hpp"

namespace lda {
namespace {

// A launch holds fewer than 2^32 work-items; kernels stride over the rest.
constexpr int64_t kMaxBlocks = 1 << 20;
constexpr int64_t kMaxWaves = 1 << 26;  // of a launch whose kernel does not stride
// 16-byte units of a table (64 MB) from which clearing it bounds a call.
constexpr int64_t kClearApart = (64 << 20) / 16;

unsigned grid_of(int64_t tiles) {
  return (unsigned)(tiles < 1 ? 1 : tiles < kMaxBlocks ? tiles : kMaxBlocks);
}

bool aligned(const void *p, int bytes) {
  return !(reinterpret_cast<uintptr_t>(p) & (uintptr_t)(bytes - 1));
}

int dtype_size(int32_t dtype) {
  switch (dtype) {
    case LDA_F32: return 4;
    case LDA_BF16:
    case LDA_F16: return 2;
    default: return 0;
  }
}

bool probability(double p) { return p >= 0.0 && p < 1.0; }

// The mask's threshold of 2^16, and the factor of what is kept.
Dropout make_dropout(double p, uint64_t seed, uint32_t step, double scale, float *factor) {
  const double q = fmin(65535.0, rint(65536.0 * p));
  *factor = (float)(scale * (65536.0 / (65536.0 - q)));
  return Dropout{(uint32_t)q, step, (uint32_t)seed, (uint32_t)(seed >> 32)};
}

template <typename T, bool GATHER>
int launch_rows(const void *x, int64_t ldx, const int32_t *word_id, void *out, int64_t ldo,
                int64_t N, int32_t V, int64_t D, double scale, double p, uint64_t seed,
                uint32_t step, hipStream_t s) {
  float factor;
  const Dropout drop = make_dropout(p, seed, step, scale, &factor);
  // the lanes of a row: the power of two that covers its 8-column units, up to
  // the workgroup
  const int64_t units = (D + 7) / 8;
  int lanes_log2 = 0;
  while ((1 << lanes_log2) < kRowThreads && (1 << lanes_log2) < units) ++lanes_log2;
  const int64_t col_tiles = (units + (1 << lanes_log2) - 1) >> lanes_log2;
  const int64_t rows = (int64_t)(kRowThreads >> lanes_log2) * kRowsEach;
  const int64_t tiles = (N + rows - 1) / rows * col_tiles;
  using S = typename T::store;
#define LDA_ROWS(DROP, WIDE)                                                                     \
  rows_kernel<T, GATHER, DROP, WIDE><<<grid_of(tiles), kRowThreads, 0, s>>>(                     \
      (const S *)x, ldx, word_id, (S *)out, ldo, N, V, D, factor, drop, lanes_log2,              \
      (uint32_t)col_tiles, tiles)
  const bool wide = lanes_log2 >= 6;
  if (drop.q && wide)
    LDA_ROWS(true, true);
  else if (drop.q)
    LDA_ROWS(true, false);
  else if (wide)
    LDA_ROWS(false, true);
  else
    LDA_ROWS(false, false);
#undef LDA_ROWS
  return launch_status();
}

// What lda_embed_grad keeps in the caller's workspace, and how the work is cut.
struct GradLayout {
  int passes, bits;        // of the sort
  int64_t sort_chunks;
  int width;               // columns of a lane
  uint32_t col_tiles;      // tiles of 64 width columns
  uint32_t chunk, chunks;  // sorted positions of a wavefront
  int64_t ld_part;
  size_t tokens[2], hist, total, crossing, part, bytes;
};

GradLayout grad_layout(int64_t N, int32_t V, int32_t D) {
  GradLayout L;
  int need = 1;  // bits of V, the key of tokens without a word
  while (need < 31 && V >> need) ++need;
  L.passes = (need + kSortMaxBits - 1) / kSortMaxBits;
  L.bits = (need + L.passes - 1) / L.passes;
  L.sort_chunks = (N + kSortChunk - 1) / kSortChunk;
  L.width = D > 256 ? 8 : D > 128 ? 4 : D > 64 ? 2 : 1;
  switch (L.width) {
    case 8: L.col_tiles = column_tiles<8>(D); break;
    case 4: L.col_tiles = column_tiles<4>(D); break;
    case 2: L.col_tiles = column_tiles<2>(D); break;
    default: L.col_tiles = column_tiles<1>(D);
  }
  // A wavefront's time grows with its run, and that of joining a frequent word's
  // parts with the number of runs, so the run grows with the root of N: 32 chunk^2
  // holds it.  Measured against half and twice the run: 1,000 tokens 13.6 us
  // (twice 15.4), 8,000 of 512 columns 32.6 (34.4, 36.5), 32,000 41.9 (47.8),
  // 32,768 of 2,048 136 (140, 142), 131,072 of 512 74.8 (83.8, 77.4), 1M of 256
  // 168 (176, 179).
  L.chunk = 8;
  while (L.chunk < 512 && (int64_t)32 * L.chunk * L.chunk < N) L.chunk *= 2;
  // (rows of many millions of columns: longer runs, up to what a launch holds)
  while ((N + L.chunk - 1) / L.chunk * L.col_tiles >= kMaxWaves) L.chunk *= 2;
  L.chunks = (uint32_t)((N + L.chunk - 1) / L.chunk);
  L.ld_part = ((int64_t)D + 7) & ~(int64_t)7;
  size_t at = 0;
  auto take = [&](size_t b) {
    const size_t o = at;
    at += (b + 255) & ~(size_t)255;
    return o;
  };
  for (int i = 0; i < 2; ++i) L.tokens[i] = take(sizeof(Token) * (size_t)N);
  L.hist = take(4 * (size_t)L.sort_chunks << L.bits);
  L.total = take(4 * (size_t)kSortMaxBins);
  L.crossing = take(4 * ((size_t)L.chunks + 1));
  L.part = take(4 * (size_t)(2 * (uint64_t)L.chunks) * (size_t)L.ld_part);
  L.bytes = at;
  return L;
}

template <typename TG, typename TO, int W>
void launch_reduce(const void *grad, int64_t ldg, void *out, int64_t ldo, int32_t D, float factor,
                   const Dropout &drop, bool accumulate, const GradLayout &L, const GradPlan &g,
                   const Token *token, char *w, hipStream_t s) {
  using SG = typename TG::store;
  using SO = typename TO::store;
  float *part = (float *)(w + L.part);
  uint32_t *crossing = (uint32_t *)(w + L.crossing);
  const unsigned grid = (unsigned)(((uint64_t)L.chunks * L.col_tiles + 3) / 4);
  // A gradient that the 256 MB behind the L2s cannot hold anyway passes them by:
  // 1M tokens of 256 bfloat16 170 us against 185, 32,768 of 2,048 136 against 139;
  // a smaller one may still be there from the launch that made it (131,072 of 256:
  // 72.4 against 70.7).  In float a lane's 32 bytes are two accesses to one line
  // (16,384 of 2,048: 131 against 129).
  constexpr bool kMayStream = sizeof(SG) == 2;
  // (one row for all tokens stays in the caches: 32,768 of 2,048 bfloat16 70 us
  // against 82 past them, 1M of 256 132 against 187)
  const int64_t read = (ldg ? (int64_t)g.N : 1) * D * (int64_t)sizeof(SG);
  const bool stream = kMayStream && read >= (int64_t)128 << 20;
#define LDA_SUM(DROP, STREAM)                                                                    \
  reduce_kernel<TG, TO, W, DROP, STREAM><<<grid, 256, 0, s>>>(                                   \
      (const SG *)grad, ldg, (SO *)out, ldo, D, factor, drop, accumulate, L.col_tiles, g, token, \
      part, crossing)
  if (drop.q && stream)
    LDA_SUM(true, kMayStream);
  else if (drop.q)
    LDA_SUM(true, false);
  else if (stream)
    LDA_SUM(false, kMayStream);
  else
    LDA_SUM(false, false);
#undef LDA_SUM
  if (L.chunks > 1)
    join_kernel<TO, W><<<512, kJoinWaves * 64, 0, s>>>((SO *)out, ldo, D, factor, accumulate,
                                                       L.col_tiles, g, token, part, crossing);
}

// N of 1 to kFewTokens: one launch, no workspace (64 tokens of 512 columns: 6 us
// against 11 with the sort).
template <typename TG, typename TO, int W>
void launch_few(const void *grad, int64_t ldg, const int32_t *word_id, void *out, int64_t ldo,
                int64_t N, int32_t V, int32_t D, float factor, const Dropout &drop,
                bool accumulate, bool clear, uint32_t col_tiles, hipStream_t s) {
  using SG = typename TG::store;
  using SO = typename TO::store;
  // about 4 KB of rows to a wavefront, so that the workgroups, which start in their
  // order, write one stretch after another
  const int64_t width = (int64_t)sizeof(SO) * D;
  const int32_t rows = width >= 4096 ? 1 : width < 256 ? 16 : (int32_t)(4096 / width);
  const unsigned clear_blocks = clear ? grid_of(((int64_t)V + 4 * rows - 1) / (4 * rows)) : 0u;
  const unsigned grid = clear_blocks + grid_of((N * col_tiles + 3) / 4);
  if (drop.q)
    few_kernel<TG, TO, W, true><<<grid, 256, 0, s>>>((const SG *)grad, ldg, word_id, (int32_t)N,
                                                     (SO *)out, ldo, V, D, factor, drop, accumulate,
                                                     col_tiles, clear_blocks, rows);
  else
    few_kernel<TG, TO, W, false><<<grid, 256, 0, s>>>((const SG *)grad, ldg, word_id, (int32_t)N,
                                                      (SO *)out, ldo, V, D, factor, drop,
                                                      accumulate, col_tiles, clear_blocks, rows);
}

template <typename TG, typename TO>
int launch_grad(const void *grad, int64_t ldg, const int32_t *word_id, void *out, int64_t ldo,
                int64_t N, int32_t V, int32_t D, double scale, double p, uint64_t seed,
                uint32_t step, bool accumulate, void *workspace, hipStream_t s) {
  const int64_t size = (int64_t)sizeof(typename TO::store);
  const GradLayout L = grad_layout(N, V, D);
  float factor;
  const Dropout drop = make_dropout(p, seed, step, scale, &factor);
  const unsigned chunks = (unsigned)L.sort_chunks;
  // each launch of the sort sets its share of the rows to zero
  const bool dense = ldo == D;
  ClearShare clear{(char *)out, size * ldo, size * D * (dense ? (int64_t)V : 1),
                   dense ? 1 : (int64_t)V, 0, N == 0 || chunks == 1 ? 1u : 2u * L.passes,
                   N <= kFewTokens ? 0u : chunks};
  // (a share of a table of a few bytes is at least one unit, so that every launch has
  // a workgroup that clears: which of them the unit falls to, clear_share decides)
  const int64_t units = ((clear.width + 15) / 16 * clear.rows + clear.parts - 1) / clear.parts;
  const int64_t clear_blocks = accumulate ? 0 : (units + kSortThreads - 1) / kSortThreads;
  // A share of more than 64 MB in workgroups of 16 KB each, which start in their
  // order and so write one stretch after another (512 MB 113 us against 129, 410 in
  // four shares 127 against 134); a smaller one in 1,024 that stride through it
  // (205 MB in four shares 84 against 87, 64 MB 20.9 against 23.5).
  const int64_t most = units > kClearApart ? kMaxBlocks : 1024;
  const unsigned extra = (unsigned)(clear_blocks < most ? clear_blocks : most);
  if (N > 0 && N <= kFewTokens) {
    // a large table is cleared by a launch of its own, as one stretch
    const bool apart = !accumulate && units > kClearApart;
    if (apart) clear_kernel<<<extra, kSortThreads, 0, s>>>(clear);
#define LDA_FEW(W)                                                                               \
  launch_few<TG, TO, W>(grad, ldg, word_id, out, ldo, N, V, D, factor, drop, accumulate,         \
                        !accumulate && !apart, L.col_tiles, s)
    switch (L.width) {
      case 8: LDA_FEW(8); break;
      case 4: LDA_FEW(4); break;
      case 2: LDA_FEW(2); break;
      default: LDA_FEW(1);
    }
#undef LDA_FEW
    return launch_status();
  }
  if (N == 0) {
    if (extra) clear_kernel<<<extra, kSortThreads, 0, s>>>(clear);
    return launch_status();
  }
  char *w = (char *)workspace;
  uint32_t *hist = (uint32_t *)(w + L.hist), *total = (uint32_t *)(w + L.total);
  uint32_t *crossing = (uint32_t *)(w + L.crossing);
  const Token *token = nullptr;
  if (chunks == 1) {
    Token *out_tokens = (Token *)(w + L.tokens[0]);
    sort_chunk_kernel<<<1 + extra, kSortThreads, 0, s>>>(word_id, (int32_t)N, V, L.passes, L.bits,
                                                         out_tokens, crossing, clear);
    token = out_tokens;
  }
  for (int pass = 0; chunks > 1 && pass < L.passes; ++pass) {
    Token *out_tokens = (Token *)(w + L.tokens[pass & 1]);
    const int shift = pass * L.bits;
    clear.part = 2 * pass;
    sort_hist_kernel<<<chunks + extra, kSortThreads, 0, s>>>(
        word_id, token, N, V, shift, L.bits, hist, pass == 0 ? crossing : nullptr, clear);
    // from 17 chunks on a launch of its own sums the chunks before each
    const bool scan = chunks > 16;
    if (scan)
      sort_scan_kernel<<<((1u << L.bits) + 63) / 64, kSortThreads, 0, s>>>(hist, total, chunks,
                                                                           1 << L.bits);
    clear.part = 2 * pass + 1;
    sort_scatter_kernel<<<chunks + extra, kSortThreads, 0, s>>>(word_id, token, N, V, shift, L.bits,
                                                                hist, scan ? total : nullptr,
                                                                out_tokens, clear);
    token = out_tokens;
  }
  const GradPlan g{(uint32_t)N, (uint32_t)V, L.chunk, L.chunks, L.ld_part};
#define LDA_REDUCE(W)                                                                           \
  launch_reduce<TG, TO, W>(grad, ldg, out, ldo, D, factor, drop, accumulate, L, g, token, w, s)
  switch (L.width) {
    case 8: LDA_REDUCE(8); break;
    case 4: LDA_REDUCE(4); break;
    case 2: LDA_REDUCE(2); break;
    default: LDA_REDUCE(1);
  }
#undef LDA_REDUCE
  return launch_status();
}

// The groups (and wavefronts) of a workgroup: the most that still give every
// compute unit two workgroups, since each workgroup reads its row's history.
// (256 rows of 100,000 logits and 4,096 tokens: 28.9 us with eight, 30.4 with four,
// 39 with one.)
int group_waves(int64_t B, int64_t V) {
  const int64_t groups = (V + kGroup - 1) / kGroup;
  int waves = kGroupWaves;
  while (waves > 1 && B * ((groups + waves - 1) / waves) < 512) waves /= 2;
  return waves;
}

int make_rules(const lda_logit_rules *r, int64_t B, int32_t V, Rules *out) {
  *out = Rules{};
  if (!r) return LDA_OK;
  const void *ptrs[] = {r->history, r->lengths, r->prompt, r->repetition, r->frequency,
                        r->presence, r->bias, r->mask};
  for (const void *p : ptrs)
    if (!aligned(p, 4)) return LDA_ERR_ALIGN;
  if (r->history) {
    if (!r->lengths) return LDA_ERR_NULL;
    if (r->capacity < 0) return LDA_ERR_SHAPE;
    if (r->capacity > LDA_HISTORY_MAX) return LDA_ERR_UNSUPPORTED;
    if (r->ld_history != 0 && r->ld_history < r->capacity) return LDA_ERR_VALUE;
  }
  if (r->bias && r->ld_bias != 0 && r->ld_bias < V) return LDA_ERR_VALUE;
  if (r->mask && r->ld_mask != 0 && r->ld_mask < ((int64_t)V + 31) / 32) return LDA_ERR_VALUE;
  *out = Rules{r->history,    r->ld_history, r->lengths, r->prompt,
               r->repetition, r->frequency,  r->presence, r->bias,
               r->ld_bias,    (const uint32_t *)r->mask,  r->ld_mask, (int32_t)r->capacity};
  return LDA_OK;
}

template <typename T>
int launch_penalise(const void *logits, int64_t ld, void *out, int64_t ldo, int64_t B, int32_t V,
                    const Rules &r, hipStream_t s) {
  using S = typename T::store;
  const int waves = group_waves(B, V);
  const int64_t slices = ((int64_t)V + waves * kGroup - 1) / (waves * kGroup), tiles = B * slices;
  const size_t lds = r.history ? 4 * (size_t)waves * kGroup : 0;
  penalise_kernel<T><<<grid_of(tiles), 64 * waves, lds, s>>>((const S *)logits, ld, (S *)out, ldo,
                                                             V, r, (uint32_t)slices, tiles);
  return launch_status();
}

template <typename T>
int launch_draw(const void *logits, int64_t ld, int64_t B, int32_t V, const Rules &r,
                const float *temperature, const float *min_p, const int64_t *seed,
                const int32_t *position, int32_t *z, float *prob, GroupSum *groups,
                hipStream_t s) {
  using S = typename T::store;
  const uint32_t per_row = (uint32_t)(((int64_t)V + kGroup - 1) / kGroup);
  // Rows of up to 32 groups: one launch, no workspace.  With every rule on, 16,000
  // logits 11 us against 19 for one row, 13.6 against 27 for 256; 32,000, 15
  // against 18 and 20 against 36; with none, 16,000 7.6 against 8.6 and 9.2 against
  // 12.3; 32,000 10.1 against 8.9 (and a launch less on the host) and 12 against 15.
  if (per_row <= kShortGroups) {
#define LDA_DRAW_SHORT(R)                                                                        \
  short_draw_kernel<T, R><<<grid_of(B), kDrawThreads,                                            \
                            r.history ? 4 * R * kDrawWaves * kGroup : 0, s>>>(                   \
      (const S *)logits, ld, B, V, r, temperature, min_p, seed, position, z, prob)
    if (per_row <= kDrawWaves)
      LDA_DRAW_SHORT(1);
    else
      LDA_DRAW_SHORT(2);
#undef LDA_DRAW_SHORT
    return launch_status();
  }
  const int waves = group_waves(B, V);
  const int64_t slices = ((int64_t)V + waves * kGroup - 1) / (waves * kGroup), tiles = B * slices;
  const size_t lds = r.history ? 4 * (size_t)waves * kGroup : 0;
  group_kernel<T, false><<<grid_of(tiles), 64 * waves, lds, s>>>(
      (const S *)logits, ld, V, r, temperature, min_p, groups, per_row, (uint32_t)slices, tiles);
  if (min_p)
    group_kernel<T, true><<<grid_of(tiles), 64 * waves, lds, s>>>(
        (const S *)logits, ld, V, r, temperature, min_p, groups, per_row, (uint32_t)slices, tiles);
  draw_kernel<T><<<grid_of(B), kDrawThreads, 0, s>>>((const S *)logits, ld, B, V, r, temperature,
                                                     min_p, seed, position, groups, per_row, z,
                                                     prob);
  return launch_status();
}

}  // namespace
}  // namespace lda

using namespace lda;

extern "C" int lda_embed(const void *table, int64_t ld_table, const int32_t *word_id, void *out,
                         int64_t ld_out, int64_t N, int32_t V, int32_t D, int32_t dtype,
                         double scale, double p, uint64_t seed, uint32_t step, void *stream) {
  if (N < 0 || V <= 0 || D <= 0) return LDA_ERR_SHAPE;
  if (N > LDA_MAX_N) return LDA_ERR_UNSUPPORTED;
  const int size = dtype_size(dtype);
  if (!size || !probability(p) || ld_table < 0 || ld_out < D) return LDA_ERR_VALUE;
  if (N == 0) return LDA_OK;
  if (!table || !word_id || !out) return LDA_ERR_NULL;
  if (!aligned(table, size) || !aligned(out, size) || !aligned(word_id, 4)) return LDA_ERR_ALIGN;
  hipStream_t s = static_cast<hipStream_t>(stream);
  switch (dtype) {
    case LDA_F32:
      return launch_rows<F32, true>(table, ld_table, word_id, out, ld_out, N, V, D, scale, p, seed,
                                    step, s);
    case LDA_BF16:
      return launch_rows<Bf16, true>(table, ld_table, word_id, out, ld_out, N, V, D, scale, p, seed,
                                     step, s);
    default:
      return launch_rows<F16, true>(table, ld_table, word_id, out, ld_out, N, V, D, scale, p, seed,
                                    step, s);
  }
}

extern "C" int lda_dropout(const void *x, int64_t ld_x, void *out, int64_t ld_out, int64_t rows,
                           int64_t cols, int32_t dtype, double p, uint64_t seed, uint32_t step,
                           void *stream) {
  if (rows < 0 || cols <= 0) return LDA_ERR_SHAPE;
  if (rows > LDA_MAX_N || cols > LDA_DROPOUT_MAX_COLS) return LDA_ERR_UNSUPPORTED;
  const int size = dtype_size(dtype);
  if (!size || !probability(p) || ld_x < 0 || ld_out < cols) return LDA_ERR_VALUE;
  if (rows == 0) return LDA_OK;
  if (!x || !out) return LDA_ERR_NULL;
  if (!aligned(x, size) || !aligned(out, size)) return LDA_ERR_ALIGN;
  hipStream_t s = static_cast<hipStream_t>(stream);
  switch (dtype) {
    case LDA_F32:
      return launch_rows<F32, false>(x, ld_x, nullptr, out, ld_out, rows, 1, cols, 1.0, p, seed,
                                     step, s);
    case LDA_BF16:
      return launch_rows<Bf16, false>(x, ld_x, nullptr, out, ld_out, rows, 1, cols, 1.0, p, seed,
                                      step, s);
    default:
      return launch_rows<F16, false>(x, ld_x, nullptr, out, ld_out, rows, 1, cols, 1.0, p, seed,
                                     step, s);
  }
}

extern "C" size_t lda_embed_grad_workspace_bytes(int64_t N, int32_t V, int32_t D) {
  if (N <= kFewTokens || V <= 0 || D <= 0 || N > LDA_COUNT_MAX_N) return 0;
  return grad_layout(N, V, D).bytes;
}

extern "C" int lda_embed_grad(const void *grad, int64_t ld_grad, const int32_t *word_id, void *out,
                              int64_t ld_out, int64_t N, int32_t V, int32_t D, int32_t grad_dtype,
                              int32_t out_dtype, double scale, double p, uint64_t seed,
                              uint32_t step, int32_t accumulate, void *workspace,
                              size_t workspace_bytes, void *stream) {
  if (N < 0 || V <= 0 || D <= 0) return LDA_ERR_SHAPE;
  if (N > LDA_COUNT_MAX_N) return LDA_ERR_UNSUPPORTED;
  const int size = dtype_size(grad_dtype), out_size = dtype_size(out_dtype);
  if (!size || !out_size || !probability(p) || ld_grad < 0 || ld_out < D) return LDA_ERR_VALUE;
  if (out_dtype != LDA_F32 && out_dtype != grad_dtype) return LDA_ERR_UNSUPPORTED;
  if (!out) return LDA_ERR_NULL;
  const size_t need = lda_embed_grad_workspace_bytes(N, V, D);
  if ((N > 0 && (!grad || !word_id)) || (need > 0 && !workspace)) return LDA_ERR_NULL;
  if (!aligned(out, out_size) || !aligned(grad, size) || !aligned(word_id, 4) ||
      !aligned(workspace, 8))
    return LDA_ERR_ALIGN;
  if (workspace_bytes < need) return LDA_ERR_WORKSPACE;
  hipStream_t s = static_cast<hipStream_t>(stream);
#define LDA_GRAD(TG, TO)                                                                       \
  launch_grad<TG, TO>(grad, ld_grad, word_id, out, ld_out, N, V, D, scale, p, seed, step,      \
                      accumulate != 0, workspace, s)
  if (grad_dtype == LDA_F32) return LDA_GRAD(F32, F32);
  if (grad_dtype == LDA_BF16)
    return out_dtype == LDA_F32 ? LDA_GRAD(Bf16, F32) : LDA_GRAD(Bf16, Bf16);
  return out_dtype == LDA_F32 ? LDA_GRAD(F16, F32) : LDA_GRAD(F16, F16);
#undef LDA_GRAD
}

extern "C" int lda_penalise_logits(const void *logits, int64_t ld_logits, void *out,
                                   int64_t ld_out, int64_t B, int32_t V, int32_t dtype,
                                   const lda_logit_rules *rules, void *stream) {
  if (B < 0 || V <= 0) return LDA_ERR_SHAPE;
  if (B > LDA_LOGITS_MAX_ROWS) return LDA_ERR_UNSUPPORTED;
  const int size = dtype_size(dtype);
  if (!size || ld_logits < 0 || ld_out < V) return LDA_ERR_VALUE;
  Rules r;
  if (const int bad = make_rules(rules, B, V, &r)) return bad;
  if (B == 0) return LDA_OK;
  if (!logits || !out) return LDA_ERR_NULL;
  if (!aligned(logits, size) || !aligned(out, size)) return LDA_ERR_ALIGN;
  hipStream_t s = static_cast<hipStream_t>(stream);
  switch (dtype) {
    case LDA_F32: return launch_penalise<F32>(logits, ld_logits, out, ld_out, B, V, r, s);
    case LDA_BF16: return launch_penalise<Bf16>(logits, ld_logits, out, ld_out, B, V, r, s);
    default: return launch_penalise<F16>(logits, ld_logits, out, ld_out, B, V, r, s);
  }
}

extern "C" size_t lda_draw_logits_workspace_bytes(int64_t B, int32_t V) {
  if (B <= 0 || V <= 0 || B > LDA_LOGITS_MAX_ROWS) return 0;
  const size_t groups = (size_t)(((int64_t)V + kGroup - 1) / kGroup);
  return groups <= kShortGroups ? 0 : sizeof(GroupSum) * (size_t)B * groups;
}

extern "C" int lda_draw_logits(const void *logits, int64_t ld_logits, int64_t B, int32_t V,
                               int32_t dtype, const lda_logit_rules *rules,
                               const float *temperature, const float *min_p, const int64_t *seed,
                               const int32_t *position, int32_t *z, float *prob, void *workspace,
                               size_t workspace_bytes, void *stream) {
  if (B < 0 || V <= 0) return LDA_ERR_SHAPE;
  if (B > LDA_LOGITS_MAX_ROWS) return LDA_ERR_UNSUPPORTED;
  const int size = dtype_size(dtype);
  if (!size || ld_logits < 0) return LDA_ERR_VALUE;
  Rules r;
  if (const int bad = make_rules(rules, B, V, &r)) return bad;
  if (B == 0) return LDA_OK;
  const size_t need = lda_draw_logits_workspace_bytes(B, V);
  if (!logits || !seed || !position || !z || !prob || (need > 0 && !workspace)) return LDA_ERR_NULL;
  if (!aligned(logits, size) || !aligned(temperature, 4) || !aligned(min_p, 4) ||
      !aligned(seed, 8) || !aligned(position, 4) || !aligned(z, 4) || !aligned(prob, 4) ||
      !aligned(workspace, 8))
    return LDA_ERR_ALIGN;
  if (workspace_bytes < need) return LDA_ERR_WORKSPACE;
  GroupSum *g = static_cast<GroupSum *>(workspace);
  hipStream_t s = static_cast<hipStream_t>(stream);
  switch (dtype) {
    case LDA_F32:
      return launch_draw<F32>(logits, ld_logits, B, V, r, temperature, min_p, seed, position, z,
                              prob, g, s);
    case LDA_BF16:
      return launch_draw<Bf16>(logits, ld_logits, B, V, r, temperature, min_p, seed, position, z,
                               prob, g, s);
    default:
      return launch_draw<F16>(logits, ld_logits, B, V, r, temperature, min_p, seed, position, z,
                              prob, g, s);
  }
}
