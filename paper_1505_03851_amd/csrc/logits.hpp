// Logits of a language model: the rules that change them, and the draw of one
// token per row.
//
// The rules, in float and in this order, for token v of row b with c uses among
// the row's generated tokens:
//   x = seen ? (x > 0 ? x / repetition : x * repetition) : x   (seen: anywhere in
//                                        the history, the prompt included)
//   x = x - frequency * c
//   x = x - presence                     where c > 0
//   x = x + bias[v]
//   x = -inf                             where the mask's bit v is 0
//
// The draw: weights w_v = exp((x_v - max) / temperature), 0 below min_p.  With
// exponential variates E, argmin E_v / w_v is token v with probability
// w_v / sum w.  It is taken in two steps, the group of kGroup tokens by
// E_g / (sum of the group's weights), then the token inside it, so a row needs
// V / kGroup + kGroup variates and not V, and the second step reads one group.
// Which token wins depends on rounding only where the best two are within
// rounding of each other (about 1e-7 of the draws), in whatever order the sums
// are made; a search of partial sums for u * S would hang on the rounding of
// every one of V partial sums.
#pragma once

#include "elements.hpp"
#include "philox.hpp"

namespace lda {

constexpr int kGroup = 1024;  // tokens of a group, the unit of a wavefront
constexpr int kSteps = kGroup / 512;
constexpr int kGroupWaves = 8;   // groups of a workgroup, at most
constexpr int kDrawThreads = 1024;  // of a row's last step: one for each token of a group
constexpr int kDrawWaves = kDrawThreads / 64;
constexpr uint32_t kSeen = 0x80000000u;

struct Rules {
  const int32_t *history;  // [B][ld_history], or null
  int64_t ld_history;
  const int32_t *lengths, *prompt;  // [B]; prompt null: 0
  const float *repetition, *frequency, *presence;  // [B] or null
  const float *bias;                               // [B][ld_bias] or null; ld_bias 0: one row
  int64_t ld_bias;
  const uint32_t *mask;  // [B][ld_mask] or null; ld_mask 0: one row
  int64_t ld_mask;
  int64_t capacity;  // history's columns
};

struct RowRules {
  float repetition, frequency, presence;
  const float *bias;
  const uint32_t *mask;
};

__device__ __forceinline__ RowRules row_rules(const Rules &r, int64_t b) {
  return RowRules{r.repetition ? r.repetition[b] : 1.0f, r.frequency ? r.frequency[b] : 0.0f,
                  r.presence ? r.presence[b] : 0.0f, r.bias ? r.bias + b * r.ld_bias : nullptr,
                  r.mask ? r.mask + b * r.ld_mask : nullptr};
}

// A product that is rounded before it is used: two kernels must find the same
// value for one logit, so neither may fuse it into a sum.
__device__ __forceinline__ float rounded(float x) {
  asm volatile("" : "+v"(x));
  return x;
}

__device__ __forceinline__ float ruled(float x, uint32_t count, const RowRules &r) {
  if (count) {
    x = x > 0.0f ? x / r.repetition : rounded(x * r.repetition);
    const uint32_t c = count & ~kSeen;
    if (c) {
      x -= rounded(r.frequency * (float)c);
      x -= r.presence;
    }
  }
  return x;
}

// A row's history, four tokens to a lane and load.
struct History {
  const int32_t *tokens;
  int64_t size, prompt;  // 0 tokens where there is no history
};

__device__ __forceinline__ History row_history(const Rules &r, int64_t b) {
  if (!r.history) return History{nullptr, 0, 0};
  int64_t n = r.lengths[b];
  n = n < r.capacity ? n : r.capacity;
  return History{r.history + b * r.ld_history, n > 0 ? n : 0, r.prompt ? r.prompt[b] : 0};
}

__device__ __forceinline__ words4 history_load(const History &h, int64_t i) {
  words4 t;
  if (i + 4 <= h.size) {
    t = *reinterpret_cast<const words4_any *>(h.tokens + i);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) t[j] = i + j < h.size ? (uint32_t)h.tokens[i + j] : 0xFFFFFFFFu;
  }
  return t;
}

// Adds the tokens t (of which the first is number i) that lie in [first, first +
// size) to `count`: generated tokens in the low bits, kSeen for the prompt's.
__device__ __forceinline__ void history_count(const History &h, int64_t i, words4 t, int64_t first,
                                              uint32_t size, uint32_t *count) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    // (a negative token is above every vocabulary as an unsigned number)
    const int64_t at = (int64_t)t[j] - first;
    if ((uint64_t)at >= size) continue;
    if (i + j < h.prompt)
      atomicOr(&count[at], kSeen);
    else
      atomicAdd(&count[at], 1u);
  }
}

// The uses of the tokens [first, first + size) in a row's history, counted in
// LDS (which the caller has cleared and synchronised) by the whole workgroup.
__device__ __forceinline__ void count_history(const History &h, int64_t first, uint32_t size,
                                              uint32_t *count) {
  const int64_t step = 4 * (int64_t)blockDim.x;
  for (int64_t i = 4 * (int64_t)threadIdx.x; i < h.size; i += 2 * step) {
    const words4 a = history_load(h, i), b = history_load(h, i + step);
    history_count(h, i, a, first, size, count);
    history_count(h, i + step, b, first, size, count);
  }
}

// The logits of 8 neighbouring tokens from v on under the rules; n of them
// exist.  `count`: their uses, or null.
__device__ __forceinline__ void apply_rules(int64_t v, int n, const uint32_t *count,
                                            const RowRules &r, float (&x)[8]) {
  if (count) {
    uint32_t c[8], any = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      c[j] = count[j];
      any |= c[j];
    }
    if (any) {
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = ruled(x[j], c[j], r);
    }
  }
  if (r.bias) {
    float b[8];
    load_elements<F32, 8>(r.bias + v, n, b);
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] += b[j];
  }
  if (r.mask) {
    const uint32_t bits = n > 0 ? r.mask[v >> 5] >> (v & 31) : 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = bits >> j & 1 ? x[j] : -INFINITY;
  }
}

// A wavefront's group of a row: its logits on their way while the workgroup
// counts the row's history, then in float under the rules (x[s][j]: token
// first + 512 s + 8 lane + j).  The whole workgroup calls it, wavefronts past the
// end of the row too.
template <typename T>
__device__ __forceinline__ void group_logits(const typename T::store *row, int64_t first, int64_t V,
                                             const History &h, const RowRules &r, uint32_t *lds,
                                             float (&x)[kSteps][8], int (&n)[kSteps]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  Packed<T, 8> v[kSteps];
#pragma unroll
  for (int s = 0; s < kSteps; ++s) {
    const int64_t left = V - first - s * 512 - lane * 8;
    n[s] = left < 8 ? (left > 0 ? (int)left : 0) : 8;
    v[s] = load_packed<T, 8>(row + first + s * 512 + lane * 8, n[s]);
  }
  if (h.size) {
    words4 *mine = reinterpret_cast<words4 *>(lds + wave * kGroup);
#pragma unroll
    for (int i = 0; i < kGroup / 256; ++i) mine[i * 64 + lane] = words4{};
    __syncthreads();
    count_history(h, first - wave * kGroup, (blockDim.x >> 6) * kGroup, lds);
    __syncthreads();
  }
#pragma unroll
  for (int s = 0; s < kSteps; ++s) {
#pragma unroll
    for (int j = 0; j < 8; ++j) x[s][j] = T::up(v[s].v[j]);
    const int at = s * 512 + lane * 8;
    apply_rules(first + at, n[s], h.size ? lds + wave * kGroup + at : nullptr, r, x[s]);
  }
}

// A workgroup takes a group of one row for each of its wavefronts.
template <typename T>
__global__ __launch_bounds__(64 * kGroupWaves) void penalise_kernel(
    const typename T::store *logits, int64_t ld, typename T::store *out, int64_t ldo, int64_t V,
    Rules rules, uint32_t slices, int64_t tiles) {
  extern __shared__ uint32_t lds[];
  for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
    const int64_t b = tile / slices;
    const int64_t first = (tile - b * slices) * (blockDim.x >> 6) * kGroup +
                          (int64_t)(threadIdx.x >> 6) * kGroup;
    float x[kSteps][8];
    int n[kSteps];
    group_logits<T>(logits + b * ld, first, V, row_history(rules, b), row_rules(rules, b), lds, x, n);
#pragma unroll
    for (int s = 0; s < kSteps; ++s)
      store_elements<T, 8>(out + b * ldo + first + s * 512 + (threadIdx.x & 63) * 8, n[s], x[s]);
    __syncthreads();
  }
}

struct GroupSum {
  float top, sum;  // the largest logit of a group, and sum exp((x - top) / temperature)
};

struct DrawRow {
  float temperature;
  float inverse;  // 1 / temperature
  float floor;    // log(min_p); -inf: none
  bool greedy;    // the row takes its largest logit
};

__device__ __forceinline__ DrawRow draw_row(const float *temperature, const float *min_p,
                                            int64_t b) {
  const float given = temperature ? temperature[b] : 1.0f;
  // an infinite temperature would make -inf * 0 of the logits that may not be drawn
  const float t = fminf(given, 1e30f);
  const float p = min_p ? min_p[b] : 0.0f;
  return DrawRow{t, 1.0f / t, p > 0.0f ? logf(fminf(p, 1.0f)) : -INFINITY, !(given > 0.0f)};
}

// exp((x - top) / temperature), 1 at the top itself whatever it is
__device__ __forceinline__ float weight(float x, float top, float inverse) {
  return x == top ? 1.0f : expf((x - top) * inverse);
}

__device__ __forceinline__ bool above_floor(float x, float top, const DrawRow &d) {
  return x == top || (x - top) * d.inverse >= d.floor;
}

__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int d = 32; d; d >>= 1) v = fmaxf(v, __shfl_xor(v, d));
  return v;
}

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
  return v;
}

// The groups' largest logits and sums of weights; NaN counts as -inf.  FLOOR:
// the groups' largest are known, and the sums of the rows with a floor are made
// again over what is above it.
template <typename T, bool FLOOR>
__global__ __launch_bounds__(64 * kGroupWaves) void group_kernel(
    const typename T::store *__restrict__ logits, int64_t ld, int64_t V, Rules rules,
    const float *temperature, const float *min_p, GroupSum *groups, uint32_t per_row,
    uint32_t slices, int64_t tiles) {
  extern __shared__ uint32_t lds[];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
    const int64_t b = tile / slices;
    const uint32_t g0 = (uint32_t)(tile - b * slices) * waves, g = g0 + wave;
    const DrawRow d = draw_row(temperature, min_p, b);
    GroupSum *mine = groups + b * per_row;
    float top = -INFINITY;
    if (FLOOR) {
      if (d.greedy || d.floor == -INFINITY) continue;
      for (uint32_t i = lane; i < per_row; i += 64) top = fmaxf(top, mine[i].top);
      top = wave_max(top);
      bool any = false;  // a group of the workgroup's that reaches the floor
      for (int w = 0; w < waves && g0 + w < per_row; ++w) any |= above_floor(mine[g0 + w].top, top, d);
      if (!any) {
        if (lane == 0 && g < per_row) mine[g].sum = 0.0f;
        continue;
      }
    }
    float x[kSteps][8];
    int n[kSteps];
    group_logits<T>(logits + b * ld, (int64_t)g * kGroup, V, row_history(rules, b),
                    row_rules(rules, b), lds, x, n);
    float m = -INFINITY, sum = 0.0f;
#pragma unroll
    for (int s = 0; s < kSteps; ++s)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        x[s][j] = j < n[s] && x[s][j] == x[s][j] ? x[s][j] : -INFINITY;
        m = fmaxf(m, x[s][j]);
      }
    m = wave_max(m);
    if (m != -INFINITY) {
#pragma unroll
      for (int s = 0; s < kSteps; ++s)
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (!FLOOR || above_floor(x[s][j], top, d)) sum += weight(x[s][j], m, d.inverse);
      sum = wave_sum(sum);
    }
    if (lane == 0 && g < per_row) mine[g] = GroupSum{m, sum};
    __syncthreads();
  }
}

// -log(1 - u), u = (y + 1/2) / 2^32 with y the first word of the counter
__device__ __forceinline__ float variate(uint32_t i, uint32_t position, uint32_t domain,
                                         uint64_t seed) {
  const uint32_t y = philox4x32_10_word0(i, position, 0u, domain, (uint32_t)seed,
                                         (uint32_t)(seed >> 32));
  const float u = fminf(fmaf((float)y, 0x1p-32f, 0x1p-33f), 1.0f - 0x1p-24f);
  return -log1pf(-u);
}

// smallest (value, index) of the workgroup; values are not negative and not NaN
__device__ __forceinline__ uint64_t block_first(float value, uint32_t index, uint64_t *waves) {
  uint64_t k = (uint64_t)__builtin_bit_cast(uint32_t, value) << 32 | index;
#pragma unroll
  for (int d = 32; d; d >>= 1) {
    const uint64_t o = __shfl_xor((unsigned long long)k, d);
    k = o < k ? o : k;
  }
  if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = k;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kDrawWaves; ++w) k = waves[w] < k ? waves[w] : k;
  __syncthreads();
  return k;
}

// One workgroup per row: the group, then the token in it, one to a thread.
template <typename T>
__global__ __launch_bounds__(kDrawThreads) void draw_kernel(
    const typename T::store *__restrict__ logits, int64_t ld, int64_t B, int64_t V, Rules rules,
    const float *temperature, const float *min_p, const int64_t *__restrict__ seed,
    const int32_t *__restrict__ position, const GroupSum *__restrict__ groups, uint32_t per_row,
    int32_t *z, float *prob) {
  __shared__ uint32_t count[kGroup];
  __shared__ uint64_t firsts[kDrawWaves];
  __shared__ float parts[2][kDrawWaves];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int64_t b = blockIdx.x; b < B; b += gridDim.x) {
    const DrawRow d = draw_row(temperature, min_p, b);
    const GroupSum *mine = groups + b * per_row;
    const uint64_t s = (uint64_t)seed[b];
    const uint32_t pos = (uint32_t)position[b];
    const History h = row_history(rules, b);
    // the first tokens of the history, on their way before the group is known
    const words4 tokens = history_load(h, 4 * threadIdx.x);
    count[threadIdx.x] = 0;
    float top = -INFINITY;
    for (uint32_t g = threadIdx.x; g < per_row; g += kDrawThreads) top = fmaxf(top, mine[g].top);
    top = wave_max(top);
    if (lane == 0) parts[0][wave] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kDrawWaves; ++w) top = fmaxf(top, parts[0][w]);
    if (top == -INFINITY) {  // nothing may be drawn
      if (threadIdx.x == 0) {
        z[b] = -1;
        prob[b] = 0.0f;
      }
      __syncthreads();
      continue;
    }
    float best = INFINITY, total = 0.0f;
    uint32_t at = 0xFFFFFFFFu;
    for (uint32_t g = threadIdx.x; g < per_row; g += kDrawThreads) {
      const GroupSum q = mine[g];
      float v;
      if (d.greedy) {
        v = q.top == top ? 0.0f : INFINITY;
      } else {
        const float w = q.top == -INFINITY ? 0.0f : weight(q.top, top, d.inverse) * q.sum;
        total += w;
        v = variate(g, pos, 2u, s) / w;
      }
      if (v < best || at == 0xFFFFFFFFu) {
        best = v;
        at = g;
      }
    }
    total = wave_sum(total);
    if (lane == 0) parts[1][wave] = total;
    const uint32_t group = (uint32_t)block_first(best, at, firsts);
    total = 0.0f;
#pragma unroll
    for (int w = 0; w < kDrawWaves; ++w) total += parts[1][w];
    const int64_t first = (int64_t)group * kGroup, token = first + threadIdx.x;
    const float group_top = mine[group].top;
    const RowRules r = row_rules(rules, b);
    const bool there = token < V;
    float x = there ? T::up(logits[b * ld + token]) : -INFINITY;
    const float bias = there && r.bias ? r.bias[token] : 0.0f;
    const uint32_t allowed = there && r.mask ? r.mask[token >> 5] : 0xFFFFFFFFu;
    if (h.size) {
      history_count(h, 4 * threadIdx.x, tokens, first, kGroup, count);
      for (int64_t i = 4 * (threadIdx.x + kDrawThreads); i < h.size; i += 4 * kDrawThreads)
        history_count(h, i, history_load(h, i), first, kGroup, count);
      __syncthreads();
      x = ruled(x, count[threadIdx.x], r);
    }
    if (r.bias) x += bias;
    if (!(allowed >> (token & 31) & 1)) x = -INFINITY;
    float v = INFINITY;
    if (d.greedy)
      v = x == top ? 0.0f : INFINITY;
    else if (x == x && x != -INFINITY && above_floor(x, top, d))
      v = variate((uint32_t)token, pos, 3u, s) / weight(x, group_top, d.inverse);
    const uint32_t won = (uint32_t)block_first(v, threadIdx.x, firsts);
    if (threadIdx.x == won) {
      z[b] = (int32_t)token;
      const double share = x == top ? 1.0 : exp(((double)x - (double)top) / (double)d.temperature);
      prob[b] = d.greedy ? 1.0f : (float)(share / (double)total);
    }
    __syncthreads();
  }
}

}  // namespace lda
