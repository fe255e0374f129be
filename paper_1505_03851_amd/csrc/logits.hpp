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

constexpr int kLogitThreads = 256;
constexpr int kLogitWaves = kLogitThreads / 64;
constexpr int kGroup = 1024;  // tokens of a group, the unit of a wavefront
constexpr int kGroupSteps = kGroup / 512;
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

// The uses of the tokens [first, first + size) in row b's history, counted in
// LDS: generated tokens in the low bits, kSeen for those of the prompt.  The
// whole workgroup calls it; false where the row has no history.
__device__ __forceinline__ bool count_history(const Rules &r, int64_t b, int64_t first, int size,
                                              uint32_t *count) {
  if (!r.history) return false;
  int64_t n = r.lengths[b];
  n = n < r.capacity ? n : r.capacity;
  if (n <= 0) return false;
  const int64_t prompt = r.prompt ? r.prompt[b] : 0;
  const int32_t *h = r.history + b * r.ld_history;
  for (int i = threadIdx.x; i < size; i += kLogitThreads) count[i] = 0;
  __syncthreads();
  for (int64_t i = threadIdx.x; i < n; i += kLogitThreads) {
    const int64_t at = (int64_t)h[i] - first;
    if (at < 0 || at >= size) continue;
    if (i < prompt)
      atomicOr(&count[at], kSeen);
    else
      atomicAdd(&count[at], 1u);
  }
  __syncthreads();
  return true;
}

// 8 logits of a row from token v on, under the rules; n of them exist
template <typename T>
__device__ __forceinline__ void ruled_logits(const typename T::store *row, int64_t v, int n,
                                             const uint32_t *count, const RowRules &r,
                                             float (&x)[8]) {
  load_elements<T, 8>(row + v, n, x);
  if (count) {
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = ruled(x[j], count[j], r);
  }
  if (r.bias) {
    float b[8];
    load_elements<F32, 8>(r.bias + v, n, b);
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] += b[j];
  }
  if (r.mask) {
    const uint32_t bits = r.mask[v >> 5] >> (v & 31);
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = bits >> j & 1 ? x[j] : -INFINITY;
  }
}

// A workgroup takes `slice` tokens of one row.
template <typename T>
__global__ __launch_bounds__(kLogitThreads) void penalise_kernel(
    const typename T::store *logits, int64_t ld, typename T::store *out, int64_t ldo, int64_t V,
    Rules rules, int slice, uint32_t slices, int64_t tiles) {
  extern __shared__ uint32_t count[];
  for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
    const int64_t b = tile / slices;
    const int64_t first = (tile - b * slices) * slice;
    const int size = V - first < slice ? (int)(V - first) : slice;
    const RowRules r = row_rules(rules, b);
    const bool counted = count_history(rules, b, first, slice, count);
    for (int i = (int)threadIdx.x * 8; i < size; i += kLogitThreads * 8) {
      float x[8];
      const int n = size - i < 8 ? size - i : 8;
      ruled_logits<T>(logits + b * ld, first + i, n, counted ? count + i : nullptr, r, x);
      store_elements<T, 8>(out + b * ldo + first + i, n, x);
    }
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

// A wavefront's group of a row, 8 logits of each of kGroupSteps steps per lane;
// NaN counts as -inf.
template <typename T>
__device__ __forceinline__ void group_logits(const typename T::store *row, int64_t first, int64_t V,
                                             const uint32_t *count, const RowRules &r,
                                             float (&x)[kGroupSteps][8]) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int s = 0; s < kGroupSteps; ++s) {
    const int i = s * 512 + lane * 8;
    const int64_t left = V - first - i;
    const int n = left < 8 ? (left > 0 ? (int)left : 0) : 8;
#pragma unroll
    for (int j = 0; j < 8; ++j) x[s][j] = -INFINITY;
    if (n > 0) ruled_logits<T>(row, first + i, n, count ? count + i : nullptr, r, x[s]);
#pragma unroll
    for (int j = 0; j < 8; ++j) x[s][j] = j < n && x[s][j] == x[s][j] ? x[s][j] : -INFINITY;
  }
}

// The groups' largest logits and sums of weights; a workgroup takes `slice`
// tokens of one row, a wavefront a group at a time.  FLOOR: the groups' largest
// are known, and the sums of the rows with a floor are made again over what is
// above it.
template <typename T, bool FLOOR>
__global__ __launch_bounds__(kLogitThreads) void group_kernel(
    const typename T::store *__restrict__ logits, int64_t ld, int64_t V, Rules rules,
    const float *temperature, const float *min_p, GroupSum *groups, uint32_t per_row, int slice,
    uint32_t slices, int64_t tiles) {
  extern __shared__ uint32_t count[];
  const int lane = threadIdx.x & 63;
  for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
    const int64_t b = tile / slices;
    const int64_t first = (tile - b * slices) * slice;
    const DrawRow d = draw_row(temperature, min_p, b);
    GroupSum *mine = groups + b * per_row;
    float top = -INFINITY;
    if (FLOOR) {
      if (d.greedy || d.floor == -INFINITY) continue;
      for (uint32_t g = lane; g < per_row; g += 64) top = fmaxf(top, mine[g].top);
      top = wave_max(top);
    }
    const RowRules r = row_rules(rules, b);
    const bool counted = count_history(rules, b, first, slice, count);
    for (int i = (int)(threadIdx.x >> 6) * kGroup; i < slice && first + i < V;
         i += kLogitWaves * kGroup) {
      const int64_t g = (first + i) / kGroup;
      if (FLOOR && !above_floor(mine[g].top, top, d)) {
        if (lane == 0) mine[g].sum = 0.0f;
        continue;
      }
      float x[kGroupSteps][8];
      group_logits<T>(logits + b * ld, first + i, V, counted ? count + i : nullptr, r, x);
      float m = -INFINITY, sum = 0.0f;
#pragma unroll
      for (int s = 0; s < kGroupSteps; ++s)
#pragma unroll
        for (int j = 0; j < 8; ++j) m = fmaxf(m, x[s][j]);
      m = wave_max(m);
      if (m != -INFINITY) {
#pragma unroll
        for (int s = 0; s < kGroupSteps; ++s)
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (!FLOOR || above_floor(x[s][j], top, d)) sum += weight(x[s][j], m, d.inverse);
        sum = wave_sum(sum);
      }
      if (lane == 0) mine[g] = GroupSum{m, sum};
    }
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
  for (int w = 0; w < kLogitWaves; ++w) k = waves[w] < k ? waves[w] : k;
  __syncthreads();
  return k;
}

// One workgroup per row: the group, then the token in it.
template <typename T>
__global__ __launch_bounds__(kLogitThreads) void draw_kernel(
    const typename T::store *__restrict__ logits, int64_t ld, int64_t B, int64_t V, Rules rules,
    const float *temperature, const float *min_p, const int64_t *__restrict__ seed,
    const int32_t *__restrict__ position, const GroupSum *__restrict__ groups, uint32_t per_row,
    int32_t *z, float *prob) {
  __shared__ uint32_t count[kGroup];
  __shared__ uint64_t firsts[kLogitWaves];
  __shared__ float parts[2][kLogitWaves];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int64_t b = blockIdx.x; b < B; b += gridDim.x) {
    const DrawRow d = draw_row(temperature, min_p, b);
    const GroupSum *mine = groups + b * per_row;
    const uint64_t s = (uint64_t)seed[b];
    const uint32_t pos = (uint32_t)position[b];
    float top = -INFINITY;
    for (uint32_t g = threadIdx.x; g < per_row; g += kLogitThreads) top = fmaxf(top, mine[g].top);
    top = wave_max(top);
    if (lane == 0) parts[0][wave] = top;
    __syncthreads();
    for (int w = 0; w < kLogitWaves; ++w) top = fmaxf(top, parts[0][w]);
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
    for (uint32_t g = threadIdx.x; g < per_row; g += kLogitThreads) {
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
    for (int w = 0; w < kLogitWaves; ++w) total += parts[1][w];
    const int64_t first = (int64_t)group * kGroup;
    const float group_top = mine[group].top;
    const RowRules r = row_rules(rules, b);
    const bool counted = count_history(rules, b, first, kGroup, count);
    best = INFINITY;
    at = 0xFFFFFFFFu;
    float mine_x = 0.0f;
    const int i = (int)threadIdx.x * 8;
    if (i < kGroup && first + i < V) {
      float x[8];
      const int n = V - first - i < 8 ? (int)(V - first - i) : 8;
      ruled_logits<T>(logits + b * ld, first + i, n, counted ? count + i : nullptr, r, x);
      for (int j = 0; j < n; ++j) {
        float v;
        if (d.greedy)
          v = x[j] == top ? 0.0f : INFINITY;
        else if (x[j] == x[j] && x[j] != -INFINITY && above_floor(x[j], top, d))
          v = variate((uint32_t)(first + i + j), pos, 3u, s) / weight(x[j], group_top, d.inverse);
        else
          v = INFINITY;
        if (v < best || at == 0xFFFFFFFFu) {
          best = v;
          at = (uint32_t)(i + j);
          mine_x = x[j];
        }
      }
    }
    const uint32_t won = (uint32_t)block_first(best, at, firsts);
    if (at == won) {
      z[b] = (int32_t)(first + won);
      const double share =
          mine_x == top ? 1.0 : exp(((double)mine_x - (double)top) / (double)d.temperature);
      prob[b] = d.greedy ? 1.0f : (float)(share / (double)total);
    }
    __syncthreads();
  }
}

}  // namespace lda
