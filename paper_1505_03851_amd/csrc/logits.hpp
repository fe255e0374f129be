// Logits of a language model: the rules that change them, and the draw of one
// token per row.
//
// The rules, in float and in this order, for token v of row b with c uses among
// the row's generated tokens:
//   x = seen ? (x > 0 ? x / repetition : x * repetition) : x   (seen: anywhere in
//                                        the history, the prompt included)
//   x = x - frequency * c                where c > 0
//   x = x - presence                     where c > 0
//   x = x + bias[v]
//   x = -inf                             where the mask's bit v is 0
//
// The draw: weights w_v = exp((x_v - max) / temperature), 0 below min_p.  With
// exponential variates E, argmin E_v / w_v is token v with probability
// w_v / sum w.  It is taken in two steps, the group of kGroup tokens by
// E_g / (sum of the group's weights), then the token inside it, so a row needs
// V / kGroup + kGroup variates and not V, and the second step reads one group.
// Which token wins depends on rounding only where the best two keys are within
// rounding of each other, in whatever order the sums are made: with a probability of
// at most the relative errors of the two, each a few 2^-24 and 2^-24 of (max - x) /
// temperature, so about 1e-6 of the draws and more where logits are large (none of
// 6M draws from 2,000 logits differed from the draw in 64 bits).  A search of
// partial sums for u * S would hang on the rounding of every one of V partial sums.
//
// What bounds them is not memory but a wavefront's chain (the row's numbers, its
// history, the counts in LDS, the rules) and, with every rule on, vector
// instructions: about 20 a logit under the rules, of which the division is half
// (it is the exact one, so that two logits that tie after a penalty tie here
// too), and 8 for its weight.  So a workgroup reads its row's history once for
// eight groups (one group to a workgroup: 39 us against 29 for the penalties of 256
// rows, 51.5 against 37 for 64 draws), rows are addressed from scalar registers (70
// vector registers are left: seven wavefronts fit a SIMD), and the logits are on
// their way while the history is counted.
//
// Measured on MI355X: 256 rows of 100,000 bfloat16 logits under a history of up
// to 4,096 tokens, a bias and masks 28 us (3.9 TB/s of the 109 MB that have to
// move; 17.6 us with no rules, 21 without the history); 64 draws from 100,000 with
// a history of up to 8,192, bias, masks, temperatures and floors 36 us (17 the
// sums, 12 the sums above the floors, 9 the races, in a trace, which keeps them
// apart); 256 plain draws from 49,999 floats 18.6 us (13 and 7); one draw from
// 32,768, in one launch, 10.5 us on the GPU and 13.5 a call.
#pragma once

#include "elements.hpp"
#include "philox.hpp"
#include "wave_ops.hpp"

namespace lda {

constexpr int kGroup = 1024;  // tokens of a group, the unit of a wavefront
constexpr int kSteps = kGroup / 512;
constexpr int kGroupWaves = 8;      // groups of a workgroup, at most
constexpr int kDrawThreads = 1024;  // of a workgroup that draws: one for each token of a group
constexpr int kDrawWaves = kDrawThreads / 64;
constexpr int kShortGroups = 2 * kDrawWaves;  // of a row that one launch draws from
constexpr uint32_t kSeen = 0x80000000u;

struct Rules {
  const int32_t *history;  // [B][ld_history], or null; ld_history 0: one row
  int64_t ld_history;
  const int32_t *lengths, *prompt;  // [B]; prompt null: 0
  const float *repetition, *frequency, *presence;  // [B] or null
  const float *bias;                               // [B][ld_bias] or null; ld_bias 0: one row
  int64_t ld_bias;
  const uint32_t *mask;  // [B][ld_mask] or null; ld_mask 0: one row
  int64_t ld_mask;
  int32_t capacity;  // history's columns
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
  x = x > 0.0f ? x / r.repetition : rounded(x * r.repetition);
  const uint32_t c = count & ~kSeen;
  const float cut = rounded(r.frequency * (float)c);
  x -= c ? cut : 0.0f;  // (an infinite frequency times 0 is NaN)
  return x - (c ? r.presence : 0.0f);
}

// Where the count of a group's token lies: a lane's two blocks of four tokens
// are 256 words apart, so that 64 lanes read 16 bytes each from neighbouring
// banks.
__device__ __forceinline__ uint32_t count_slot(uint32_t at) {
  return (at & ~511u) | (at & 4) << 6 | (at >> 1 & 252) | (at & 3);
}

// A row's history; the first `prompt` of its tokens are not generated.
struct History {
  const int32_t *tokens;
  int32_t size, prompt;  // 0 tokens where there is no history; the prompt as given
};

__device__ __forceinline__ History row_history(const Rules &r, int64_t b) {
  if (!r.history) return History{nullptr, 0, 0};
  const int32_t n = r.lengths[b] < r.capacity ? r.lengths[b] : r.capacity;
  return History{r.history + b * r.ld_history, n > 0 ? n : 0, r.prompt ? r.prompt[b] : 0};
}

// Four tokens from number i on; those past the end are -1.
__device__ __forceinline__ words4 history_load(const History &h, uint32_t i) {
  words4 t;
  if (i + 4 <= (uint32_t)h.size) {
    t = *reinterpret_cast<const words4_any *>(h.tokens + i);
  } else {
#pragma unroll
    for (uint32_t j = 0; j < 4; ++j)
      t[j] = i + j < (uint32_t)h.size ? (uint32_t)h.tokens[i + j] : 0xFFFFFFFFu;
  }
  return t;
}

// Adds the tokens t (of which the first is number i) that lie in [first, first +
// size) to `count`: generated tokens in the low bits, kSeen for the prompt's.
// (As an unsigned number a negative token lies past every vocabulary: where the
// difference wraps into the range, it is to a place past the row's end.)
__device__ __forceinline__ void history_count(const History &h, uint32_t i, words4 t,
                                              uint32_t first, uint32_t size, uint32_t *count) {
  const int32_t prompt = h.prompt - (int32_t)i;  // (neither is negative)
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint32_t at = t[j] - first;
    if (at >= size) continue;
    if (j < prompt)
      atomicOr(&count[count_slot(at)], kSeen);
    else
      atomicAdd(&count[count_slot(at)], 1u);
  }
}

// The first of a row's history, two loads of a lane, which can be on their way
// while other things are.
struct Tokens {
  words4 t[2];
};

__device__ __forceinline__ Tokens load_tokens(const History &h) {
  const uint32_t i = 4 * threadIdx.x;
  return Tokens{{history_load(h, i), history_load(h, i + 4 * blockDim.x)}};
}

// The uses of the tokens [first, first + size) in a row's history, counted in
// LDS (which the caller has cleared and synchronised) by the whole workgroup;
// `ahead`: load_tokens of it.
__device__ __forceinline__ void count_history(History h, Tokens ahead, uint32_t first,
                                              uint32_t size, uint32_t *count) {
  // A negative prompt is an empty one.  The maximum is taken here and not where the
  // prompt is read (the compiler would move it back there): it waits for the read,
  // which is to be on its way with the logits' (penalties of 256 rows of 100,000
  // logits 28.8 us against 30.1).
  asm volatile("" : "+v"(h.prompt));
  h.prompt = h.prompt > 0 ? h.prompt : 0;
  const uint32_t step = 4 * blockDim.x;
  for (uint32_t i = 4 * threadIdx.x, start = 0; start < (uint32_t)h.size;
       i += 2 * step, start += 2 * step) {
    // the next two loads on their way while these are counted
    Tokens next;
    const bool more = start + 2 * step < (uint32_t)h.size;
    if (more) next = Tokens{{history_load(h, i + 2 * step), history_load(h, i + 3 * step)}};
    history_count(h, i, ahead.t[0], first, size, count);
    history_count(h, i + step, ahead.t[1], first, size, count);
    if (more) ahead = next;
  }
}

// A wavefront's group of a row as loaded: token first + 512 s + 8 lane + j is
// element j of step s; n[s] of a lane's 8 exist.
template <typename T>
struct Group {
  Packed<T, 8> x[kSteps];
  uint32_t allowed[kSteps];  // mask bits of the lane's tokens, from bit 0
  int n[kSteps];
};

template <typename T>
__device__ __forceinline__ void load_group(const typename T::store *row, int64_t first, int64_t V,
                                           const RowRules &r, Group<T> &g) {
  // (row and first are the same for the wavefront: 32-bit offsets from there)
  const int64_t rest = V - first;
  const int32_t left = rest < 0 ? 0 : rest < kGroup ? (int32_t)rest : kGroup;
  const typename T::store *x = row + first;
  const uint32_t *mask = r.mask + (first >> 5);
#pragma unroll
  for (int s = 0; s < kSteps; ++s) {
    const uint32_t at = s * 512 + (threadIdx.x & 63) * 8;
    const int32_t n = left - (int32_t)at;
    g.n[s] = n < 0 ? 0 : n < 8 ? n : 8;
    g.x[s] = load_packed<T, 8>(x + at, g.n[s]);
    g.allowed[s] = r.mask && g.n[s] > 0 ? mask[at >> 5] >> (at & 31) : 0xFFu;
  }
}

// The group's logits in float under the rules.  `count`: the uses of the group's
// tokens in LDS, or null.
template <typename T>
__device__ __forceinline__ void rule_group(const Group<T> &g, int64_t first, const uint32_t *count, const RowRules &r,
                                           float (&x)[kSteps][8]) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int s = 0; s < kSteps; ++s) {
    float bias[8];
    if (r.bias) load_elements<F32, 8>(r.bias + first + (uint32_t)(s * 512 + lane * 8), g.n[s], bias);
#pragma unroll
    for (int j = 0; j < 8; ++j) x[s][j] = T::up(g.x[s].v[j]);
    if (count) {
      const words4 *mine = reinterpret_cast<const words4 *>(count + s * 512) + lane;
      const words4 low = mine[0], high = mine[64];
      uint32_t c[8], any = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        c[j] = j < 4 ? low[j & 3] : high[j & 3];
        any |= c[j];
      }
      if (any) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          if (c[j]) x[s][j] = ruled(x[s][j], c[j], r);
        }
      }
    }
    if (r.bias) {
#pragma unroll
      for (int j = 0; j < 8; ++j) x[s][j] += bias[j];
    }
    if (r.mask) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        // all ones where allowed; two instructions a logit
        const uint32_t keep = (uint32_t)((int32_t)(g.allowed[s] << (31 - j)) >> 31);
        const uint32_t bits = __builtin_bit_cast(uint32_t, x[s][j]);
        x[s][j] = __builtin_bit_cast(float, (bits & keep) | (0xFF800000u & ~keep));
      }
    }
  }
}

// a wavefront's own group
__device__ __forceinline__ void clear_counts(uint32_t *count) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int i = 0; i < 2 * kSteps; ++i) reinterpret_cast<words4 *>(count)[i * 64 + lane] = words4{};
}

// A workgroup takes a group of one row for each of its wavefronts; the logits
// are on their way while it counts the row's history.
template <typename T>
__global__ __launch_bounds__(64 * kGroupWaves) void penalise_kernel(
    const typename T::store *logits, int64_t ld, typename T::store *out, int64_t ldo, int64_t V,
    Rules rules, uint32_t slices, int64_t tiles) {
  extern __shared__ uint32_t lds[];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
  uint32_t *count = lds + wave * kGroup;
  for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
    const int64_t b = tile / slices, start = (tile - b * slices) * waves * kGroup;
    const int64_t first = start + wave * kGroup;
    const RowRules r = row_rules(rules, b);
    const History h = row_history(rules, b);
    const Tokens ahead = load_tokens(h);
    Group<T> g;
    load_group<T>(logits + b * ld, first, V, r, g);
    if (h.size) {
      clear_counts(count);
      __syncthreads();
      count_history(h, ahead, (uint32_t)start, waves * kGroup, lds);
      __syncthreads();
    }
    float x[kSteps][8];
    rule_group<T>(g, first, h.size ? count : nullptr, r, x);
#pragma unroll
    for (int s = 0; s < kSteps; ++s)
      store_elements<T, 8, true>(out + b * ldo + first + (uint32_t)(s * 512 + (threadIdx.x & 63) * 8),
                           g.n[s], x[s]);
    __syncthreads();
  }
}

struct GroupSum {
  float top, sum;  // the largest logit of a group, and sum exp((x - top) / temperature)
};

struct DrawRow {
  float temperature;
  float scale;  // log2(e) / temperature
  float floor;  // log2(min_p); -inf: none
  bool greedy;  // the row takes its largest logit
};

__device__ __forceinline__ DrawRow draw_row(const float *temperature, const float *min_p,
                                            int64_t b) {
  const float given = temperature ? temperature[b] : 1.0f;
  // an infinite temperature would make -inf * 0 of the logits that may not be drawn
  const float t = fminf(given, 1e30f);
  const float p = min_p ? min_p[b] : 0.0f;
  return DrawRow{t, fminf(1.44269504f / t, 3e38f),
                 p > 0.0f ? log2f(fminf(p, 1.0f)) : -INFINITY, !(given > 0.0f)};
}

// exp((x - top) / temperature), 1 at the top itself whatever it is
__device__ __forceinline__ float weight(float x, float top, const DrawRow &d) {
  return x == top ? 1.0f : __builtin_amdgcn_exp2f((x - top) * d.scale);
}

__device__ __forceinline__ bool above_floor(float x, float top, const DrawRow &d) {
  return x == top || (x - top) * d.scale >= d.floor;
}

// The smallest value of a wavefront (not negative, not NaN: their bits are in
// their order) and the lowest index that has it.
struct First {
  uint32_t value, index;
};

__device__ __forceinline__ First wave_first(First mine) {
  const uint32_t v = wave_min(mine.value);
  return First{v, wave_min(mine.value == v ? mine.index : 0xFFFFFFFFu)};
}

// -log(1 - u), u = (y + 1/2) / 2^32 with y the first word of the counter
__device__ __forceinline__ float variate(uint32_t i, uint32_t position, uint32_t domain,
                                         uint64_t seed) {
  const uint32_t y = philox4x32_10_word0(i, position, 0u, domain, (uint32_t)seed,
                                         (uint32_t)(seed >> 32));
  const float u = fminf(fmaf((float)y, 0x1p-32f, 0x1p-33f), 1.0f - 0x1p-24f);
  return -log1pf(-u);
}

// The largest logit of a wavefront's group (NaN, and what does not exist: -inf)
// and the sum of its weights to that, over what lies above the floor under
// `row_top` where FLOOR.
template <bool FLOOR>
__device__ __forceinline__ GroupSum group_sum(float (&x)[kSteps][8], const int (&n)[kSteps],
                                              bool full, float row_top, const DrawRow &d) {
  float top = -INFINITY, sum = 0.0f;
#pragma unroll
  for (int s = 0; s < kSteps; ++s)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if (!full) x[s][j] = j < n[s] ? x[s][j] : -INFINITY;
      x[s][j] = fmaxf(x[s][j], -INFINITY);  // (the maximum of NaN and a number is the number)
      top = fmaxf(top, x[s][j]);
    }
  top = wave_max(top);
  if (top == -INFINITY || (d.greedy && !FLOOR)) return GroupSum{top, 0.0f};
  if (FLOOR) {
#pragma unroll
    for (int s = 0; s < kSteps; ++s)
#pragma unroll
      for (int j = 0; j < 8; ++j)
        x[s][j] = above_floor(x[s][j], row_top, d) ? x[s][j] : -INFINITY;
  }
  if (top == INFINITY) {  // shared by the logits of +inf
#pragma unroll
    for (int s = 0; s < kSteps; ++s)
#pragma unroll
      for (int j = 0; j < 8; ++j) sum += x[s][j] == top ? 1.0f : 0.0f;
  } else {
#pragma unroll
    for (int s = 0; s < kSteps; ++s)
#pragma unroll
      for (int j = 0; j < 8; ++j) sum += __builtin_amdgcn_exp2f((x[s][j] - top) * d.scale);
  }
  return GroupSum{top, wave_sum(sum)};
}

// The groups' largest logits and sums of weights, a group to a wavefront.
// FLOOR: the groups' largest are known, and the sums of the rows with a floor
// are made again over what is above it.
template <typename T, bool FLOOR>
__global__ __launch_bounds__(64 * kGroupWaves) void group_kernel(
    const typename T::store *__restrict__ logits, int64_t ld, int64_t V, Rules rules,
    const float *temperature, const float *min_p, GroupSum *groups, uint32_t per_row,
    uint32_t slices, int64_t tiles) {
  extern __shared__ uint32_t lds[];
  const int lane = threadIdx.x & 63, waves = blockDim.x >> 6;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  uint32_t *count = lds + wave * kGroup;
  for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
    const int64_t b = tile / slices;
    const uint32_t g0 = (uint32_t)(tile - b * slices) * waves, g = g0 + wave;
    const DrawRow d = draw_row(temperature, min_p, b);
    GroupSum *mine = groups + b * per_row;
    float top = -INFINITY;
    if (FLOOR && (d.greedy || d.floor == -INFINITY)) continue;
    const int64_t first = (int64_t)g * kGroup;
    const RowRules r = row_rules(rules, b);
    const History h = row_history(rules, b);
    const Tokens ahead = load_tokens(h);
    Group<T> q;
    load_group<T>(logits + b * ld, first, V, r, q);
    if (FLOOR) {
      for (uint32_t i = lane; i < per_row; i += 64) top = fmaxf(top, mine[i].top);
      top = wave_max(top);
      // whether a group of the workgroup's reaches the floor
      const bool reaches =
          lane < waves && g0 + lane < per_row && above_floor(mine[g0 + lane].top, top, d);
      if (!__ballot(reaches)) {
        if (lane == 0 && g < per_row) mine[g].sum = 0.0f;
        continue;
      }
    }
    if (h.size) {
      clear_counts(count);
      __syncthreads();
      count_history(h, ahead, g0 * kGroup, waves * kGroup, lds);
      __syncthreads();
    }
    float x[kSteps][8];
    rule_group<T>(q, first, h.size ? count : nullptr, r, x);
    const GroupSum sum = group_sum<FLOOR>(x, q.n, first + kGroup <= V, top, d);
    if (lane == 0 && g < per_row) {
      // (with a floor the row's other workgroups still read the groups' largest)
      if (FLOOR)
        mine[g].sum = sum.sum;
      else
        mine[g] = sum;
    }
    __syncthreads();
  }
}

// The last step of a workgroup that has a token to each thread: the one with the
// smallest key `v` is drawn, and its share of `total` its probability.
__device__ __forceinline__ void choose_token(float v, float x, float top, float total,
                                             uint32_t token, const DrawRow &d, First *firsts,
                                             int32_t *z, float *prob) {
  const int lane = threadIdx.x & 63;
  const First of_wave = wave_first(First{__builtin_bit_cast(uint32_t, v), threadIdx.x});
  if (lane == 0) firsts[threadIdx.x >> 6] = of_wave;
  __syncthreads();
  const First won = wave_first(lane < kDrawWaves ? firsts[lane] : First{0xFFFFFFFFu, 0xFFFFFFFFu});
  if (threadIdx.x != won.index) return;
  *z = (int32_t)token;
  // the exponent in 64 bits: in 32 its rounding would be the largest error
  const double y = ((double)x - (double)top) / (double)d.temperature * 1.4426950408889634;
  const double whole = rint(y);
  const float share =
      x == top ? 1.0f
               : ldexpf(__builtin_amdgcn_exp2f((float)(y - whole)), (int)fmax(whole, -1000.0));
  *prob = d.greedy ? 1.0f : share / total;
}

// One workgroup per row: the groups' race (by every wavefront for itself), then
// the race of the group's tokens, one to a thread.
template <typename T>
__global__ __launch_bounds__(kDrawThreads) void draw_kernel(
    const typename T::store *__restrict__ logits, int64_t ld, int64_t B, int64_t V, Rules rules,
    const float *__restrict__ temperature, const float *__restrict__ min_p,
    const int64_t *__restrict__ seed, const int32_t *__restrict__ position,
    const GroupSum *__restrict__ groups, uint32_t per_row, int32_t *__restrict__ z,
    float *__restrict__ prob) {
  __shared__ uint32_t count[kGroup];
  __shared__ First firsts[kDrawWaves];
  const int lane = threadIdx.x & 63;
  for (int64_t b = blockIdx.x; b < B; b += gridDim.x) {
    const DrawRow d = draw_row(temperature, min_p, b);
    const GroupSum *mine = groups + b * per_row;
    const uint64_t s = (uint64_t)seed[b];
    const uint32_t pos = (uint32_t)position[b];
    const RowRules r = row_rules(rules, b);
    const History h = row_history(rules, b);
    // the first of the history's tokens, on their way before the group is known
    const Tokens ahead = load_tokens(h);
    count[threadIdx.x] = 0;
    float top = -INFINITY;
    for (uint32_t g = lane; g < per_row; g += 64) top = fmaxf(top, mine[g].top);
    top = wave_max(top);
    if (top == -INFINITY) {  // nothing may be drawn
      if (threadIdx.x == 0) {
        z[b] = -1;
        prob[b] = 0.0f;
      }
      continue;
    }
    First best{0x7F800000u, 0xFFFFFFFFu};
    float total = 0.0f;
    for (uint32_t g = lane; g < per_row; g += 64) {
      const GroupSum q = mine[g];
      float v;
      if (d.greedy) {
        v = q.top == top ? 0.0f : INFINITY;
      } else {
        const float w = q.top == -INFINITY ? 0.0f : weight(q.top, top, d) * q.sum;
        total += w;
        v = variate(g, pos, 2u, s) / w;
      }
      const uint32_t bits = __builtin_bit_cast(uint32_t, v);
      if (bits < best.value || best.index == 0xFFFFFFFFu) best = First{bits, g};
    }
    total = wave_sum(total);
    const uint32_t group = wave_first(best).index;
    const uint32_t first = group * kGroup;
    const int64_t token = (int64_t)first + threadIdx.x;
    const float group_top = mine[group].top;
    const bool there = token < V;
    float x = there ? T::up(logits[b * ld + token]) : -INFINITY;
    const float bias = there && r.bias ? r.bias[token] : 0.0f;
    const uint32_t allowed = there && r.mask ? r.mask[token >> 5] : 0xFFFFFFFFu;
    // a token's own variate, on its way with its logit
    const float own = d.greedy ? 0.0f : variate((uint32_t)token, pos, 3u, s);
    if (h.size) {
      __syncthreads();
      count_history(h, ahead, first, kGroup, count);
      __syncthreads();
      const uint32_t c = count[count_slot(threadIdx.x)];
      if (c) x = ruled(x, c, r);
    }
    if (r.bias) x += bias;
    // (what lies past the row's end may have met a rule: its number in the history)
    if (!there || !(allowed >> (token & 31) & 1)) x = -INFINITY;
    float v = INFINITY;
    if (d.greedy)
      v = x == top ? 0.0f : INFINITY;
    else if (x == x && x != -INFINITY && above_floor(x, top, d))
      v = own / weight(x, group_top, d);
    choose_token(v, x, top, total, (uint32_t)token, d, firsts, z + b, prob + b);
    __syncthreads();
  }
}

// A short row (up to R kDrawWaves groups) in one workgroup and one launch: R groups
// to a wavefront, whose logits under the rules stay in registers for the floor's
// second sums and for the race of the tokens.
template <typename T, int R>
__global__ __launch_bounds__(kDrawThreads) void short_draw_kernel(
    const typename T::store *__restrict__ logits, int64_t ld, int64_t B, int64_t V, Rules rules,
    const float *__restrict__ temperature, const float *__restrict__ min_p,
    const int64_t *__restrict__ seed, const int32_t *__restrict__ position, int32_t *__restrict__ z,
    float *__restrict__ prob) {
  constexpr int kGroups = R * kDrawWaves;
  static_assert(kGroups <= 64, "a group to a lane");
  extern __shared__ uint32_t lds[];  // the counts of all groups, where there is a history
  __shared__ GroupSum sums[kGroups];
  __shared__ float again[kGroups], winners[kGroup];
  __shared__ First firsts[kDrawWaves];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  for (int64_t b = blockIdx.x; b < B; b += gridDim.x) {
    const RowRules r = row_rules(rules, b);
    const History h = row_history(rules, b);
    const Tokens ahead = load_tokens(h);
    Group<T> q[R];
#pragma unroll
    for (int i = 0; i < R; ++i)
      load_group<T>(logits + b * ld, (int64_t)(i * kDrawWaves + wave) * kGroup, V, r, q[i]);
    const DrawRow d = draw_row(temperature, min_p, b);
    const uint64_t s = (uint64_t)seed[b];
    const uint32_t pos = (uint32_t)position[b];
    if (h.size) {
#pragma unroll
      for (int i = 0; i < R; ++i) clear_counts(lds + (i * kDrawWaves + wave) * kGroup);
      __syncthreads();
      count_history(h, ahead, 0, kGroups * kGroup, lds);
      __syncthreads();
    }
    float x[R][kSteps][8];
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int g = i * kDrawWaves + wave;
      const int64_t first = (int64_t)g * kGroup;
      rule_group<T>(q[i], first, h.size ? lds + g * kGroup : nullptr, r, x[i]);
      const GroupSum sum = group_sum<false>(x[i], q[i].n, first + kGroup <= V, 0.0f, d);
      if (lane == 0) sums[g] = sum;
    }
    // a lane's group, whose variate does not wait for its sum
    const float own = lane < kGroups ? variate(lane, pos, 2u, s) : 0.0f;
    __syncthreads();
    GroupSum mine = lane < kGroups ? sums[lane] : GroupSum{-INFINITY, 0.0f};
    const float top = wave_max(mine.top);
    if (top == -INFINITY) {  // nothing may be drawn
      if (threadIdx.x == 0) {
        z[b] = -1;
        prob[b] = 0.0f;
      }
      __syncthreads();
      continue;
    }
    if (!d.greedy && d.floor != -INFINITY) {
#pragma unroll
      for (int i = 0; i < R; ++i) {
        const int g = i * kDrawWaves + wave;
        float sum = 0.0f;
        if (above_floor(sums[g].top, top, d))
          sum = group_sum<true>(x[i], q[i].n, true, top, d).sum;
        if (lane == 0) again[g] = sum;
      }
      __syncthreads();
      mine.sum = lane < kGroups ? again[lane] : 0.0f;
    }
    const float w = mine.top == -INFINITY || d.greedy ? 0.0f : weight(mine.top, top, d) * mine.sum;
    const float total = wave_sum(w);
    const float key = d.greedy ? (mine.top == top ? 0.0f : INFINITY) : own / w;
    const uint32_t group =
        wave_first(First{lane < kGroups ? __builtin_bit_cast(uint32_t, key) : 0xFFFFFFFFu,
                         (uint32_t)lane}).index;
    const uint32_t token = group * kGroup + threadIdx.x;
    const float token_own = d.greedy ? 0.0f : variate(token, pos, 3u, s);
#pragma unroll
    for (int i = 0; i < R; ++i) {
      if ((uint32_t)(i * kDrawWaves + wave) != group) continue;
#pragma unroll
      for (int k = 0; k < kSteps; ++k)
#pragma unroll
        for (int j = 0; j < 8; ++j) winners[k * 512 + lane * 8 + j] = x[i][k][j];
    }
    const float group_top = sums[group].top;
    __syncthreads();
    const float mine_x = winners[threadIdx.x];
    float v = INFINITY;
    if (d.greedy)
      v = mine_x == top ? 0.0f : INFINITY;
    else if (mine_x != -INFINITY && above_floor(mine_x, top, d))
      v = token_own / weight(mine_x, group_top, d);
    choose_token(v, mine_x, top, total, token, d, firsts, z + b, prob + b);
    __syncthreads();
  }
}

}  // namespace lda
