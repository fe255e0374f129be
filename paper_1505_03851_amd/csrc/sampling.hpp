// The next token of each row of logits by the row's uniform number, among the likeliest.
//
//   w_v = exp((x_v - max) / temperature); tokens in the order of falling x, equal ones by
//   number: the first top_k stay, of those the fewest whose w reach the share top_p, of
//   those the ones of at least min_p.  z = the first token, by number, up to which the
//   weights that stay sum to more than u times all of them.
//
// Whether u S lies before or after a partial sum hangs on every digit of it: with sums in
// float one draw in a thousand would be its neighbour's.  So weights are computed in
// double and held as whole multiples of 2^-F (F = 46, less for more than 131,072 tokens):
// their sums are exact, whatever their order, and so are all comparisons of sums.  What
// is below half a step of the largest weight is never drawn.
//
// Every question (the k-th token, the token that reaches a share, a tie's number, the
// token at u S) is one search: in an interval of keys (a logit's order, or a token's
// number) that holds the answer, members add their amounts (1, or their weight) to 2,048
// bins in LDS, the bin where the running sum reaches the target becomes the interval,
// until it is one key.
#pragma once

#include "elements.hpp"
#include "wave_ops.hpp"

namespace lda {

constexpr int kSampleThreads = 1024;
constexpr int kSampleWaves = kSampleThreads / 64;
constexpr int kBins = 2 * kSampleThreads;

// Logits as keys that rise as they fall: 32 bits of a float, 16 of a 16-bit type.
template <typename T>
struct OrderKey;
template <>
struct OrderKey<F32> {
  static constexpr int kShift = 0;
};
template <>
struct OrderKey<Bf16> {
  static constexpr int kShift = 16;
};
template <>
struct OrderKey<F16> {
  static constexpr int kShift = 13;  // a half's digits as a float
};

template <typename T>
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t b = __builtin_bit_cast(uint32_t, x + 0.0f);  // (-0 is 0)
  return ~(b & 0x80000000u ? ~b : b | 0x80000000u) >> OrderKey<T>::kShift;
}

template <typename T>
__device__ __forceinline__ float logit_of(uint32_t key) {
  const uint32_t b = ~(key << OrderKey<T>::kShift | ((1u << OrderKey<T>::kShift) - 1));
  const uint32_t bits = b & 0x80000000u ? b & 0x7FFFFFFFu : ~b;
  return __builtin_bit_cast(float, bits & ~((1u << OrderKey<T>::kShift) - 1));
}

// A row's weights.
struct Weights {
  float top;
  double per;    // log2(e) / temperature
  double floor;  // min_p
  int digits;    // F

  // the weight in steps of 2^-F; 0 where it is below the floor
  __device__ __forceinline__ uint64_t of(float x) const {
    double w;
    if (x == top)
      w = 1.0;
    else if (top == __builtin_inff() || !(x > -__builtin_inff()))
      w = 0.0;
    else
      w = exp2(((double)x - (double)top) * per);
    return w >= floor ? (uint64_t)rint(ldexp(w, digits)) : 0;
  }
};

__device__ __forceinline__ uint64_t wave_inclusive_sum(uint64_t x) {
  const auto step = [&](uint32_t lo, uint32_t hi) { x += (uint64_t)hi << 32 | lo; };
#define LDA_STEP(CONTROL, ROWS) \
  step(moved<CONTROL, ROWS>(0, (uint32_t)x), moved<CONTROL, ROWS>(0, (uint32_t)(x >> 32)))
  LDA_STEP(0x111, 0xF);
  LDA_STEP(0x112, 0xF);
  LDA_STEP(0x114, 0xF);
  LDA_STEP(0x118, 0xF);
  LDA_STEP(0x142, 0xA);
  LDA_STEP(0x143, 0xC);
#undef LDA_STEP
  return x;
}

struct Found {
  uint32_t key;     // the first key up to which the amounts reach the target
  uint64_t before;  // the sum of those before it
  uint64_t at;      // the sum of its own
  bool there;       // false: all of them do not reach it
};

struct SampleShared {
  unsigned long long bins[kBins];
  uint64_t sums[kSampleWaves];
  uint64_t before, at;
  uint32_t bin;
  float tops[kSampleWaves];
  uint32_t firsts[kSampleWaves];
};

// The search over the members' keys from lo to hi.  each(lo, hi, add) calls add(key,
// amount) for the members (others than those of lo .. hi are passed over, and it may
// leave them out); target(sum of all) is at least 1.
template <typename Each, typename Target>
__device__ Found search(SampleShared &sh, uint32_t lo, uint32_t hi, Target target_of, Each each) {
  const int t = (int)threadIdx.x, lane = t & 63, wave = t >> 6;
  uint64_t before = 0, target = 0;
  for (bool first = true;; first = false) {
    const uint32_t range = hi - lo;
    const int shift = range < (uint32_t)kBins ? 0 : 32 - __builtin_clz(range) - 11;
    sh.bins[2 * t] = 0;
    sh.bins[2 * t + 1] = 0;
    __syncthreads();
    each(lo, hi, [&](uint32_t key, uint64_t amount) {
      if (key - lo <= range && amount) atomicAdd(&sh.bins[(key - lo) >> shift], (unsigned long long)amount);
    });
    __syncthreads();
    const uint64_t one = sh.bins[2 * t], two = sh.bins[2 * t + 1];
    uint64_t upto = wave_inclusive_sum(one + two);
    if (lane == 63) sh.sums[wave] = upto;
    __syncthreads();
    uint64_t all = 0;
#pragma unroll
    for (int i = 0; i < kSampleWaves; ++i) {
      if (i == wave) upto += all;
      all += sh.sums[i];
    }
    if (first) {
      target = target_of(all);
      if (all < target) {
        __syncthreads();  // `sums` is read
        return Found{0, all, 0, false};
      }
    }
    upto += before;
    const uint64_t mid = upto - two, start = mid - one;
    if (start < target && target <= upto) {
      const bool second = mid < target;
      sh.bin = (uint32_t)(2 * t + (second ? 1 : 0));
      sh.before = second ? mid : start;
      sh.at = second ? two : one;
    }
    __syncthreads();
    before = sh.before;
    lo += sh.bin << shift;
    if (shift == 0) return Found{lo, before, sh.at, true};
    hi = hi - lo < (1u << shift) ? hi : lo + (1u << shift) - 1;
  }
}

template <typename T>
__global__ __launch_bounds__(kSampleThreads) void sample_kernel(
    const typename T::store *logits, int64_t ld, int64_t B, int32_t V, int digits,
    const float *u, const float *temperature, const int32_t *top_k, const float *top_p,
    const float *min_p, int32_t *z, float *prob) {
  __shared__ SampleShared sh;
  const int t = (int)threadIdx.x, lane = t & 63, wave = t >> 6;
  const uint32_t chunks = ((uint32_t)V + 7) / 8;
  const float none = -__builtin_inff();
  for (int64_t row = blockIdx.x; row < B; row += gridDim.x) {
    const typename T::store *x = logits + row * ld;
    // f(number, logit) of the tokens from chunk `from` to `to`
    const auto tokens = [&](uint32_t from, uint32_t to, auto f) {
      for (uint32_t c = from + t; c <= to; c += kSampleThreads) {
        const int n = (uint32_t)V - 8 * c < 8 ? (int)((uint32_t)V - 8 * c) : 8;
        float v[8];
        load_elements<T, 8>(x + 8 * (int64_t)c, n, v);
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (j < n) f(8 * c + j, v[j]);
      }
    };
    float top = none;
    tokens(0, chunks - 1, [&](uint32_t, float v) { top = fmaxf(top, v); });
    top = wave_max(top);
    if (lane == 0) sh.tops[wave] = top;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kSampleWaves; ++i) top = fmaxf(top, sh.tops[i]);
    const float heat = temperature ? temperature[row] : 1.0f;
    if (top == none || !(heat > 0.0f)) {  // nothing to draw, or the largest
      uint32_t first = 0xFFFFFFFFu;
      tokens(0, chunks - 1, [&](uint32_t i, float v) {
        if (v == top && i < first) first = i;
      });
      first = wave_min(first);
      if (lane == 0) sh.firsts[wave] = first;
      __syncthreads();
      if (t == 0) {
        for (int i = 1; i < kSampleWaves; ++i) first = sh.firsts[i] < first ? sh.firsts[i] : first;
        z[row] = top == none ? -1 : (int32_t)first;
        prob[row] = top == none ? 0.0f : 1.0f;
      }
      __syncthreads();
      continue;
    }
    Weights weights{top, 1.4426950408889634 / (double)heat, 0.0, digits};
    // the tokens that stay: up to key `last`, of that one those up to number `tie`
    const uint32_t first_key = key_of<T>(top), last_key = key_of<T>(-3.4028234663852886e38f) + 1;
    uint32_t last = last_key, tie = 0xFFFFFFFFu;
    const auto stays = [&](uint32_t key, uint32_t i) { return key < last || (key == last && i <= tie); };
    const auto everyone = [&](uint32_t, uint32_t, auto add, auto amount) {
      tokens(0, chunks - 1, [&](uint32_t i, float v) {
        if (v > none) {
          const uint32_t key = key_of<T>(v);
          if (stays(key, i)) add(key, amount(v));
        }
      });
    };
    // cuts after `many` of the tokens of key `at`, of which there are `all`
    const auto cut = [&](uint32_t at, uint64_t many, uint64_t all) {
      const uint32_t before = at == last ? tie : 0xFFFFFFFFu;
      last = at;
      tie = before;
      if (many >= all) return;
      const Found f = search(sh, 0, (uint32_t)V - 1, [&](uint64_t) { return many; },
                             [&](uint32_t lo, uint32_t hi, auto add) {
                               tokens(lo / 8, hi / 8, [&](uint32_t i, float v) {
                                 if (v > none && key_of<T>(v) == at && i <= before) add(i, 1);
                               });
                             });
      tie = f.key;
    };
    const int32_t k = top_k ? top_k[row] : 0;
    if (k > 0 && k < V) {
      const Found f = search(sh, first_key, last_key, [&](uint64_t) { return (uint64_t)k; },
                             [&](uint32_t lo, uint32_t hi, auto add) {
                               everyone(lo, hi, add, [](float) { return (uint64_t)1; });
                             });
      if (f.there) cut(f.key, (uint64_t)k - f.before, f.at);
    }
    const float p = top_p ? top_p[row] : 1.0f;
    if (p < 1.0f) {
      uint64_t target = 1;
      const Found f = search(sh, first_key, last_key,
                             [&](uint64_t all) {
                               const double share = ceil((double)all * (double)p);
                               target = share < 1.0 ? 1 : share < (double)all ? (uint64_t)share : all;
                               return target;
                             },
                             [&](uint32_t lo, uint32_t hi, auto add) {
                               everyone(lo, hi, add, [&](float v) { return weights.of(v); });
                             });
      const uint64_t each = weights.of(logit_of<T>(f.key));
      const uint64_t many = (target - f.before + each - 1) / each;
      // (ties up to an earlier cut's number, where it was made at this key)
      cut(f.key, many, f.at / each);
    }
    const float floor_at = min_p ? min_p[row] : 0.0f;
    weights.floor = floor_at > 0.0f ? fmin((double)floor_at, 1.0) : 0.0;
    uint64_t total = 0;
    const Found f = search(sh, 0, (uint32_t)V - 1,
                           [&](uint64_t all) {
                             total = all;
                             const double at = floor((double)u[row] * (double)all);
                             const uint64_t below = at > 0.0 ? at < (double)all ? (uint64_t)at : all : 0;
                             return below < all ? below + 1 : all;
                           },
                           [&](uint32_t lo, uint32_t hi, auto add) {
                             tokens(lo / 8, hi / 8, [&](uint32_t i, float v) {
                               if (v > none && stays(key_of<T>(v), i)) add(i, weights.of(v));
                             });
                           });
    if (t == 0) {
      z[row] = (int32_t)f.key;
      prob[row] = (float)((double)f.at / (double)total);
    }
    __syncthreads();
  }
}

}  // namespace lda
