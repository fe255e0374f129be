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
// One workgroup of 1,024 lanes takes a row, which stays in registers (up to 131,072
// logits of 16 bits, 65,536 floats; longer ones are read again from the caches).
//   * Few stay (top_k up to 512, or up to 1,024 tokens in all): the k-th largest of the
//     lanes' largest logits is a bound below which none of the first k lies.  What is above
//     it, k and a few, goes to a list in LDS.  Up to 256 of them each find the number and
//     the weight of those before them by comparing with all; more are searched as rows are.
//   * Otherwise each question (the k-th token, the token that reaches a share, a tie's
//     number) is a search: in an interval of keys (a logit's order, or a token's number)
//     that holds the answer, members add their amounts (1, or their weight) to 2,048 bins in
//     LDS; the bin where the running sum reaches the target is the next interval, until it
//     is one key.  A token with less than (1 - top_p) / V of all weight cannot be the one
//     that reaches top_p: only those above add theirs.
//   * z is found by the wavefronts' sums (each holds a stretch of the row), then one
//     wavefront's chunks, lanes and elements.
#pragma once

#include "elements.hpp"
#include "wave_ops.hpp"

namespace lda {

constexpr int kSampleThreads = 1024;
constexpr int kSampleWaves = kSampleThreads / 64;
constexpr int kBins = 2 * kSampleThreads;
constexpr int kListed = kSampleThreads;  // tokens of a list, one to a lane
constexpr int kCompared = 256;           // of those that are compared with each other
constexpr int kFewest = 512;             // the largest top_k that is looked for by a bound

// Logits as keys that rise as they fall, from the bits of a float, bfloat16 or half (0 for
// -0).  Positive NaN have keys below +inf's, negative ones above -inf's.
template <typename T>
struct Keys {
  using S = typename T::store;
  using S_bits = typename Raw<sizeof(S)>::type;
  static constexpr uint32_t kSign = sizeof(S) == 4 ? 0x80000000u : 0x8000u;
  static constexpr uint32_t kRest = kSign - 1;

  static __device__ __forceinline__ uint32_t of(uint32_t bits) {
    return bits & kSign ? bits : bits ^ kRest;
  }
  static __device__ __forceinline__ float logit(uint32_t key) {
    return T::up(__builtin_bit_cast(S, (S_bits)(key & kSign ? key : key ^ kRest)));
  }
  static __device__ __forceinline__ uint32_t bits(float x) {
    return (uint32_t)__builtin_bit_cast(S_bits, T::down(x));
  }
  static __device__ __forceinline__ uint32_t infinity() { return bits(__builtin_inff()) ^ kRest; }
  static __device__ __forceinline__ uint32_t none() { return bits(-__builtin_inff()); }
};

// a b + c with c in scalar registers: left to itself the compiler keeps the polynomial's
// coefficients in twenty vector registers, which the row needs.
__device__ __forceinline__ double fma_by(double a, double b, double c) {
  double d;
  asm("v_fma_f64 %0, %1, %2, %3" : "=v"(d) : "v"(a), "v"(b), "s"(c));
  return d;
}

// A row's weights, in steps of 2^-F.
struct Weights {
  double top;    // the largest logit
  double per;    // log2(e) / temperature
  double floor;  // min_p in steps
  double least;  // of the exponent: what is below has no weight
  int digits;    // F

  // 2^y of y = n + f, |f| <= 1/2, as a polynomial in f that interpolates (2^f - 1) / f at ten
  // Chebyshev points: off by 2^-50.6 of itself at most.
  __device__ __forceinline__ uint64_t of(float x) const {
    const double y = fmax(((double)x - top) * per, least);  // (NaN: least)
    const double n = rint(y), f = y - n;
    double p = fma_by(7.070977866508138e-09, f, 1.0205905413765595e-07);
    p = fma_by(p, f, 1.3215451633221434e-06);
    p = fma_by(p, f, 1.5252672924850737e-05);
    p = fma_by(p, f, 0.00015403530424776529);
    p = fma_by(p, f, 0.0013333558200794592);
    p = fma_by(p, f, 0.009618129107618665);
    p = fma_by(p, f, 0.05550410866465167);
    p = fma_by(p, f, 0.24022650695910075);
    p = fma_by(p, f, 0.6931471805599462);
    p = fma(p, f, 1.0);
    // times 2^(n + F), in the exponent's bits
    const uint64_t bits = __builtin_bit_cast(uint64_t, p);
    const uint32_t high = (uint32_t)(bits >> 32) + ((uint32_t)((int)n + digits) << 20);
    const double w = __builtin_bit_cast(double, (uint64_t)high << 32 | (uint32_t)bits);
    // rounded to a whole number by the last place of 2^52
    const uint64_t whole = __builtin_bit_cast(uint64_t, w + 0x1p52) & 0xFFFFFFFFFFFFFull;
    return w >= floor ? whole : 0;
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

__device__ __forceinline__ uint64_t from_lane(uint64_t x, int lane) {
  return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(x >> 32), lane) << 32 |
         (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)x, lane);
}

// What all lanes know alike, in scalar registers.
__device__ __forceinline__ uint32_t uniform(uint32_t x) {
  return (uint32_t)__builtin_amdgcn_readfirstlane((int)x);
}
__device__ __forceinline__ uint64_t uniform(uint64_t x) {
  return (uint64_t)uniform((uint32_t)(x >> 32)) << 32 | uniform((uint32_t)x);
}
__device__ __forceinline__ double uniform(double x) {
  return __builtin_bit_cast(double, uniform(__builtin_bit_cast(uint64_t, x)));
}

struct Found {
  uint32_t key;     // the first key up to which the amounts reach the target
  uint64_t before;  // the sum of those before it
  uint64_t at;      // the sum of its own
  bool there;       // false: all of them do not reach it
};

struct SampleShared {
  union {
    unsigned long long bins[kBins];
    struct {
      uint64_t place[kListed], weight[kListed];  // key << 32 | number
    } list;
  };
  unsigned long long before[kCompared], mass[kCompared];
  uint32_t rank[kCompared];
  uint64_t sums[kSampleWaves];
  uint32_t tops[kSampleWaves];
  uint64_t pick_before, pick_at;
  uint32_t bin, listed;
  unsigned long long total;
};

// The search over the members' keys from lo to hi.  each(add) calls add(key, amount) for
// the members (others than those of lo .. hi are passed over, their amount not asked for).  target is at least 1.
// `levels` 1: the interval of the answer that one level gives, its last key.
template <typename Each>
__device__ Found search(SampleShared &sh, uint32_t lo, uint32_t hi, uint64_t target, int levels,
                        Each each) {
  const int t = (int)threadIdx.x, lane = t & 63, wave = (int)uniform((uint32_t)t >> 6);
  uint64_t before = 0;
  for (bool first = true;; first = false) {
    const uint32_t range = hi - lo;
    const int shift = range < (uint32_t)kBins ? 0 : 32 - __builtin_clz(range) - 11;
    sh.bins[2 * t] = 0;
    sh.bins[2 * t + 1] = 0;
    __syncthreads();
    each([&](uint32_t key, auto amount) {
      if (key - lo <= range) {
        const uint64_t a = amount();
        if (a) atomicAdd(&sh.bins[(key - lo) >> shift], (unsigned long long)a);
      }
    });
    __syncthreads();
    const uint64_t one = sh.bins[2 * t], two = sh.bins[2 * t + 1];
    uint64_t upto = wave_inclusive_sum(one + two);
    if (lane == 63) sh.sums[wave] = upto;
    __syncthreads();
    uint64_t all = before;
#pragma unroll
    for (int i = 0; i < kSampleWaves; ++i) {
      if (i == wave) upto += all;
      all += uniform(sh.sums[i]);
    }
    if (first && all < target) {
      __syncthreads();  // `sums` is read
      return Found{0, all, 0, false};
    }
    const uint64_t mid = upto - two, start = mid - one;
    if (start < target && target <= upto) {
      const bool second = mid < target;
      sh.bin = (uint32_t)(2 * t + (second ? 1 : 0));
      sh.pick_before = second ? mid : start;
      sh.pick_at = second ? two : one;
    }
    __syncthreads();
    before = uniform((uint64_t)sh.pick_before);
    lo += uniform(sh.bin) << shift;
    hi = shift == 0 ? lo : hi - lo < (1u << shift) ? hi : lo + (1u << shift) - 1;
    if (shift == 0 || --levels == 0) return Found{hi, before, uniform((uint64_t)sh.pick_at), true};
  }
}

// A row of V logits.  A wavefront holds `each` chunks of 64 times 8 of them, one stretch
// of the row: chunk i of lane l starts at token (((wave each + i) 64) + l) 8.  CHUNKS: those
// that stay in registers, of which a loop's turn takes one by its (scalar) number; 0: all
// are read from memory every time.
template <typename T, int CHUNKS>
struct SampleRow {
  using S = typename T::store;
  static constexpr int kWords = 2 * (int)sizeof(S);  // of a chunk
  typedef uint32_t held __attribute__((ext_vector_type(CHUNKS ? CHUNKS : 2)));
  typedef uint32_t chunk __attribute__((ext_vector_type(kWords)));

  const S *x;
  int32_t V;
  int each;
  held words[kWords];

  __device__ __forceinline__ uint32_t first(int i) const {
    return ((uniform(threadIdx.x >> 6) * (uint32_t)each + (uint32_t)i) * 64 + (threadIdx.x & 63)) * 8;
  }
  // as in memory, with 0 for -0 and -inf past the end
  __device__ __forceinline__ chunk read(int i) const {
    const uint32_t at = first(i);
    const int n = i >= each || at >= (uint32_t)V ? 0 : (uint32_t)V - at < 8 ? (int)((uint32_t)V - at) : 8;
    Packed<T, 8> p = load_packed<T, 8>(x + (n ? at : 0), n);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      uint32_t b = __builtin_bit_cast(typename Raw<sizeof(S)>::type, p.v[j]);
      b = b == Keys<T>::kSign ? 0 : b;
      b = j < n ? b : Keys<T>::none();
      p.v[j] = __builtin_bit_cast(S, (typename Raw<sizeof(S)>::type)b);
    }
    return __builtin_bit_cast(chunk, p);
  }
  __device__ __forceinline__ void load() {
    if constexpr (CHUNKS > 0) {
#pragma unroll
      for (int i = 0; i < CHUNKS; ++i) {
        const chunk c = read(i);
#pragma unroll
        for (int w = 0; w < kWords; ++w) words[w][i] = c[w];
      }
    }
  }
  // f(number, key) of this lane's chunk i
  template <typename F>
  __device__ __forceinline__ void visit(int i, F f) const {
    chunk c;
    if constexpr (CHUNKS > 0) {
#pragma unroll
      for (int w = 0; w < kWords; ++w) c[w] = words[w][i];
    } else {
      c = read(i);
    }
    const uint32_t at = first(i);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      f(at + j, Keys<T>::of(sizeof(S) == 4 ? c[j % kWords] : c[j / 2] >> (16 * (j & 1)) & 0xFFFFu));
      if (j & 1) __builtin_amdgcn_sched_barrier(0);  // (two weights' registers at a time)
    }
  }
  // f(number, key) of all of this lane's
  template <typename F>
  __device__ __forceinline__ void all(F f) const {
#pragma unroll 1
    for (int i = 0; i < each; ++i) visit(i, f);
  }
};

// The tokens that stay by their order: keys from `first` to before `last`, and of `last`
// the numbers below `end`.
struct Stay {
  uint32_t first, last, end;
  __device__ __forceinline__ bool before(uint32_t key) const { return key - first < last - first; }
  __device__ __forceinline__ bool operator()(uint32_t key, uint32_t i) const {
    return before(key) || (key == last && i < end);
  }
};

// The weight that a share of `all` asks for, at least 1.
__device__ __forceinline__ uint64_t share_of(uint64_t all, float p) {
  const double share = ceil((double)all * (double)p);
  return share < 1.0 ? 1 : share < (double)all ? (uint64_t)share : all;
}

// The sum that a token's is the first to pass.
__device__ __forceinline__ uint64_t point_of(uint64_t all, float u) {
  const double at = floor((double)u * (double)all);
  const uint64_t below = at > 0.0 ? at < (double)all ? (uint64_t)at : all : 0;
  return below < all ? below : all - 1;
}

struct SampleSettings {
  uint64_t k;  // 0: none
  float p, u;
  double floor;  // in steps
};

// The choice among the n tokens of the list, each compared with all others.
template <typename T>
__device__ void choose_compared(SampleShared &sh, int n, Weights weights, const SampleSettings &s,
                                int32_t *z, float *prob) {
  const int t = (int)threadIdx.x;
  const int width = n <= 64 ? 64 : n <= 128 ? 128 : 256;  // (wavefronts see one `part` each)
  const int i = t & (width - 1), part = __builtin_amdgcn_readfirstlane(t / width);
  const int parts = kSampleThreads / width;
  if (t < kCompared) {
    sh.before[t] = sh.mass[t] = 0;
    sh.rank[t] = 0;
  }
  if (t == 0) sh.total = 0;
  uint64_t weight = 0;
  const uint64_t mine = i < n ? sh.list.place[i] : ~0ull;
  if (part == 0 && i < n) {
    weight = weights.of(Keys<T>::logit((uint32_t)(mine >> 32)));
    sh.list.weight[i] = weight;
  }
  __syncthreads();
  uint32_t rank = 0;
  uint64_t mass = 0;
  for (int j = part; j < n; j += parts)
    if (sh.list.place[j] < mine) {
      ++rank;
      mass += sh.list.weight[j];
    }
  if (i < n && rank) {
    atomicAdd(&sh.rank[i], rank);
    atomicAdd(&sh.mass[i], (unsigned long long)mass);
  }
  __syncthreads();
  const bool in = part == 0 && i < n && (s.k == 0 || sh.rank[i] < s.k);
  if (part == 0) {
    const uint64_t sum = wave_inclusive_sum(in ? weight : 0);
    if ((t & 63) == 63) atomicAdd(&sh.total, (unsigned long long)sum);
  }
  __syncthreads();
  if (part == 0) {
    const bool stays = in && (!(s.p < 1.0f) || sh.mass[i] < share_of(sh.total, s.p)) &&
                       (double)weight >= s.floor;
    weight = stays ? weight : 0;
    if (i < n) sh.list.weight[i] = weight;
  }
  __syncthreads();
  // by number: the sums before each
  const uint32_t number = (uint32_t)mine;
  uint64_t before = 0, all = 0;
  for (int j = part; j < n; j += parts) {
    const uint64_t w = sh.list.weight[j];
    all += w;
    if ((uint32_t)sh.list.place[j] < number) before += w;
  }
  if (t == 0) sh.total = 0;
  if (i < n && before) atomicAdd(&sh.before[i], (unsigned long long)before);
  __syncthreads();
  if (i == 0) atomicAdd(&sh.total, (unsigned long long)all);
  __syncthreads();
  if (part == 0 && weight) {
    const uint64_t point = point_of(sh.total, s.u) - sh.before[i];  // (wraps where it is before)
    if (point < weight) {
      *z = (int32_t)number;
      *prob = (float)((double)weight / (double)sh.total);
    }
  }
}

template <typename T, int CHUNKS>
__global__ __launch_bounds__(kSampleThreads) void sample_kernel(
    const typename T::store *logits, int64_t ld, int64_t B, int32_t V, int digits,
    const float *u, const float *temperature, const int32_t *top_k, const float *top_p,
    const float *min_p, int32_t *z, float *prob) {
  __shared__ SampleShared sh;
  const int t = (int)threadIdx.x, lane = t & 63, wave = (int)uniform((uint32_t)t >> 6);
  SampleRow<T, CHUNKS> row;
  row.V = V;
  row.each = (int)(((uint32_t)V + 8 * kSampleThreads - 1) / (8 * kSampleThreads));
  const uint32_t infinity = Keys<T>::infinity(), none = Keys<T>::none();
  for (int64_t b = blockIdx.x; b < B; b += gridDim.x) {
    row.x = logits + b * ld;
    const float heat = temperature ? temperature[b] : 1.0f;
    const int32_t k = top_k ? top_k[b] : 0;
    const float share = top_p ? top_p[b] : 1.0f, low = min_p ? min_p[b] : 0.0f;
    SampleSettings s{k > 0 && k < V ? (uint64_t)k : 0, share, u[b],
                     uniform(low > 0.0f ? ldexp(fmin((double)low, 1.0), digits) : 0.0)};
    row.load();
    uint32_t best = none;  // of this lane
    row.all([&](uint32_t, uint32_t key) {
      if (key - infinity < best - infinity) best = key;
    });
    const uint32_t wave_best = wave_min(best);
    if (lane == 0) sh.tops[wave] = wave_best;
    if (t == 0) sh.listed = 0;
    __syncthreads();
    uint32_t top = uniform(sh.tops[0]);
#pragma unroll
    for (int i = 1; i < kSampleWaves; ++i) {
      const uint32_t other = uniform(sh.tops[i]);
      top = other < top ? other : top;
    }
    if (top == none || !(heat > 0.0f)) {  // nothing to draw, or the largest
      uint32_t first = 0xFFFFFFFFu;
      row.all([&](uint32_t i, uint32_t key) {
        if (key == top && i < first) first = i;
      });
      first = wave_min(first);
      __syncthreads();  // `tops` is read
      if (lane == 0) sh.tops[wave] = first;
      __syncthreads();
      if (t == 0) {
        for (int i = 1; i < kSampleWaves; ++i) first = sh.tops[i] < first ? sh.tops[i] : first;
        z[b] = top == none ? -1 : (int32_t)first;
        prob[b] = top == none ? 0.0f : 1.0f;
      }
      __syncthreads();
      continue;
    }
    // Where logits are infinite only those stay, with the weight 1 each (y is NaN, so `least`).
    const bool endless = top == infinity;
    Weights weights{uniform((double)Keys<T>::logit(top)),
                    uniform(endless ? 0.0 : 1.4426950408889634 / (double)heat), 0.0,
                    endless ? 0.0 : -(double)(digits + 2), digits};
    const auto weight_of = [&](uint32_t key) { return weights.of(Keys<T>::logit(key)); };
    const uint32_t lowest = endless ? top : none - 1;
    Stay stay{top, lowest + 1, 0};

    // ---- few: a list
    const bool all_listed = V <= kListed;
    if (all_listed || (s.k && s.k <= kFewest)) {
      uint32_t bound = lowest;
      if (!all_listed) {
        const Found f = search(sh, top, lowest, s.k, 1, [&](auto add) { add(best, [] { return (uint64_t)1; }); });
        // (not there: fewer lanes than k hold any)
        if (f.there) bound = f.key;
      }
      __syncthreads();  // bins and list share their memory
      row.all([&](uint32_t i, uint32_t key) {
        if (key - top <= bound - top) {
          const uint32_t at = atomicAdd(&sh.listed, 1);
          if (at < (uint32_t)kListed) sh.list.place[at] = (uint64_t)key << 32 | i;
        }
      });
      __syncthreads();
      const int n = (int)uniform(sh.listed);
      if (n <= kCompared) {
        choose_compared<T>(sh, n, weights, s, z + b, prob + b);
        __syncthreads();
        continue;
      }
    }

    const auto everyone = [&](auto add, auto amount) {
      row.all([&](uint32_t i, uint32_t key) {
        if (stay(key, i)) add(key, [&] { return amount(key); });
      });
    };
    // cuts after `many` of the tokens of key `at`, of which there are `all`
    const auto cut = [&](uint32_t at, uint64_t many, uint64_t all) {
      const uint32_t end = at == stay.last ? stay.end : 0xFFFFFFFFu;
      stay.last = at;
      stay.end = end;
      if (many >= all) return;
      const Found f = search(sh, 0, (uint32_t)V - 1, many, 32, [&](auto add) {
        row.all([&](uint32_t i, uint32_t key) {
          if (key == at && i < end) add(i, [] { return (uint64_t)1; });
        });
      });
      stay.end = f.key + 1;
    };
    if (s.k) {
      const Found f = search(sh, top, lowest, s.k, 32, [&](auto add) {
        everyone(add, [](uint32_t) { return (uint64_t)1; });
      });
      if (f.there) cut(f.key, s.k - f.before, f.at);
    }
    const auto row_total = [&](uint64_t mine) {  // the wavefronts' sums stay in `sums`
      const uint64_t sum = wave_inclusive_sum(mine);
      __syncthreads();  // `sums` is read
      if (lane == 63) sh.sums[wave] = sum;
      __syncthreads();
      uint64_t all = 0;
#pragma unroll
      for (int i = 0; i < kSampleWaves; ++i) all += uniform((uint64_t)sh.sums[i]);
      return all;
    };
    if (s.p < 1.0f) {
      uint64_t mine = 0;
      row.all([&](uint32_t i, uint32_t key) {
        if (stay(key, i)) mine += weight_of(key);
      });
      const uint64_t all = row_total(mine);
      const uint64_t target = uniform(share_of(all, s.p));
      // Tokens with less than (1 - p) / V of all weight hold less than 1 - p together, so
      // p is reached before them: what is below half of that is not asked for its weight.
      uint32_t bound = lowest;
      if (!endless) {
        const double part = (1.0 - fmax((double)s.p, 0.0)) * 0.5 / V * (double)all / (double)(1ull << digits);
        const float reach = (float)(weights.top + (double)heat * log(part));
        const uint32_t key = uniform(Keys<T>::of(Keys<T>::bits(reach)) + 2);  // (roundings upwards)
        bound = key - top < lowest - top ? key : lowest;
      }
      __syncthreads();
      const Found f = search(sh, top, bound, target, 32, [&](auto add) { everyone(add, weight_of); });
      const uint64_t each = uniform(weight_of(f.key));
      cut(f.key, (target - f.before + each - 1) / each, f.at / each);
    }
    weights.floor = s.floor;
    uint64_t mine = 0;
    row.all([&](uint32_t i, uint32_t key) {
      if (stay(key, i)) mine += weight_of(key);
    });
    const uint64_t total = row_total(mine);
    uint64_t point = uniform(point_of(total, s.u));
    // the wavefront whose stretch holds it, its chunk, lane and element
    int holder = 0;
    for (; holder < kSampleWaves - 1 && point >= uniform((uint64_t)sh.sums[holder]); ++holder)
      point -= uniform((uint64_t)sh.sums[holder]);
    if (wave == holder) {
      for (int i = 0; i < row.each; ++i) {
        uint64_t sum = 0;
        row.visit(i, [&](uint32_t at, uint32_t key) { sum += stay(key, at) ? weight_of(key) : 0; });
        const uint64_t upto = wave_inclusive_sum(sum), all = from_lane(upto, 63);
        if (point >= all) {
          point -= all;
          continue;
        }
        uint64_t rest = point - (upto - sum);  // (wraps where it lies before this lane)
        if (rest < sum)
          row.visit(i, [&](uint32_t at, uint32_t key) {
            const uint64_t w = stay(key, at) ? weight_of(key) : 0;
            if (rest < w) {  // (never again: past it, rest wraps)
              z[b] = (int32_t)at;
              prob[b] = (float)((double)w / (double)total);
            }
            rest -= w;
          });
        break;
      }
    }
    __syncthreads();
  }
}

}  // namespace lda
