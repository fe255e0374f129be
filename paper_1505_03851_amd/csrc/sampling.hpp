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
//     it, k and a few, goes to a list, one to a lane, which is sorted by logit, cut, sorted
//     by number and searched.
//   * Otherwise a cut is found in two steps: all add their amounts (1 for top_k, their
//     weight for top_p) to 1,024 bins in LDS, evenly spaced in x over the logits that have a
//     weight; those of the bin where the running sum reaches its target go to a list, which
//     is compared or sorted.  Where they are more than 1,024 (equal logits, most often) bins
//     narrow down on the logit's bits instead, then on the tokens' numbers.  min_p is
//     applied with top_p's cut, by its own bin; up to 1,024 tokens that top_k leaves go
//     to a list at once.
//   * Each wavefront holds a stretch of the row and has bins of its own, so the sums of the
//     stretches' weights that stay are there after the last cut.  z is found by them, then by
//     the stretch's chunks, one to a wavefront, lanes and elements.
#pragma once

#include "elements.hpp"
#include "wave_ops.hpp"

namespace lda {

constexpr int kSampleThreads = 1024;
constexpr int kSampleWaves = kSampleThreads / 64;
constexpr int kBins = 2 * kSampleThreads;
constexpr int kSpaced = kSampleThreads;  // bins of a wavefront
constexpr int kQueue = 1024;             // logits on a wavefront's way to their weights
constexpr int kListed = kSampleThreads;  // tokens of a list, one to a lane
constexpr int kCompared = 256;           // of those that are compared with each other
constexpr int kFewest = 512;             // the largest top_k that is looked for by a bound

// Logits as keys that rise as they fall, from the bits of a float, bfloat16 or half.
template <typename T>
struct Keys {
  using S = typename T::store;
  using S_bits = typename Raw<sizeof(S)>::type;
  static constexpr uint32_t kSign = sizeof(S) == 4 ? 0x80000000u : 0x8000u;
  static constexpr uint32_t kRest = kSign - 1;

  static __device__ __forceinline__ uint32_t of(float x) {  // (-0 as 0)
    const uint32_t bits = (uint32_t)__builtin_bit_cast(S_bits, T::down(x + 0.0f));
    return bits & kSign ? bits : bits ^ kRest;
  }
  static __device__ __forceinline__ float logit(uint32_t key) {
    return T::up(__builtin_bit_cast(S, (S_bits)(key & kSign ? key : key ^ kRest)));
  }
};

// What all lanes know alike, in scalar registers.
__device__ __forceinline__ uint32_t uniform(uint32_t x) {
  return (uint32_t)__builtin_amdgcn_readfirstlane((int)x);
}
__device__ __forceinline__ uint64_t uniform(uint64_t x) {
  return (uint64_t)uniform((uint32_t)(x >> 32)) << 32 | uniform((uint32_t)x);
}
__device__ __forceinline__ float uniform(float x) {
  return __builtin_bit_cast(float, uniform(__builtin_bit_cast(uint32_t, x)));
}
__device__ __forceinline__ double uniform(double x) {
  return __builtin_bit_cast(double, uniform(__builtin_bit_cast(uint64_t, x)));
}

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
  double shift;  // 1.5 2^52 + F: what rounds y to whole numbers, F added
  float least;   // logits up to this have no weight

  // 2^(F + y) of y = n + f, |f| <= 1/2, as a polynomial in f that interpolates (2^f - 1) / f at
  // ten Chebyshev points (off by 2^-50.6 of itself at most), its exponent raised by n + F.
  // Where not `there` (which x must be above `least` for) a number that rounds to 0.
  __device__ __forceinline__ double of(float x, bool there) const {
    // (y's product fused by name: a token has the same weight, to the last bit, wherever this is
    // inlined, or sums of bins and of rows would not be the same)
    const double d = (double)x - top, m = fma(d, per, shift), f = fma(d, per, -(m - shift));
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
    words2 bits = __builtin_bit_cast(words2, p);
    bits[1] += __builtin_bit_cast(words2, m)[0] << 20;
    bits[1] = there ? bits[1] : 0;
    return __builtin_bit_cast(double, bits);
  }
  // the same as a whole number, by the last place of 2^52
  static __device__ __forceinline__ double rounded(double w) { return (w + 0x1p52) - 0x1p52; }
  static __device__ __forceinline__ uint64_t steps(double w) {
    return __builtin_bit_cast(uint64_t, w + 0x1p52) & 0xFFFFFFFFFFFFFull;
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

struct SampleShared {
  union {
    unsigned long long bins[kBins];
    struct {
      uint64_t place[kListed], weight[kListed];  // place: key << 32 | number
    } list;
    float queue[kSampleWaves][kQueue];
    unsigned long long spaced[kSampleWaves][kSpaced];
  };
  uint64_t sums[2][kSampleWaves];
  unsigned long long kept[kSampleWaves];
  uint32_t tops[kSampleWaves];
  uint64_t pick_before, pick_at;
  uint32_t bin, listed;
  unsigned long long mass[kCompared], before[kCompared], total;
  uint32_t rank[kCompared], worst[kSampleWaves];
};

// The sum of the lanes' x up to this one, and of all; the wavefronts' sums stay in
// sh.sums[turn].
__device__ __forceinline__ uint64_t block_inclusive_sum(SampleShared &sh, int turn, uint64_t x,
                                                        uint64_t *total) {
  const int lane = (int)threadIdx.x & 63, wave = (int)uniform(threadIdx.x >> 6);
  uint64_t upto = wave_inclusive_sum(x), all = 0;
  if (lane == 63) sh.sums[turn][wave] = upto;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kSampleWaves; ++i) {
    if (i == wave) upto += all;
    all += uniform(sh.sums[turn][i]);
  }
  *total = all;
  return upto;
}

struct Found {
  uint32_t key;     // the answer; of bins that were not narrowed down, its bin
  uint64_t before;  // the sum of the amounts before it
  uint64_t at;      // the sum of its own
  bool there;       // false: all of them do not reach the target
};

// Where the running sum over the lanes' two bins, from `before` on, reaches target(sum of
// all).
template <typename Target>
__device__ Found reached(SampleShared &sh, uint64_t before, uint64_t one, uint64_t two,
                         Target target_of) {
  const int t = (int)threadIdx.x;
  uint64_t all;
  const uint64_t upto = before + block_inclusive_sum(sh, 0, one + two, &all);
  const uint64_t target = target_of(before + all);
  if (before + all < target) {
    __syncthreads();  // `sums` is read
    return Found{0, before + all, 0, false};
  }
  const uint64_t mid = upto - two, start = mid - one;
  if (start < target && target <= upto) {
    const bool second = mid < target;
    sh.bin = (uint32_t)(2 * t + (second ? 1 : 0));
    sh.pick_before = second ? mid : start;
    sh.pick_at = second ? two : one;
  }
  __syncthreads();
  return Found{uniform(sh.bin), uniform((uint64_t)sh.pick_before), uniform((uint64_t)sh.pick_at), true};
}

__device__ __forceinline__ void clear_bins(SampleShared &sh) {
  sh.bins[2 * threadIdx.x] = 0;
  sh.bins[2 * threadIdx.x + 1] = 0;
  __syncthreads();
}

// The search over the members' keys from lo to hi for the first up to which the amounts
// reach target(sum of all), which is at least 1.  each(add) calls add(key, amount) for the
// members (others than those of lo .. hi are passed over, their amount not asked for).
// Where `levels` come to their end first: the last key of the interval that holds it.
template <typename Target, typename Each>
__device__ Found search(SampleShared &sh, uint32_t lo, uint32_t hi, int levels, Target target_of,
                        Each each) {
  uint64_t before = 0, target = 0;
  for (bool first = true;; first = false) {
    const uint32_t range = hi - lo;
    const int shift = range < (uint32_t)kBins ? 0 : 32 - __builtin_clz(range) - 11;
    clear_bins(sh);
    each([&](uint32_t key, auto amount) {
      if (key - lo <= range) {
        const uint64_t a = amount();
        if (a) atomicAdd(&sh.bins[(key - lo) >> shift], (unsigned long long)a);
      }
    });
    __syncthreads();
    const Found f = reached(sh, before, sh.bins[2 * threadIdx.x], sh.bins[2 * threadIdx.x + 1], [&](uint64_t all) {
      if (first) target = uniform(target_of(all));
      return target;
    });
    if (!f.there) return f;
    before = f.before;
    lo += f.key << shift;
    hi = shift == 0 ? lo : hi - lo < (1u << shift) ? hi : lo + (1u << shift) - 1;
    if (shift == 0 || --levels == 0) return Found{hi, before, f.at, true};
  }
}

// The value of lane `lane ^ apart`, apart < 64: within 16 lanes by data-parallel moves.
template <int CONTROL>
__device__ __forceinline__ uint64_t moved_pair(uint64_t v) {
  return (uint64_t)moved<CONTROL, 0xF>(0, (uint32_t)(v >> 32)) << 32 | moved<CONTROL, 0xF>(0, (uint32_t)v);
}
__device__ __forceinline__ uint64_t across(uint64_t v, int apart) {
  switch (apart) {
    case 1: return moved_pair<0xB1>(v);                     // of four lanes 1 0 3 2
    case 2: return moved_pair<0x4E>(v);                     // 2 3 0 1
    case 4: return moved_pair<0x1B>(moved_pair<0x141>(v));  // of eight 7 .. 0, of four 3 .. 0
    case 8: return moved_pair<0x128>(v);                    // of sixteen turned by eight
    default:
      return (uint64_t)(uint32_t)__shfl_xor((int)(v >> 32), apart) << 32 |
             (uint32_t)__shfl_xor((int)(uint32_t)v, apart);
  }
}

// Sorts the lanes' values, of which those of lanes from WIDTH on are not looked at: lane t
// then holds the t-th.  A bitonic network: exchanges within wavefronts by lane, others
// through `room`.
template <int WIDTH>
__device__ __forceinline__ uint64_t sorted(uint64_t v, uint64_t *room) {
  const int t = (int)threadIdx.x;
  const bool idle = uniform((uint32_t)t & ~63u) >= (uint32_t)WIDTH;
#pragma unroll
  for (int size = 2; size <= WIDTH; size *= 2)
#pragma unroll
    for (int apart = size / 2; apart > 0; apart /= 2) {
      uint64_t other = v;
      if (apart >= 64) {
        __syncthreads();
        room[t] = v;
        __syncthreads();
        other = room[t ^ apart];
      } else if (!idle) {
        other = across(v, apart);
      }
      // (the lane's number made new, so that a hundred such conditions are not kept in
      // registers from row to row)
      int lane = t;
      asm volatile("" : "+v"(lane));
      const bool smaller = ((lane & apart) == 0) == ((lane & size) == 0 || size == WIDTH);
      v = smaller == (other < v) ? other : v;
    }
  return v;
}

__device__ __forceinline__ uint64_t sorted(uint64_t v, int n, uint64_t *room) {
  static_assert(kListed == 1024, "the widths");
  return n <= 512 ? sorted<512>(v, room) : sorted<1024>(v, room);
}

// A row of V logits.  A wavefront holds `each` chunks of 64 times 8 of them, one stretch
// of the row: chunk i of lane l starts at token (((wave each + i) 64) + l) 8.  CHUNKS: those
// that stay in registers, of which a loop's turn takes one by its (scalar) number; 0: all
// are read from memory every time.
template <typename T, int CHUNKS>
struct SampleRow {
  using S = typename T::store;
  static constexpr int kWords = 2 * (int)sizeof(S);  // of a chunk
  // sixteen registers that a scalar numbers: word w of chunk i is register i kPart + w % kPart
  // of vector w / kPart
  static constexpr int kPart = CHUNKS ? 16 / CHUNKS : 1;
  typedef uint32_t held __attribute__((ext_vector_type(16)));
  typedef uint32_t chunk __attribute__((ext_vector_type(kWords)));

  const S *x;
  int32_t V;
  int each;
  held words[CHUNKS ? kWords / kPart : 1];

  __device__ __forceinline__ uint32_t first(int wave, int i) const {
    return (((uint32_t)wave * (uint32_t)each + (uint32_t)i) * 64 + (threadIdx.x & 63)) * 8;
  }
  // NaN past the end: never chosen
  __device__ __forceinline__ chunk read(int wave, int i) const {
    const uint32_t at = first(wave, i);
    const int n = i >= each || at >= (uint32_t)V ? 0 : (uint32_t)V - at < 8 ? (int)((uint32_t)V - at) : 8;
    Packed<T, 8> p = load_packed<T, 8>(x + (n ? at : 0), n);
    if (n < 8) {
#pragma unroll
      for (int j = 0; j < 8; ++j) p.v[j] = j < n ? p.v[j] : T::down(__builtin_nanf(""));
    }
    return __builtin_bit_cast(chunk, p);
  }
  static __device__ __forceinline__ float element(const chunk &c, int j) {
    if constexpr (sizeof(S) == 4)
      return __builtin_bit_cast(float, (uint32_t)c[j]);
    else
      return T::up((S)(c[j / 2] >> (16 * (j & 1))));
  }
  __device__ __forceinline__ void load() {
    if constexpr (CHUNKS > 0) {
      const int wave = (int)uniform(threadIdx.x >> 6);
#pragma unroll
      for (int i = 0; i < CHUNKS; ++i) {
        const chunk c = read(wave, i);
#pragma unroll
        for (int w = 0; w < kWords; ++w) words[w / kPart][i * kPart + w % kPart] = c[w];
      }
    }
  }
  // f(number of its first, chunk) of this lane's chunks
  template <typename F>
  __device__ __forceinline__ void chunks(F f) const {
    const int wave = (int)uniform(threadIdx.x >> 6);
#pragma unroll 1
    for (int i = 0; i < each; ++i) {
      chunk c;
      if constexpr (CHUNKS > 0) {
#pragma unroll
        for (int w = 0; w < kWords; ++w) c[w] = words[w / kPart][i * kPart + w % kPart];
      } else {
        c = read(wave, i);
      }
      f(first(wave, i), c);
    }
  }
  // f(number of a chunk's first, place in the chunk, logit) of all of this lane's
  template <typename F>
  __device__ __forceinline__ void all(F f) const {
    chunks([&](uint32_t at, const chunk &c) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        f(at, j, element(c, j));
        if (j & 1) __builtin_amdgcn_sched_barrier(0);  // (two weights' registers at a time)
      }
    });
  }
};

// The tokens that stay by their order: logits above `last`, and of those at it the
// numbers below `end` (2^31 - 1 at most).
struct Stay {
  float last, above;
  uint32_t end;
  __device__ __forceinline__ Stay(float l, uint32_t e)
      : last(l), above(uniform(nextafterf(l, __builtin_inff()))), end(e) {}
  __device__ __forceinline__ bool operator()(float x, uint32_t at, int j) const {
    return x >= (j < (int32_t)(end - at) ? last : above);
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
  double floor;  // min_p in steps: of weights as they are, before they are rounded to whole ones
};

// Of up to 256 listed tokens: each compared with all others.  The lanes of a list's width
// (wavefronts of `part` 0) get their token's place, its amount (amount(logit)), its rank and
// the amounts of those before it; sh.list.weight holds the amounts.  A lane compares its token
// with those from `begin` to `end`: one after the other, so that a read of LDS brings two.
struct Compared {
  int i, part, begin, end;
  uint64_t place, amount, before;
  uint32_t rank;
};

template <typename T, typename Amount>
__device__ __forceinline__ Compared compared(SampleShared &sh, int n, Amount amount) {
  const int t = (int)threadIdx.x;
  const int width = n <= 64 ? 64 : n <= 128 ? 128 : 256;  // (a wavefront's lanes share a `part`)
  const int part = (int)uniform((uint32_t)t / (uint32_t)width);
  const int share = (int)(((uint32_t)n * (uint32_t)width + kSampleThreads - 1) / kSampleThreads);
  const int begin = part * share, end = begin + share < n ? begin + share : n;
  Compared c{t & (width - 1), part, begin, end, 0, 0, 0, 0};
  if (t < kCompared) {
    sh.mass[t] = sh.before[t] = 0;
    sh.rank[t] = 0;
  }
  if (t == 0) sh.total = 0;
  c.place = c.i < n ? sh.list.place[c.i] : ~0ull;
  if (c.part == 0) {
    c.amount = c.i < n ? amount(Keys<T>::logit((uint32_t)(c.place >> 32))) : 0;
    sh.list.weight[c.i] = c.amount;
  }
  __syncthreads();
  uint32_t rank = 0;
  uint64_t mass = 0;
#pragma unroll 8
  for (int j = c.begin; j < c.end; ++j) {
    const uint64_t other = sh.list.weight[j];
    const bool earlier = sh.list.place[j] < c.place;
    rank += earlier ? 1 : 0;
    mass += earlier ? other : 0;
  }
  if (c.i < n && rank) {
    atomicAdd(&sh.rank[c.i], rank);
    atomicAdd(&sh.mass[c.i], (unsigned long long)mass);
  }
  __syncthreads();
  c.rank = sh.rank[c.i];
  c.before = sh.mass[c.i];
  return c;
}

// The choice among the n tokens of the list, up to 256: first by their order, then by number.
template <typename T>
__device__ void choose_compared(SampleShared &sh, int n, const Weights &weights,
                                const SampleSettings &s, int32_t *z, float *prob) {
  const int t = (int)threadIdx.x;
  bool heavy = false;  // at least min_p, which is asked of a weight before it is rounded
  const Compared c = compared<T>(sh, n, [&](float x) {
    const double w = weights.of(x, x > weights.least);
    heavy = w >= s.floor;
    return Weights::steps(w);
  });
  uint64_t weight = c.amount;
  if (c.part == 0) {
    weight = s.k == 0 || c.rank < s.k ? weight : 0;
    const uint64_t sum = wave_inclusive_sum(weight);
    if ((t & 63) == 63) atomicAdd(&sh.total, (unsigned long long)sum);
  }
  __syncthreads();
  if (c.part == 0) {
    const bool stays = !(s.p < 1.0f) || c.before < share_of(sh.total, s.p);
    weight = stays && heavy ? weight : 0;
    sh.list.weight[c.i] = weight;
  }
  __syncthreads();
  const uint32_t number = (uint32_t)c.place;
  uint64_t before = 0, all = 0;
#pragma unroll 8
  for (int j = c.begin; j < c.end; ++j) {
    const uint64_t other = sh.list.weight[j];
    all += other;
    before += (uint32_t)sh.list.place[j] < number ? other : 0;
  }
  if (t == 0) sh.total = 0;
  if (c.i < n && before) atomicAdd(&sh.before[c.i], (unsigned long long)before);
  __syncthreads();
  if (c.i == 0) atomicAdd(&sh.total, (unsigned long long)all);
  __syncthreads();
  if (c.part == 0 && weight) {
    const uint64_t point = point_of(sh.total, s.u) - sh.before[c.i];  // (wraps where it lies before)
    if (point < weight) {
      *z = (int32_t)number;
      *prob = (float)((double)weight / (double)sh.total);
    }
  }
}

// The choice among the n tokens of the list, sorted.  `whole`: the list is the row, so that
// its tokens' numbers are places too.
template <typename T>
__device__ void choose_sorted(SampleShared &sh, int n, bool whole, const Weights &weights,
                              const SampleSettings &s, int32_t *z, float *prob) {
  const int t = (int)threadIdx.x;
  const bool cuts = s.k || s.p < 1.0f;
  uint64_t place = t < n ? sh.list.place[t] : ~0ull;
  if (cuts || !whole) place = sorted(place, n, sh.list.weight);
  const bool there = place != ~0ull;
  const float x = Keys<T>::logit((uint32_t)(place >> 32));
  const double w = weights.of(x, there && x > weights.least);
  uint64_t weight = s.k == 0 || (uint64_t)t < s.k ? Weights::steps(w) : 0, all = 0;
  if (cuts) {
    const uint64_t upto = block_inclusive_sum(sh, 0, weight, &all);
    weight = !(s.p < 1.0f) || upto - weight < share_of(all, s.p) ? weight : 0;
  }
  weight = w >= s.floor ? weight : 0;
  // by number
  uint32_t number = (uint32_t)place;
  __syncthreads();  // what was there is read
  if (whole && cuts) {
    sh.list.weight[t] = 0;
    __syncthreads();
    if (there) sh.list.weight[number] = weight;
    __syncthreads();
    weight = sh.list.weight[t];
    number = (uint32_t)t;
  } else if (!whole) {
    // what does not stay has no part in it
    sh.list.place[t] = weight;
    const uint64_t by =
        sorted((uint64_t)(weight ? number : 0xFFFFFFFFu) << 32 | (uint32_t)t, n, sh.list.weight);
    __syncthreads();
    weight = t < n ? sh.list.place[(uint32_t)by] : 0;
    number = (uint32_t)(by >> 32);
  }
  const uint64_t sum = block_inclusive_sum(sh, 1, weight, &all);
  const uint64_t point = point_of(all, s.u);
  if (sum - weight <= point && point < sum) {
    *z = (int32_t)number;
    *prob = (float)((double)weight / (double)all);
  }
}

template <typename T, int CHUNKS>
__global__ __launch_bounds__(kSampleThreads) void sample_kernel(
    const typename T::store *logits, int64_t ld, int32_t V, int digits,
    const float *u, const float *temperature, const int32_t *top_k, const float *top_p,
    const float *min_p, int32_t *z, float *prob) {
  __shared__ SampleShared sh;
  const int t = (int)threadIdx.x, lane = t & 63, wave = (int)uniform((uint32_t)t >> 6);
  const float infinity = __builtin_inff();
  const auto one = [] { return (uint64_t)1; };
  SampleRow<T, CHUNKS> row;
  row.V = V;
  row.each = (int)(((uint32_t)V + 8 * kSampleThreads - 1) / (8 * kSampleThreads));
  const uint32_t b = blockIdx.x;
  row.x = logits + b * ld;
  const float heat = temperature ? temperature[b] : 1.0f;
  const int32_t k = top_k ? top_k[b] : 0;
  const float low = min_p ? min_p[b] : 0.0f;
  SampleSettings s{k > 0 && k < V ? (uint64_t)k : 0, top_p ? top_p[b] : 1.0f, u[b],
                   uniform(low > 0.0f ? ldexp(fmin((double)low, 1.0), digits) : 0.0)};
  row.load();
  float best = -infinity;  // of this lane
  row.all([&](uint32_t, int, float x) { best = fmaxf(best, x); });
  const uint32_t best_key = Keys<T>::of(best);
  const uint32_t wave_best = wave_min(best_key), wave_worst = ~wave_min(~best_key);
  if (lane == 0) {
    sh.tops[wave] = wave_best;
    sh.worst[wave] = wave_worst;
  }
  if (t == 0) sh.listed = 0;
  __syncthreads();
  uint32_t top_key = uniform(sh.tops[0]);
#pragma unroll
  for (int i = 1; i < kSampleWaves; ++i) {
    const uint32_t other = uniform(sh.tops[i]);
    top_key = other < top_key ? other : top_key;
  }
  const float top = uniform(Keys<T>::logit(top_key));
  const bool greedy = !(heat > 0.0f);
  if (top == -infinity) {
    if (t == 0) {
      z[b] = -1;
      prob[b] = 0.0f;
    }
    return;
  }
  if (greedy || top == infinity) {
    // The largest, or infinite ones, which all have the same weight and no other has any:
    // the rules leave the first of them by number.
    uint64_t stay = 1, point = 0;
    const Found f = search(
        sh, 0, (uint32_t)V - 1, 32,
        [&](uint64_t all) {
          if (!greedy) {
            stay = s.k && s.k < all ? s.k : all;
            stay = s.p < 1.0f ? share_of(stay, s.p) : stay;
            point = point_of(stay, s.u);
          }
          return point + 1;
        },
        [&](auto add) {
          row.all([&](uint32_t at, int j, float x) {
            if (x == top) add(at + j, one);
          });
        });
    if (t == 0) {
      z[b] = (int32_t)f.key;
      prob[b] = (float)(1.0 / (double)stay);
    }
    return;
  }
  const double per = uniform(1.4426950408889634 / (double)heat);
  // (2^-(F + 2) is nothing; rounded downwards, so that no logit with a weight is left out)
  const double nothing = (double)top - (double)(digits + 2) / per;
  // the largest float that is at most v, and below the top
  const auto below = [&](double v) {
    float x = (float)fmax(v, -3.4028234663852886e38);
    x = (double)x > v ? nextafterf(x, -infinity) : x;
    return uniform(x < top ? x : nextafterf(top, -infinity));
  };
  const float least = below(nothing);
  const Weights weights{uniform((double)top), per, uniform(0x1.8p52 + (double)digits), least};

  const auto list = [&](uint32_t number, float x) {
    const uint32_t n = atomicAdd(&sh.listed, 1);
    if (n < (uint32_t)kListed) sh.list.place[n] = (uint64_t)Keys<T>::of(x) << 32 | number;
  };

  // ---- few: a list
  const bool all_listed = V <= kListed;
  if (all_listed || (s.k && s.k <= kFewest)) {
    float bound = -3.4028234663852886e38f;
    if (!all_listed) {
      uint32_t worst_key = 0;
      for (int i = 0; i < kSampleWaves; ++i) worst_key = sh.worst[i] > worst_key ? sh.worst[i] : worst_key;
      const uint32_t end = Keys<T>::of(-infinity) - 1;
      worst_key = uniform(worst_key < end ? worst_key : end);
      const Found f = search(
          sh, top_key, worst_key, 2, [&](uint64_t) { return s.k; },
          [&](auto add) { add(best_key, one); });
      // (not there: fewer lanes than k hold any)
      if (f.there) bound = uniform(Keys<T>::logit(f.key));
    }
    __syncthreads();  // bins and list share their memory
    if (all_listed) {
      const float x = t < V ? T::up(row.x[t]) : -infinity;
      sh.list.place[t] = x > -infinity ? (uint64_t)Keys<T>::of(x) << 32 | (uint32_t)t : ~0ull;
    } else {
      row.all([&](uint32_t at, int j, float x) {
        if (x >= bound) list(at + j, x);
      });
    }
    __syncthreads();
    const int n = all_listed ? V : (int)uniform(sh.listed);
    if (n <= kListed) {
      if (n <= kCompared)
        choose_compared<T>(sh, n, weights, s, z + b, prob + b);
      else
        choose_sorted<T>(sh, n, all_listed, weights, s, z + b, prob + b);
      return;
    }
  }

  // ---- many: cuts
  Stay stay{weights.least, 0};
  bool known = false;  // sh.kept holds the stretches' sums of what stays
  // The bins reach down to the lowest logit that has a weight.
  float lowest = top;
  if (s.k || s.p < 1.0f) {
    row.all([&](uint32_t, int, float x) { lowest = x > least ? fminf(lowest, x) : lowest; });
    const uint32_t key = ~wave_min(~Keys<T>::of(lowest));
    __syncthreads();  // `tops` is read
    if (lane == 0) sh.tops[wave] = key;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kSampleWaves; ++i) lowest = fminf(lowest, Keys<T>::logit(sh.tops[i]));
    lowest = uniform(lowest);
  }
  // Bins evenly spaced from `from` on, down to `to` (which x is not below), and one of them.
  // Reckoned in double, whose x - top a weight needs too: x - from times the scale, rounded to
  // a whole number by the last place of 2^52, at most (from - to) scale, which rounds to the last.
  struct Spaced {
    double from, scale;
    float high, low;
    int at;
    __device__ __forceinline__ Spaced(double f, double to)
        : from(f), scale(uniform(f > to ? (kSpaced - 1) / (to - f) : 0.0)), high(0), low(0), at(0) {}
    __device__ __forceinline__ int bin(float x) const {
      return (int)__builtin_bit_cast(words2, fma((double)x - from, scale, 0x1.8p52))[0];
    }
    // bin `which`; high and low: its logits, and a hundredth of a bin around them for
    // the roundings (all logits, where the bins have no width)
    __device__ __forceinline__ void choose(int which) {
      const double width = 1.0 / scale;
      at = which;
      high = uniform(scale < 0.0 ? (float)(from + ((double)which - 0.51) * width) : __builtin_inff());
      low = uniform(scale < 0.0 ? (float)(from + ((double)which + 0.51) * width) : -__builtin_inff());
    }
    __device__ __forceinline__ bool wide() const { return !(high - low < __builtin_inff()); }
    __device__ __forceinline__ bool has(float x) const {
      return x <= high && x >= low && bin(x) == at;
    }
  };
  // f(place, logit) of a chunk's logits that are among(place, logit), the lanes' next ones
  // side by side: few, so that a branch for each logit would be taken for one lane.
  const auto each_of = [&](const typename SampleRow<T, CHUNKS>::chunk &c, auto among, auto f) {
    uint32_t places = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) places |= among(j, row.element(c, j)) ? 1u << j : 0;
    for (; places; places &= places - 1) {
      const int j = __builtin_ctz(places);
      float x = row.element(c, 0);
#pragma unroll
      for (int i = 1; i < 8; ++i) x = i == j ? row.element(c, i) : x;
      f(j, x);
    }
  };
  // What min_p cuts off, by logits: up to `bar` all, from `pass` on nothing.  The weight itself
  // decides between: 1e-9 of its logarithm, and two roundings of a logit as large as the top, which
  // are more of the logarithm where logits lie far from 0 and close together.
  float bar = least, pass = least;
  if (s.floor > 0.0) {
    const double at = log2(s.floor) - (double)digits, off = 0x1p-51 * fabs((double)top);
    const double up = (double)top + (at + 1e-9) / per + off;
    bar = below((double)top + (at - 1e-9) / per - off);
    pass = (float)up;
    pass = uniform((double)pass < up ? nextafterf(pass, infinity) : pass);
    pass = pass < top ? pass : top;
  }
  // Cuts after the token, in their order, up to which the amounts reach target(sum of all).
  // `floors`: the amounts are weights, and min_p follows at once, so that the sums of what
  // stays are known without another pass over the row: where its bin comes before the
  // target's, that bin's tokens are the ones it decides on.
  const auto cut = [&](auto target_of, auto amount, bool floors) {
    uint64_t target = 0, before = 0;
    known = false;
    // among the n tokens of the list, `before` before them (n <= kListed)
    const auto of_list = [&](int n, bool whole, bool sums) {
      uint64_t place, amount_at = 0, upto;
      if (n <= kCompared && !whole) {
        const Compared c = compared<T>(sh, n, amount);
        place = c.place;
        if (c.part == 0) amount_at = c.amount;
        upto = before + c.before + amount_at;
      } else {
        place = sorted(t < n ? sh.list.place[t] : ~0ull, n, sh.list.weight);
        if (t < n) amount_at = amount(Keys<T>::logit((uint32_t)(place >> 32)));
        uint64_t all;
        upto = before + block_inclusive_sum(sh, 1, amount_at, &all);
        if (whole) target = uniform(target_of(all));
      }
      if (upto - amount_at < target && target <= upto) sh.pick_at = place;
      __syncthreads();
      const uint64_t end = uniform((uint64_t)sh.pick_at);
      if (amount_at && place <= end &&
          (!floors || weights.of(Keys<T>::logit((uint32_t)(place >> 32)), true) >= s.floor))
        atomicAdd(&sh.kept[(uint32_t)place / (512u * (uint32_t)row.each)],
                  (unsigned long long)amount_at);
      stay = Stay{uniform(Keys<T>::logit((uint32_t)(end >> 32))), (uint32_t)end + 1};
      known = floors && (sums || s.floor == 0.0);
    };
    // What a small top_k leaves is a list as it is (256 x 100,000 with all settings 61 us, 63 by
    // bins here too).
    if (floors && s.k && s.k <= kListed) {
      __syncthreads();  // what was there is read
      if (t == 0) sh.listed = 0;
      if (t < kSampleWaves) sh.kept[t] = 0;
      __syncthreads();
      row.chunks([&](uint32_t at, const typename SampleRow<T, CHUNKS>::chunk &c) {
        each_of(c, [&](int j, float x) { return stay(x, at, j); },
                [&](int j, float x) { list(at + j, x); });
      });
      __syncthreads();
      const int n = (int)uniform(sh.listed);
      if (n <= kListed) {
        of_list(n, true, true);
        return;
      }
    }
    Spaced bins(weights.top, (double)lowest), last = bins;
    // the bin, then, where it holds too many, a bin of the bin
    for (int level = 0; level < 2; ++level) {
      const auto member = [&](uint32_t at, int j, float x) {
        return stay(x, at, j) && (level == 0 || last.has(x));
      };
      __syncthreads();  // what was there is read
      for (int i = t; i < kSampleWaves * kSpaced; i += kSampleThreads) (&sh.spaced[0][0])[i] = 0;
      if (t == 0) sh.listed = 0;
      __syncthreads();
      const auto add = [&](auto in) {
        row.all([&](uint32_t at, int j, float x) {
          if (in(at, j, x)) atomicAdd(&sh.spaced[wave][bins.bin(x)], (unsigned long long)amount(x));
        });
      };
      // (a first cut asks no numbers, and its bins share a weight's steps: the sums of 49,999
      // floats' weights take 16 us against 19)
      if (level == 0 && stay.end == 0)
        add([&](uint32_t, int, float x) { return x >= stay.above; });
      else
        add(member);
      __syncthreads();
      uint64_t mine = 0;  // (`reached` takes two to a lane: bin t is its bin 2 t)
#pragma unroll
      for (int i = 0; i < kSampleWaves; ++i) mine += sh.spaced[i][t];
      const Found f = reached(sh, before, mine, 0, [&](uint64_t all) {
        if (level == 0) target = uniform(target_of(all));
        return target;
      });
      if (!f.there) return;
      int chosen = (int)f.key / 2;
      bool by_floor = false;
      if (floors && level == 0 && bar > least) {
        const int first = bins.bin(fmaxf(pass, lowest)),
                  end = bins.bin(fmaxf(nextafterf(bar, infinity), lowest));
        if (first < chosen) {
          by_floor = floors = first == end;  // (else min_p's border lies over two bins)
          if (by_floor) chosen = first;
        }
      }
      bins.choose(chosen);
      before = f.before;
      // the stretches' sums up to the bin
      uint64_t kept = 0;
#pragma unroll
      for (int i = 0; i < kSpaced; i += 64) {
        const uint64_t sum = sh.spaced[wave][i + lane];
        kept += i + lane < bins.at ? sum : 0;
      }
      kept = wave_inclusive_sum(kept);
      if (lane == 63) sh.kept[wave] = level == 0 ? kept : sh.kept[wave] + kept;
      __syncthreads();  // bins and list share their memory
      // (most chunks have none: what is next to the bin's middle decides, without a branch for
      // each; 49,999 floats 2.5 us against 4)
      const float middle = uniform(bins.wide() ? 0.0f : 0.5f * bins.high + 0.5f * bins.low);
      const float reach =
          uniform(bins.wide() ? infinity : fmaxf(bins.high - middle, middle - bins.low));
      row.chunks([&](uint32_t at, const typename SampleRow<T, CHUNKS>::chunk &c) {
        float nearest = infinity;
#pragma unroll
        for (int j = 0; j < 8; ++j) nearest = fminf(nearest, fabsf(row.element(c, j) - middle));
        if (!(nearest <= reach)) return;
        each_of(c, [&](int, float x) { return fabsf(x - middle) <= reach; }, [&](int j, float x) {
          if (x <= bins.high && x >= bins.low && member(at, j, x) && bins.bin(x) == bins.at)
            list(at + j, x);
        });
      });
      __syncthreads();
      const int n = (int)uniform(sh.listed);
      if (by_floor) {
        stay = Stay{bar, 0};
        known = n <= kListed;
        if (t < n && known) {
          const uint64_t place = sh.list.place[t];
          const double w = weights.of(Keys<T>::logit((uint32_t)(place >> 32)), true);
          if (w >= s.floor)
            atomicAdd(&sh.kept[(uint32_t)place / (512u * (uint32_t)row.each)],
                      (unsigned long long)Weights::steps(w));
        }
        return;
      }
      if (n <= kListed) {
        of_list(n, false, level == 0);
        return;
      }
      last = bins;
      if (last.wide()) break;
      bins = Spaced((double)last.high, (double)fmaxf(last.low, lowest));
    }
    const Found g = search(
        sh, top_key, Keys<T>::of(-infinity) - 1, 32, [&](uint64_t) { return target; },
        [&](auto add) {
          row.all([&](uint32_t at, int j, float x) {
            if (stay(x, at, j)) add(Keys<T>::of(x), [&] { return amount(x); });
          });
        });
    const float at = uniform(Keys<T>::logit(g.key));
    const uint64_t each = uniform(amount(at)), many = (target - g.before + each - 1) / each;
    const uint32_t end = at == stay.last ? stay.end : 0x7FFFFFFFu;
    const Found h = search(
        sh, 0, (uint32_t)V - 1, 32, [&](uint64_t) { return many; },
        [&](auto add) {
          row.all([&](uint32_t first, int j, float x) {
            if (x == at && first + j < end) add(first + j, one);
          });
        });
    stay = Stay{at, h.key + 1};
  };
  if (s.k) cut([&](uint64_t) { return s.k; }, [](float) { return (uint64_t)1; }, false);
  const auto weight_of = [&](float x) { return Weights::steps(weights.of(x, true)); };
  if (s.p < 1.0f) cut([&](uint64_t all) { return share_of(all, s.p); }, weight_of, true);

  // ---- the choice
  // (a lane's weights add up to 2^53 at most, exactly in double)
  const auto staying = [&](float x) {
    const double w = weights.of(x, true);
    return w >= s.floor ? Weights::rounded(w) : 0.0;
  };
  if (!known && bar > stay.last) stay = Stay{bar, 0};
  uint64_t total = 0;
  if (known) {
    __syncthreads();
  } else {
    // Those that stay are often few: a wavefront puts them in a row and takes the weights
    // of 64 at a time (6 us less for 256 x 100,000 with min_p, where this pass is the only one).
    __syncthreads();  // `kept`, and what was where the queue is, are read
    float *queue = sh.queue[wave];
    uint32_t put = 0, taken = 0;
    double mine = 0.0;
    if (!s.k && !(s.p < 1.0f) && s.floor == 0.0) {
      row.all([&](uint32_t at, int j, float x) {
        if (stay(x, at, j)) mine += staying(x);
      });
    } else row.chunks([&](uint32_t at, const typename SampleRow<T, CHUNKS>::chunk &c) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float x = row.element(c, j);
        const bool in = stay(x, at, j);
        const uint64_t lanes = __builtin_amdgcn_ballot_w64(in);
        const uint32_t before = __builtin_amdgcn_mbcnt_hi(
            (uint32_t)(lanes >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)lanes, 0));
        if (in) queue[(put + before) % kQueue] = x;
        put += (uint32_t)__builtin_popcountll(lanes);
      }
      for (; put - taken >= 64; taken += 64) mine += staying(queue[(taken + lane) % kQueue]);
    });
    if ((uint32_t)lane < put - taken) mine += staying(queue[(taken + lane) % kQueue]);
    const uint64_t sum = wave_inclusive_sum((uint64_t)mine);
    if (lane == 63) sh.kept[wave] = sum;
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < kSampleWaves; ++i) total += uniform((uint64_t)sh.kept[i]);
  uint64_t point = uniform(point_of(total, s.u));
  // the wavefront whose stretch holds it
  int holder = 0;
  for (; holder < kSampleWaves - 1; ++holder) {
    const uint64_t sum = uniform((uint64_t)sh.kept[holder]);
    if (point < sum) break;
    point -= sum;
  }
  // its chunks, one to a wavefront at a time, lanes and elements
  for (int first = 0, turn = 0; first < row.each; first += kSampleWaves, turn ^= 1) {
    const typename SampleRow<T, CHUNKS>::chunk c = row.read(holder, first + wave);
    const uint32_t at = row.first(holder, first + wave);
    double sum = 0.0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float x = row.element(c, j);
      if (stay(x, at, j)) sum += staying(x);
      if (j & 1) __builtin_amdgcn_sched_barrier(0);
    }
    uint64_t all;
    const uint64_t own = (uint64_t)sum, upto = block_inclusive_sum(sh, turn, own, &all);
    if (point >= all) {
      point -= all;
      continue;
    }
    const uint64_t owner = __builtin_amdgcn_ballot_w64(upto - own <= point && point < upto);
    if (owner) {  // its wavefront takes the lane's eight side by side
      const int from = __builtin_ctzll(owner);
      const uint64_t gone = upto - own;
      const uint64_t rest =
          point - ((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(gone >> 32), from) << 32 |
                   (uint32_t)__builtin_amdgcn_readlane((int)gone, from));
      const uint32_t v = (uint32_t)__builtin_amdgcn_readlane((int)at, from) + (uint32_t)lane;
      const bool one_of = lane < 8 && v < (uint32_t)V;
      const float x = T::up(row.x[one_of ? v : 0]);
      const uint64_t w = one_of && stay(x, v, 0) ? (uint64_t)staying(x) : 0;
      const uint64_t sum_to = wave_inclusive_sum(w);
      if (sum_to - w <= rest && rest < sum_to) {
        z[b] = (int32_t)v;
        prob[b] = (float)((double)w / (double)total);
      }
    }
    break;
  }
}

}  // namespace lda
