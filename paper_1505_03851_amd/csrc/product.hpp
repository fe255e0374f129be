// Products of 8-bit rows with 8-bit weights:
//
//   out[m][n] = (sum over k of q[m][k] w[n][k]) scale[m] weight_scale[n] + bias[n]
//
// The sums are whole numbers in 32 bits, exact (K is at most 131,071); they become
// float once, take the two scales and the bias there, and are rounded to the output's
// type.  Both operands have k contiguous, as v_mfma_i32_16x16x64_i8 takes them: lane l
// holds 16 bytes of row l % 16 from k = 16 (l / 16) on.  The weights are its first
// operand, so that a lane's four sums are those of four channels next to each other:
// row l % 16 of q, channels 4 (l / 16) + 0 .. 3.
//
// direct_product_kernel: a tile of 16 rows and 16 channels to a workgroup, whose wavefronts
// share the length of K and read what they multiply straight into registers; their sums
// meet in LDS (whole numbers: in any order the same).  For up to 16 rows, and for lines too
// short or too far apart for the other.
//
// tiled_product_kernel: larger tiles, through LDS.
#pragma once

#include "elements.hpp"

namespace lda {

typedef int32_t ints4 __attribute__((ext_vector_type(4)));
typedef ints4 ints4_any __attribute__((aligned(1), may_alias));

template <int N>
struct Count {
  static constexpr int value = N;
};

constexpr int kStep = 64;  // bytes of K that one matrix instruction takes

template <typename T>
struct ProductArgs {
  const int8_t *q, *w;
  const float *scale, *weight_scale, *bias;
  typename T::store *out;
  int64_t ldq, ldw, ldo, M;
  int32_t N, K;
};

// What a sum becomes: the second product and the bias (0: none) rounded together, by name, so
// that a row is the same alone and among others, whichever kernel takes it.
__device__ __forceinline__ float scaled(float sum, float scale, float weight_scale, float bias) {
  return __builtin_fmaf(sum * scale, weight_scale, bias);
}

// The 16 bytes of a line of K >= 16 from byte `at` on, zero from its end on, in two steps:
// where the line ends among them those that end with it are loaded, and moved down later.
// So loads have no branch that others would wait in.
__device__ __forceinline__ ints4 load_piece(const int8_t *line, int at, int K) {
  const int from = at <= K - 16 ? at : at < K ? K - 16 : 0;
  return *reinterpret_cast<const ints4_any *>(line + from);
}

__device__ __forceinline__ ints4 own_piece(const ints4 &v, int at, int K) {
  const int down = at <= K - 16 ? 0 : at < K ? 8 * (16 - (K - at)) : 128;  // bits
  uint64_t low = (uint64_t)(uint32_t)v[1] << 32 | (uint32_t)v[0];
  uint64_t high = (uint64_t)(uint32_t)v[3] << 32 | (uint32_t)v[2];
  low = down >= 64 ? high : low;
  high = down >= 64 ? 0 : high;
  const int rest = down & 63;
  low = rest ? low >> rest | high << (64 - rest) : low;
  high >>= rest;
  low = down == 128 ? 0 : low;
  return ints4{(int)low, (int)(low >> 32), (int)high, (int)(high >> 32)};
}

// The same of a line of any length.
__device__ __forceinline__ ints4 piece_of_any(const int8_t *line, int at, int K) {
  if (K >= 16) return own_piece(load_piece(line, at, K), at, K);
  ints4 v = {0, 0, 0, 0};
#pragma unroll
  for (int j = 0; j < 16; ++j)
    if (at + j < K) v[j / 4] |= (int)((uint32_t)(uint8_t)line[at + j] << (8 * (j % 4)));
  return v;
}

// The wavefronts of a workgroup share the length of K.
template <typename T>
__global__ __launch_bounds__(256) void direct_product_kernel(ProductArgs<T> a, uint32_t col_tiles,
                                                             int64_t tiles) {
  constexpr int kTile = 16, kPitch = kTile + 4;
  __shared__ int32_t joined[kTile * kPitch];
  const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int waves = (int)blockDim.x >> 6;
  const int line = lane & 15, part = lane >> 4;
  // this wavefront's share of K, in steps; the last may be a piece of one
  const int steps = (a.K + kStep - 1) / kStep;
  const int from = (int)((int64_t)steps * wave / waves), to = (int)((int64_t)steps * (wave + 1) / waves);
  const int whole = to * kStep <= a.K ? to : to - 1;
  for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
    const int64_t row_tile = tile / col_tiles;
    const int64_t m0 = row_tile * kTile, n0 = (tile - row_tile * col_tiles) * kTile;
    for (int i = (int)threadIdx.x; i < kTile * kPitch; i += (int)blockDim.x) joined[i] = 0;
    const int64_t m_in = m0 + line < a.M ? m0 + line : a.M - 1;
    const int64_t n_in = n0 + line < a.N ? n0 + line : a.N - 1;
    const int8_t *q_line = a.q + m_in * a.ldq, *w_line = a.w + n_in * a.ldw;
    const int8_t *q = q_line + 16 * part, *w = w_line + 16 * part;
    ints4 sum = {0, 0, 0, 0};
    // (loads first: a matrix instruction keeps the compiler from unrolling a loop)
    const auto steps_at = [&](auto count, int s) {
      constexpr int kCount = decltype(count)::value;
      ints4 x[kCount], y[kCount];
#pragma unroll
      for (int i = 0; i < kCount; ++i) {
        y[i] = *reinterpret_cast<const ints4_any *>(w + (s + i) * kStep);
        x[i] = *reinterpret_cast<const ints4_any *>(q + (s + i) * kStep);
      }
#pragma unroll
      for (int i = 0; i < kCount; ++i)
        sum = __builtin_amdgcn_mfma_i32_16x16x64_i8(y[i], x[i], sum, 0, 0, 0);
    };
    int s = from;
    for (; s + 8 <= whole; s += 8) steps_at(Count<8>(), s);
    if (s + 4 <= whole) steps_at(Count<4>(), s), s += 4;
    if (s + 2 <= whole) steps_at(Count<2>(), s), s += 2;
    if (s < whole) steps_at(Count<1>(), s);
    if (from < to && whole < to) {
      const int at = whole * kStep + 16 * part;
      sum = __builtin_amdgcn_mfma_i32_16x16x64_i8(piece_of_any(w_line, at, a.K),
                                                  piece_of_any(q_line, at, a.K), sum, 0, 0, 0);
    }
    __syncthreads();  // cleared
    if (from < to) {
#pragma unroll
      for (int r = 0; r < 4; ++r) atomicAdd(&joined[line * kPitch + 4 * part + r], sum[r]);
    }
    __syncthreads();
    for (int i = (int)threadIdx.x; i < kTile * kTile; i += (int)blockDim.x) {
      const int64_t m = m0 + i / kTile, n = n0 + i % kTile;
      if (m >= a.M || n >= a.N) continue;
      const float sum_mn = (float)joined[i / kTile * kPitch + i % kTile];
      a.out[m * a.ldo + n] =
          T::down(scaled(sum_mn, a.scale[m], a.weight_scale[n], a.bias ? a.bias[n] : 0.0f));
    }
    __syncthreads();  // read before the next tile clears it
  }
}

// ---- tiles through LDS
//
// A workgroup takes BM rows by BN channels: WM x WN wavefronts with (BM / WM) x
// (BN / WN) of them each, GROUPS times over, the groups sharing the length of K.  It
// passes by in stages of 128 bytes for each group, each line of which goes from memory to
// LDS without passing registers while the one before it is multiplied.  A line's 16-byte
// pieces lie in LDS in the order piece ^ (line % 8): a matrix operand's
// 16 lines would otherwise be in the same banks.  Lines past the last are the last one
// again (their sums are not stored); pieces past K are piece 0 again, and the rows'
// operand is cleared there.  ANY: lines that do not start at 16 bytes, or K that is no
// multiple of 16, pass through registers.
//
// Workgroups start at different stages: lines often lie a power of two apart, so that the
// same stage of all of them is in a few of the memory's channels (64 x 100,000 x 4,096 110 us
// where all start at the first, 92 here, 256 x 8,192 36 against 21).  Tiles of 128 and more, which
// share lines through their XCD's L2, start alike within an XCD (8,192 x 8,192 x 4,096 on the
// same operands again and again 236 us; each elsewhere 256, all alike 238).
//
// A workgroup takes tile after tile, the next one's first stage on its way while this
// one's sums go out: by rows through LDS, whole lines of memory at a time.

constexpr int kStage = 128;

typedef __attribute__((address_space(3))) void *lds_pointer;
typedef const __attribute__((address_space(1))) void *global_pointer;

// Waits for what this wavefront asked of memory and of LDS, then for the other wavefronts.
__device__ __forceinline__ void arrive() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(7 << 4);  // vmcnt(0), lgkmcnt(0)
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

template <typename T, int BM, int BN, int WM, int WN, int GROUPS, bool ANY>
__global__ __launch_bounds__(64 * WM * WN * GROUPS) void tiled_product_kernel(ProductArgs<T> a,
                                                                               uint32_t row_tiles,
                                                                               uint32_t tiles) {
  using S = typename T::store;
  constexpr int kWaves = WM * WN * GROUPS, kRows = BM / WM, kCols = BN / WN;
  constexpr int MT = kRows / 16, NT = kCols / 16;
  // a wavefront's loads a stage, 8 lines each
  constexpr int kQ = BM * GROUPS / 8 / kWaves, kW = BN * GROUPS / 8 / kWaves;
  constexpr int kBytes = (BM + BN) * GROUPS * kStage;  // of a stage
  constexpr int kFirstW = BM * GROUPS;                 // lines of a stage before the weights'
  static_assert(kQ * 8 * kWaves == BM * GROUPS && kW * 8 * kWaves == BN * GROUPS, "whole loads");
  static_assert(GROUPS == 1 || (GROUPS - 1) * BM * BN * 4 <= kBytes, "room for the groups' sums");
  // one array to a stage: the compiler then knows that a stage is not written while
  // another one is read
  __shared__ __attribute__((aligned(16))) int8_t stage0[kBytes], stage1[kBytes];
  const int lane = (int)threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int group = wave / (WM * WN), place = wave % (WM * WN);
  const int line = lane & 15, part = lane >> 4;
  const int first_q = place / WN * kRows, first_w = place % WN * kCols;
  const int piece = ((lane & 7) ^ (lane >> 3)) * 16;
  const int stages = (a.K + kStage * GROUPS - 1) / (kStage * GROUPS);
  const int turn = (int)((blockIdx.x % 8 * 4 + (BM >= 128 ? 0 : blockIdx.x / 8)) % (uint32_t)stages);
  const auto turned = [&](int s) { return s + turn < stages ? s + turn : s + turn - stages; };

  int64_t m0, n0;
  uint32_t q_at[kQ], w_at[kW];
  const auto take = [&](uint32_t tile) {
    m0 = (int64_t)(tile % row_tiles) * BM;
    n0 = (int64_t)(tile / row_tiles) * BN;
#pragma unroll
    for (int i = 0; i < kQ; ++i) {
      const int64_t r = (wave * kQ + i) * 8 % BM + (lane >> 3), most = a.M - 1 - m0;
      q_at[i] = (uint32_t)((r < most ? r : most) * a.ldq);
    }
#pragma unroll
    for (int i = 0; i < kW; ++i) {
      const int64_t r = (wave * kW + i) * 8 % BN + (lane >> 3), most = a.N - 1 - n0;
      w_at[i] = (uint32_t)((r < most ? r : most) * a.ldw);
    }
  };
  // f(number, line in memory, line of the stage, byte of the line) of this lane's loads
  const auto each_load = [&](int stage, auto f) {
    const int8_t *q = a.q + m0 * a.ldq, *w = a.w + n0 * a.ldw;
#pragma unroll
    for (int i = 0; i < kQ; ++i) {
      const int at = (stage * GROUPS + (wave * kQ + i) * 8 / BM) * kStage + piece;
      f(i, q + q_at[i], (wave * kQ + i) * 8, at);
    }
#pragma unroll
    for (int i = 0; i < kW; ++i) {
      const int at = (stage * GROUPS + (wave * kW + i) * 8 / BN) * kStage + piece;
      f(kQ + i, w + w_at[i], kFirstW + (wave * kW + i) * 8, at);
    }
  };
  const auto bring = [&](int s, int8_t *to) {
    each_load(turned(s), [&](int, const int8_t *from, int first, int at) {
      __builtin_amdgcn_global_load_lds((global_pointer)(from + (at < a.K ? at : 0)),
                                       (lds_pointer)(to + first * kStage), 16, 0, 0);
    });
  };
  ints4 held[ANY ? kQ + kW : 1];  // a stage on its way through registers
  const auto fetch = [&](int s) {
    each_load(turned(s), [&](int i, const int8_t *from, int, int at) {
      held[i] = load_piece(from, at, a.K);
    });
  };
  const auto keep = [&](int s, int8_t *to) {
    const int stage = turned(s);
    if ((stage + 1) * GROUPS * kStage > a.K)
      each_load(stage, [&](int i, const int8_t *, int, int at) { held[i] = own_piece(held[i], at, a.K); });
    each_load(stage, [&](int i, const int8_t *, int first, int) {
      *reinterpret_cast<ints4 *>(to + first * kStage + lane * 16) = held[i];
    });
  };
  ints4 sum[MT][NT];
  const auto multiply = [&](int s, const int8_t *from) {
    const int k0 = (turned(s) * GROUPS + group) * kStage;
    const bool tail = k0 + kStage > a.K;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const int8_t *at = from + ((4 * half + part) ^ (line & 7)) * 16 + line * kStage;
      ints4 x[MT], y[NT];
#pragma unroll
      for (int j = 0; j < NT; ++j)
        y[j] = *reinterpret_cast<const ints4 *>(at + (kFirstW + group * BN + first_w + 16 * j) * kStage);
#pragma unroll
      for (int i = 0; i < MT; ++i)
        x[i] = *reinterpret_cast<const ints4 *>(at + (group * BM + first_q + 16 * i) * kStage);
      if (tail && k0 + (4 * half + part) * 16 >= a.K) {
#pragma unroll
        for (int i = 0; i < MT; ++i) x[i] = ints4{0, 0, 0, 0};
      }
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j)
          sum[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(y[j], x[i], sum[i][j], 0, 0, 0);
    }
  };
  // stage s, in `here`; the next one goes to `there`, which was read last (through registers
  // no further ahead either: with the stage after it on its way too 4,000 x 4,001 x 4,001
  // took a fifth longer)
  const auto step = [&](int s, const int8_t *here, int8_t *there) {
    const bool more = s + 1 < stages;
    arrive();
    if constexpr (ANY) {
      if (more) fetch(s + 1);
      multiply(s, here);
      if (more) keep(s + 1, there);
    } else {
      if (more) bring(s + 1, there);
      multiply(s, here);
    }
  };
  const auto first_stage = [&](int8_t *to) {
    if constexpr (ANY) {
      fetch(0);
      keep(0, to);
    } else {
      bring(0, to);
    }
  };

  uint32_t tile = blockIdx.x;
  take(tile);
  first_stage(stage0);
  while (true) {
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < NT; ++j) sum[i][j] = ints4{0, 0, 0, 0};
    for (int s = 0; s < stages; s += 2) {
      step(s, stage0, stage1);
      if (s + 1 < stages) step(s + 1, stage1, stage0);
    }
    arrive();  // everyone has read the last stage
    if constexpr (GROUPS > 1) {  // the first group adds the others' sums to its own
      ints4 *room = reinterpret_cast<ints4 *>(stage1) + (size_t)place * MT * NT * 64 + lane;
      constexpr int kGroup = BM * BN / 4;
      if (group > 0) {
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
          for (int j = 0; j < NT; ++j) room[(group - 1) * kGroup + (i * NT + j) * 64] = sum[i][j];
      }
      arrive();
      if (group == 0) {
#pragma unroll
        for (int g = 0; g < GROUPS - 1; ++g)
#pragma unroll
          for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < NT; ++j) sum[i][j] += room[g * kGroup + (i * NT + j) * 64];
      }
      arrive();  // read, before rows go out through the same memory
    }
    const int64_t m_out = m0 + first_q, n_out = n0 + first_w;
    tile += gridDim.x;
    const bool more = tile < tiles;
    if (more) {
      take(tile);
      first_stage(stage0);
    }
    // The sums leave through this wavefront's share of the second stage's memory, as
    // many rows at a time as fit.
    constexpr int kPitch = kCols * (int)sizeof(S) + 16;
    constexpr int kShare = kBytes / (WM * WN) / 16 * 16;
    constexpr int kRoom = kShare / kPitch / 16 * 16;
    constexpr int kPass = kRoom < kRows ? kRoom : kRows;
    static_assert(kPass >= 16, "room for 16 rows");
    constexpr int kLaneCols = 16 / (int)sizeof(S), kLanes = kCols / kLaneCols;  // of a row
    int8_t *room = stage1 + place * kShare;
    float ws[NT][4], b[NT][4];
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      const int64_t n = n_out + 16 * j + 4 * part;
      const int left = a.N - n < 0 ? 0 : a.N - n < 4 ? (int)(a.N - n) : 4;
      load_elements<F32, 4>(a.weight_scale + (left ? n : 0), left, ws[j]);
      load_elements<F32, 4>(a.bias + (a.bias && left ? n : 0), a.bias ? left : 0, b[j]);
    }
#pragma unroll
    for (int r0 = 0; r0 < kRows && group == 0; r0 += kPass) {
#pragma unroll
      for (int i = r0 / 16; i < (r0 + kPass < kRows ? r0 + kPass : kRows) / 16; ++i) {
        const int64_t m = m_out + 16 * i + line;
        const float s = a.scale[m < a.M ? m : a.M - 1];
#pragma unroll
        for (int j = 0; j < NT; ++j) {
          Packed<T, 4> v;
#pragma unroll
          for (int r = 0; r < 4; ++r)
            v.v[r] = T::down(scaled((float)sum[i][j][r], s, ws[j][r], b[j][r]));
          *reinterpret_cast<Packed<T, 4> *>(room + (16 * i - r0 + line) * kPitch +
                                            (16 * j + 4 * part) * (int)sizeof(S)) = v;
        }
      }
      __builtin_amdgcn_wave_barrier();
      // (LDS works in order within a wavefront)
#pragma unroll
      for (int i = 0; i < kPass; i += 64 / kLanes) {
        const int r = i + lane / kLanes, c = lane % kLanes * kLaneCols;
        const int64_t m = m_out + r0 + r, n = n_out + c;
        if (r0 + r >= kRows || r >= kPass || m >= a.M || n >= a.N) continue;
        const auto *from = reinterpret_cast<const Packed<T, kLaneCols> *>(
            room + r * kPitch + c * (int)sizeof(S));
        S *to = a.out + m * a.ldo + n;
        if (a.N - n >= kLaneCols) {
          *reinterpret_cast<words4_any *>(to) = __builtin_bit_cast(words4, *from);
        } else {
          for (int e = 0; e < (int)(a.N - n); ++e) to[e] = from->v[e];
        }
      }
      __builtin_amdgcn_wave_barrier();
    }
    if (!more) break;
  }
}

}  // namespace lda
