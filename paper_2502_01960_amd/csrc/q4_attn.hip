// Attention over contexts held in 4 bits (gfx950).  Arguments and result: mpic_q4.h; layout of the cache: q4.h.
//
// With K_j = low + code * scale for every group of 64 values,
//   <q, K_j> = sum over groups of  scale_j * <q, code_j> + low_j * sum(q)
//   O        = sum_j (p_j scale_j) code_j + sum_j p_j low_j          (per group of columns)
// so both products run on the codes themselves: whole numbers below 16, exact in bf16.  A pair of codes becomes a pair of
// bf16 with one shift and one and-or, as 1 + code / 16 (the code in the upper mantissa bits of 1.0).  The ones are taken off
// again: of K by (low - 16 scale) in place of low, of V by one more product with a matrix of ones, which sums the very weights
// (rounded) that met the codes.  There half the range of the codes goes too, 8 * scale moving to the lows with the unrounded
// weights: what the rounding of a weight to bf16 is multiplied with is then at most 8 scales, not 15, and an output is off by
// what rounding the weights costs over a context in bf16 (two bf16 parts would end that, 24 contexts of up to 32K tokens 86
// us against 91).
//
// Transposed formulation: S^T = K Q^T, O^T = V^T P^T on 16x16x32 tiles whose columns are 16 flattened rows (query, head in
// the kv group).  A lane then holds the scores of its column for tokens 4g .. 4g + 3 of both blocks of a unit of 32 tokens,
// which is just what it has to hold of P^T for the second product: nothing crosses lanes, and since V lies in the cache
// by columns of four tokens, nothing goes through LDS either.  Softmax statistics are per lane; the reference point m of a
// column moves only when a score exceeds it by 2^8, the one case where lanes exchange it.
//
// With more than eight rows vector instructions are what it costs, so there the lows go through the matrix cores as well: the
// pairs of K as they lie in the cache, (scale, low), against (-sum(q), sum(q) / 16) in three bf16 parts; those of V, taken apart
// into rows of scales and of lows, against the weights in two bf16 parts (16 bits: a group may be small and far from zero, and
// its middle, low + 8 scale, has as many bits as its spread then; with one part values of 64 and -64 that cancel leave 0.04 behind, and
// a launch takes 2 to 6 % less).  A V that is no number would reach rows that do not see it
// that way (0 * inf), so units that not every row sees whole keep to the vector instructions.  32 rows a workgroup, two tiles
// of columns for every operand made of codes: 424 vector instructions for 32 rows (they are issued 79 % of the
// time, the matrix cores busy 29 %; 32 heads over 8, 4 requests of 8192 tokens with 200 new ones: 220 us, 480 TFLOP/s; 16 rows a
// workgroup 257 us).
//
// A workgroup of four wavefronts takes a split of a request's keys for one kv head and 8 to 32 rows; its wavefronts take the
// units in turn and meet in LDS at the end.  Where the keys are cut into several splits, a second launch merges them.
// With few rows the kernel is bound by HBM bandwidth as long as enough loads are in flight: every wavefront has two units of LDS
// of its own (three with 32 rows, where fewer wavefronts are there), filled by direct global->LDS loads (five a unit, no
// registers, no barrier) while it works on another one.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "common.h"
#include "mpic_q4.h"
#include "q4.h"
#include "wave_ops.h"

namespace mpic {
namespace {

using namespace q4;

constexpr int kWaves = 4;
constexpr int kUnit = 32;            // tokens a wavefront takes at a time: two blocks
constexpr float kSlack = 8.0f;       // a column's reference point may lag behind its greatest score by this much, log2 units
constexpr float kLowest = -3e38f;    // reference point of a column that has seen nothing
constexpr float kLn2 = 0.6931471805599453f;

// s_waitcnt lgkmcnt(0) only
#define MPIC_WAIT_LGKMCNT0() __builtin_amdgcn_s_waitcnt(0xC07F)

struct Q4AttnArgs {
  const char* q;
  const char* cache;
  const int32_t* q_off;
  const int32_t* table;
  const int32_t* lens;
  char* out;
  float* lse;
  float* ws_o;    // [rows][Hq][n_splits][D] normalised partial outputs
  float* ws_lse;  // [rows][Hq][n_splits] their log-sum-exp in log2 units, -inf: nothing seen
  int64_t n_rows, q_stride, table_width;  // q_stride in bytes
  int32_t n_blocks, page_blocks, max_q, max_len, n_splits, n_q_heads, n_kv_heads, group;
  int32_t split_units;  // units of a split
  float scale_log2;  // softmax_scale * log2(e)
};

// Queries of a request, within what the arguments allow whatever the device arrays hold
struct Request {
  int64_t first;  // first row
  int n, len;
};
__device__ inline Request request_of(const Q4AttnArgs& a, int b) {
  Request r;
  r.len = min(max(a.lens[b], 0), a.max_len);
  if (!a.q_off) {
    r.first = b;
    r.n = 1;
  } else {
    const int64_t lo = min(max(static_cast<int64_t>(a.q_off[b]), int64_t{0}), a.n_rows);
    const int64_t hi = min(max(static_cast<int64_t>(a.q_off[b + 1]), lo), a.n_rows);
    r.first = lo;
    r.n = static_cast<int>(min(hi - lo, static_cast<int64_t>(a.max_q)));
    // (the queries belong to the last tokens: those beyond max_q are the last of them)
    r.len = static_cast<int>(max(static_cast<int64_t>(r.len) - (hi - lo - r.n), int64_t{0}));
  }
  return r;
}

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// Two codes of a word as two bf16: those in bits 4n.. and 16 + 4n.., as 1 + code / 16, or exactly (for fp32) as code - 8
template <bool kExact, int n>
__device__ inline uint32_t pair_of(uint32_t w) {
  if (kExact) {
    const float lo = static_cast<float>(w >> (4 * n) & 15u) - 8.f, hi = static_cast<float>(w >> (16 + 4 * n) & 15u) - 8.f;
    return __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, hi), __builtin_bit_cast(uint32_t, lo), 0x07060302u);
  }
  const uint32_t moved = n == 0 ? w << 3 : w >> (4 * n - 3);
  // (one instruction, which takes a single constant from a scalar register: the mask stands in a vector register)
  uint32_t r;
  asm("v_and_or_b32 %0, %1, %2, %3" : "=v"(r) : "v"(moved), "v"(0x00780078u), "s"(0x3F803F80u));
  return r;
}
template <bool kExact>
__device__ inline bf16x8 keys_of(uint32_t w) {
  const u32x4 r = {pair_of<kExact, 0>(w), pair_of<kExact, 1>(w), pair_of<kExact, 2>(w), pair_of<kExact, 3>(w)};
  return __builtin_bit_cast(bf16x8, r);
}
// columns 2 * half and 2 * half + 1 of a V word of both blocks: tokens (0, 2), (1, 3) of either
template <bool kExact, int odd>
__device__ inline bf16x8 values_of(uint32_t w0, uint32_t w1) {
  const u32x4 r = {pair_of<kExact, odd>(w0), pair_of<kExact, 2 + odd>(w0), pair_of<kExact, odd>(w1), pair_of<kExact, 2 + odd>(w1)};
  return __builtin_bit_cast(bf16x8, r);
}

__device__ inline f32x4 mfma(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

template <int kParts>
struct Parts {
  bf16x8 p[kParts];
};
// x as a sum of kParts bf16 vectors (three hold the 24 bits of an fp32)
template <int kParts>
__device__ inline Parts<kParts> split_parts(f32x8 x) {
  Parts<kParts> r;
#pragma unroll
  for (int i = 0; i < kParts; ++i) {
    r.p[i] = __builtin_convertvector(x, bf16x8);
    if (i + 1 < kParts) x -= __builtin_convertvector(r.p[i], f32x8);
  }
  return r;
}

// How a wavefront's tiles of 16 columns are used.  Wide: a column is a row, and a lane works on all groups of its tokens.
// Narrow (head_dim 128, up to eight rows): the eight rows stand in the columns twice, the lower eight columns work on the
// first group of 64 values, the upper eight on the second.  A lane then reads, unpacks and applies the pairs of one group
// only, and what it lacks of a score is in the lane eight further: four wavefronts fit a SIMD instead of three (24 contexts of
// up to 32K tokens 87 us against 92 with a wide tile, 4 of 19841 17.4 against 18.6).
// Folded: lows through the matrix cores (fp32 pairs would not fit its operands, narrow tiles would gain nothing).
template <typename T, int D, bool kNarrow_, int kTiles_ = 1>
struct Shape {
  using Type = T;
  using B = Block<T, D>;
  static constexpr int kDim = D;
  static constexpr bool kNarrow = kNarrow_;
  static constexpr bool kExact = std::is_same<T, float>::value;
  static constexpr int kParts = kExact ? 3 : 1;
  static constexpr int kGroups = B::kGroups;
  static constexpr int kLaneGroups = kNarrow ? 1 : kGroups;  // groups a lane works on
  static constexpr bool kFolded = !kExact && !kNarrow;
  static constexpr int kTiles = kTiles_;                // of columns
  static constexpr int kRing = kTiles > 1 ? 3 : 2;      // units of LDS of a wavefront
  static constexpr int kTileRows = kNarrow ? 8 : 16;
  static constexpr int kRows = kTiles * kTileRows;      // flattened rows of a workgroup
  static constexpr int kWords = B::kLaneBytes / 4;
  static constexpr float kCode = kExact ? 1.f : 16.f;  // what a product with the codes has to be multiplied with
  static_assert(!kNarrow || (kGroups == 2 && !kExact), "two groups share the columns");
  static_assert(!kFolded || kGroups == 2, "four sums of two groups");
};

// A unit in LDS: the codes of its two blocks (K, then V), then the pairs of the first block (K, V), then of the second
template <typename T, int D>
struct Unit {
  using B = Block<T, D>;
  static constexpr int kCodes = 2 * B::kCodes;         // of a block
  static constexpr int kPairs = 2 * B::kPairs;
  static constexpr int kBytes = 2 * (kCodes + kPairs);
  static constexpr int kLoads = 2 * (kCodes / 1024) + 1;  // direct loads of a wavefront
  static_assert(kCodes % 1024 == 0 && 2 * kPairs <= 1024, "whole wavefronts load the codes, part of one the pairs");
};
template <typename T, int D>
struct Held {
  typedef uint32_t words __attribute__((ext_vector_type(Block<T, D>::kLaneBytes / 4)));
  typedef T pairs __attribute__((ext_vector_type(8)));  // scale, low of four tokens
};
// Block b's codes (kV: of V) and pairs of group g in this lane
template <typename T, int D, bool kV>
__device__ inline typename Held<T, D>::words codes_in(const char* unit, int b, int lane) {
  using U = Unit<T, D>;
  return *reinterpret_cast<const typename Held<T, D>::words*>(unit + b * U::kCodes + (kV ? U::B::kV : 0) + lane * U::B::kLaneBytes);
}
template <typename T, int D, bool kV>
__device__ inline typename Held<T, D>::pairs pairs_in(const char* unit, int b, int g, int quarter) {
  using U = Unit<T, D>;
  return *reinterpret_cast<const typename Held<T, D>::pairs*>(unit + 2 * U::kCodes + b * U::kPairs + (kV ? U::B::kPairs : 0) +
                                                              (g * kTokens + 4 * quarter) * U::B::kPair);
}

// Direct loads of 1024 and 2 x 1024 contiguous bytes to LDS, 16 a lane: base in scalar registers, the lane's offset in one
// vector register (an instruction's offset moves both addresses).  No compiler-visible load: the wait is by hand.
// Non-temporal: a decode step reads its contexts once (24 contexts, 421 MB: 82 us, 90 with ordinary loads).
__device__ inline void stage_1k(const char* base, uint32_t offset, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1 nt" : : "v"(offset), "s"(base), "s"(lds) : "memory", "m0");
}
__device__ inline void stage_2k(const char* base, uint32_t offset, uint32_t lds) {
  asm volatile(
      "s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1 nt\n\tglobal_load_lds_dwordx4 %0, %1 offset:1024 nt"
      :
      : "v"(offset), "s"(base), "s"(lds)
      : "memory", "m0");
}
template <typename T, int D>
__device__ inline void stage_unit(const char* block0, const char* block1, int lane, uint32_t lds) {
  using U = Unit<T, D>;
  constexpr int kLanes = U::kPairs / 16;  // lanes that load the pairs of a block
  if (U::kCodes == 2048) {
    stage_2k(block0, 16 * lane, lds);
    stage_2k(block1, 16 * lane, lds + U::kCodes);
  } else {
    stage_1k(block0, 16 * lane, lds);
    stage_1k(block1, 16 * lane, lds + U::kCodes);
  }
  if (lane < 2 * kLanes)
    load_to_lds_16B((lane < kLanes ? block0 : block1) + U::kCodes + 16 * (lane % kLanes), lds + 2 * U::kCodes);
}

// State of a column tile in one wavefront
template <typename S>
struct Columns {
  Parts<S::kParts> q[S::kGroups][2];  // (narrow: zeros where a column does not work on the group)
  float q_sum[S::kLaneGroups];
  bf16x8 q_pairs;              // folded: what the pairs of K meet, (-sum(q), sum(q) / 16) of both groups in parts
  f32x4 o[S::kGroups][4];      // O^T: lane (column, quarter c) holds columns 64 g + 16 c + 4 r + tile of the output
  f32x4 ones[S::kLaneGroups];  // sums of the rounded weights
  f32x4 sums;                  // folded: sums p scale of both groups, then p low
  float low[S::kLaneGroups];   // sum p * (low + 8 scale), this lane's tokens (folded: of masked units)
  float m, l;                  // reference point (log2 units, the same in the lanes of a column), sum p of this lane's tokens
  int limit;                   // positions 0 .. limit - 1 are seen
};

// What the lane eight further among sixteen holds
__device__ inline float other_half(float x) {
  const int i = __builtin_bit_cast(int, x);
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(i, i, 0x128, 0xf, 0xf, true));  // rotation of the row by eight
}

// (fmaxf makes a second instruction of every operand that may be a signalling NaN; a score that is none shows in its weight)
__device__ inline float max3(float a, float b, float c) {
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}

// One unit of 32 tokens.  masked: not every token is seen by every column (or a block is missing: bit of `have`).
template <typename S>
__device__ inline void attend_unit(Columns<S> (&s)[S::kTiles], const char* unit, int pos, bool masked, int have, int lane, float factor) {
  using T = typename S::Type;
  using U = Unit<T, S::kDim>;
  constexpr int D = S::kDim, kTiles = S::kTiles;
  typedef typename Held<T, D>::words words;
  typedef typename Held<T, D>::pairs pairs;
  const int quarter = lane >> 4, my_group = S::kNarrow ? (lane >> 3 & 1) : 0;
  float x[kTiles][2][4];
#pragma unroll
  for (int b = 0; b < 2; ++b) {
    const words k = codes_in<T, D, false>(unit, b, lane);
    f32x4 acc[kTiles][S::kLaneGroups], lows[kTiles];
    if (S::kFolded) {
      const uint32_t pair = *reinterpret_cast<const uint32_t*>(unit + 2 * U::kCodes + b * U::kPairs + ((quarter & 1) * kTokens + (lane & 15)) * 4);
      const u32x4 four = {pair, pair, pair, pair};
#pragma unroll
      for (int t = 0; t < kTiles; ++t) lows[t] = mfma(__builtin_bit_cast(bf16x8, four), s[t].q_pairs, f32x4{0});
    }
#pragma unroll
    for (int g = 0; g < S::kGroups; ++g) {
      const int lg = S::kNarrow ? 0 : g;
      const bf16x8 keys[2] = {keys_of<S::kExact>(k[2 * g]), keys_of<S::kExact>(k[2 * g + 1])};
#pragma unroll
      for (int t = 0; t < kTiles; ++t) {
        if (!S::kNarrow || g == 0) acc[t][lg] = f32x4{0};
        // (the small parts first)
#pragma unroll
        for (int i = S::kParts - 1; i >= 0; --i)
#pragma unroll
          for (int w = 0; w < 2; ++w) acc[t][lg] = mfma(keys[w], s[t].q[g][w].p[i], acc[t][lg]);
      }
    }
    f32x4 sum[kTiles];
#pragma unroll
    for (int t = 0; t < kTiles; ++t) sum[t] = S::kFolded ? lows[t] : f32x4{0};
#pragma unroll
    for (int g = 0; g < S::kLaneGroups; ++g) {
      const pairs p = pairs_in<T, D, false>(unit, b, S::kNarrow ? my_group : g, quarter);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float scale = static_cast<float>(p[2 * r]);
        float low = static_cast<float>(p[2 * r + 1]);
        low = fmaf(S::kExact ? 8.f : -16.f, scale, low);  // (what the codes' operands lack, or have too much)
#pragma unroll
        for (int t = 0; t < kTiles; ++t)
          sum[t][r] = fmaf(scale, acc[t][g][r], S::kFolded ? sum[t][r] : g ? fmaf(low, s[t].q_sum[g], sum[t][r]) : low * s[t].q_sum[g]);
      }
    }
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) x[t][b][r] = S::kNarrow ? sum[t][r] + other_half(sum[t][r]) : sum[t][r];
  }
  if (masked) {
    asm volatile("");  // (a branch: few units are, and the others should not pay for it)
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const bool seen = (have >> b & 1) && pos + kTokens * b + 4 * quarter + r < s[t].limit;
          x[t][b][r] = seen ? x[t][b][r] : -INFINITY;
        }
  }
  float p[kTiles][2][4];
#pragma unroll
  for (int t = 0; t < kTiles; ++t) {
    const float top = max3(max3(x[t][0][0], x[t][0][1], x[t][0][2]), max3(x[t][0][3], x[t][1][0], x[t][1][1]), max3(x[t][1][2], x[t][1][3], x[t][1][3])) * factor;
    if (__any(top > s[t].m + kSlack)) {
      float m = fmaxf(s[t].m, top);
      m = fmaxf(m, __shfl_xor(m, 16));
      m = fmaxf(m, __shfl_xor(m, 32));
      const float f = __builtin_amdgcn_exp2f(s[t].m - m);
      s[t].m = m;
      s[t].l *= f;
      if (S::kFolded) s[t].sums *= f;
#pragma unroll
      for (int g = 0; g < S::kLaneGroups; ++g) {
        s[t].low[g] *= f;
        if (!S::kExact) s[t].ones[g] *= f;
      }
#pragma unroll
      for (int g = 0; g < S::kGroups; ++g)
#pragma unroll
        for (int c = 0; c < 4; ++c) s[t].o[g][c] *= f;
    }
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        p[t][b][r] = __builtin_amdgcn_exp2f(fmaf(x[t][b][r], factor, -s[t].m));
        s[t].l += p[t][b][r];
      }
  }
  float scaled[kTiles][S::kLaneGroups][2][4], low[kTiles][S::kLaneGroups][2][4];
#pragma unroll
  for (int g = 0; g < S::kLaneGroups; ++g)
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const pairs vp = pairs_in<T, D, true>(unit, b, S::kNarrow ? my_group : g, quarter);
#pragma unroll
      for (int t = 0; t < kTiles; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          scaled[t][g][b][r] = p[t][b][r] * static_cast<float>(vp[2 * r]);
          if (!S::kFolded) low[t][g][b][r] = fmaf(8.f, scaled[t][g][b][r], p[t][b][r] * static_cast<float>(vp[2 * r + 1]));
        }
    }
  if (masked) {  // (the pairs of what is not seen may be no number)
    asm volatile("");
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
#pragma unroll
      for (int g = 0; g < S::kLaneGroups; ++g)
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          pairs vp;
          if (S::kFolded) vp = pairs_in<T, D, true>(unit, b, g, quarter);
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            if (S::kFolded) low[t][g][b][r] = fmaf(8.f, scaled[t][g][b][r], p[t][b][r] * static_cast<float>(vp[2 * r + 1]));
            if (x[t][b][r] == -INFINITY) scaled[t][g][b][r] = low[t][g][b][r] = 0.f;
            if (S::kFolded) s[t].low[g] += low[t][g][b][r];
          }
        }
  } else if (S::kFolded) {
    // rows of the operand, four times over: the scales of both groups, then the lows; tokens as in the weights
    const char* at = unit + 2 * U::kCodes + U::B::kPairs + ((lane & 1) * kTokens + 4 * quarter) * 4;
    const uint32_t take = lane & 2 ? 0x07060302u : 0x05040100u;
    u32x4 four;
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const u32x4 raw = *reinterpret_cast<const u32x4*>(at + b * U::kPairs);
      four[2 * b] = __builtin_amdgcn_perm(raw[2], raw[0], take);
      four[2 * b + 1] = __builtin_amdgcn_perm(raw[3], raw[1], take);
    }
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
      // the weights in two parts: their upper halves as they are, and what is left
      u32x4 high;
      f32x8 rest;
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          const uint32_t x0 = __builtin_bit_cast(uint32_t, p[t][b][r]), x2 = __builtin_bit_cast(uint32_t, p[t][b][r + 2]);
          high[2 * b + r] = __builtin_amdgcn_perm(x2, x0, 0x07060302u);
          rest[4 * b + 2 * r] = p[t][b][r] - __builtin_bit_cast(float, x0 & 0xFFFF0000u);
          rest[4 * b + 2 * r + 1] = p[t][b][r + 2] - __builtin_bit_cast(float, x2 & 0xFFFF0000u);
        }
      s[t].sums = mfma(__builtin_bit_cast(bf16x8, four), __builtin_convertvector(rest, bf16x8), s[t].sums);
      s[t].sums = mfma(__builtin_bit_cast(bf16x8, four), __builtin_bit_cast(bf16x8, high), s[t].sums);
    }
  }
  Parts<S::kParts> weights[kTiles][S::kLaneGroups];
#pragma unroll
  for (int t = 0; t < kTiles; ++t)
#pragma unroll
    for (int g = 0; g < S::kLaneGroups; ++g) {
      f32x8 w;
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          w[4 * b + (r & 1) * 2 + (r >> 1)] = scaled[t][g][b][r];  // tokens (0, 2), (1, 3)
          if (!S::kFolded) s[t].low[g] += low[t][g][b][r];
        }
      weights[t][g] = split_parts<S::kParts>(w);
    }
  if (!S::kExact) {
    const u32x4 one = {0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u};
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
#pragma unroll
      for (int g = 0; g < S::kLaneGroups; ++g) s[t].ones[g] = mfma(__builtin_bit_cast(bf16x8, one), weights[t][g].p[0], s[t].ones[g]);
  }
  const words v0 = codes_in<T, D, true>(unit, 0, lane), v1 = codes_in<T, D, true>(unit, 1, lane);
#pragma unroll
  for (int g = 0; g < S::kGroups; ++g)
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const bf16x8 even = values_of<S::kExact, 0>(v0[2 * g + c], v1[2 * g + c]), odd = values_of<S::kExact, 1>(v0[2 * g + c], v1[2 * g + c]);
#pragma unroll
      for (int t = 0; t < kTiles; ++t)
#pragma unroll
        for (int i = S::kParts - 1; i >= 0; --i) {
          s[t].o[g][2 * c] = mfma(even, weights[t][S::kNarrow ? 0 : g].p[i], s[t].o[g][2 * c]);
          s[t].o[g][2 * c + 1] = mfma(odd, weights[t][S::kNarrow ? 0 : g].p[i], s[t].o[g][2 * c + 1]);
        }
    }
}

// LDS: the units of every wavefront; at the end their partial results (rows of D + 4 floats, reference points, sums)
template <typename S>
struct AttnLds {
  using U = Unit<typename S::Type, S::kDim>;
  static constexpr int kRow = S::kDim + 4;
  static constexpr int kWave = S::kRing * U::kBytes;
  static constexpr int kMerge = kWaves * S::kTileRows * (kRow + 2) * 4;
  static constexpr int kBytes = kWaves * kWave > kMerge ? kWaves * kWave : kMerge;
  static_assert(kBytes <= 65536, "no opt-in needed");
};

template <typename S, int kWavesPerSimd>
__global__ __launch_bounds__(kWaves * 64, kWavesPerSimd) void q4_attn_kernel(Q4AttnArgs a) {
  using T = typename S::Type;
  constexpr int D = S::kDim;
  using B = Block<T, D>;
  using L = AttnLds<S>;
  using U = Unit<T, D>;
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  typedef float PartRows[S::kTileRows][L::kRow];
  typedef float PartCols[S::kTileRows];
  PartRows* part_o = reinterpret_cast<PartRows*>(lds);
  PartCols* part_m = reinterpret_cast<PartCols*>(part_o + kWaves);
  PartCols* part_l = part_m + kWaves;
  const int lane = threadIdx.x & 63, col = lane & (S::kTileRows - 1), quarter = lane >> 4;
  const int my_group = S::kNarrow ? (lane >> 3 & 1) : 0;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // heads first: neighbouring workgroups go to different L2 domains, which thus get the same share of every split, and the
  // row tiles of a head that read the same keys run together
  const int head = blockIdx.x % a.n_kv_heads, split = blockIdx.y, b = blockIdx.z;
  const int row0 = static_cast<int>(blockIdx.x / a.n_kv_heads) * S::kRows;
  // The way to the first keys is a chain of loads: what the table says of this wavefront's blocks is asked for before the
  // length is known, and the first unit before the queries are converted.
  const int unit0 = split * a.split_units + wave;
  const int32_t* table = a.table + b * a.table_width;
  // entry of the block that a lane looks after, two lanes a unit, from the wavefront's unit i0 on
  const auto block_of_lane = [&](int i0) { return 2 * (unit0 + (i0 + (lane >> 1)) * kWaves) + (lane & 1); };
  const auto entry_of = [&](int block) {
    const int page = block / a.page_blocks;
    return page < a.table_width ? table[page] : -1;
  };
  int entry = entry_of(block_of_lane(0));
  const Request rq = request_of(a, b);
  const int n_flat = rq.n * a.group;
  if (row0 >= n_flat) return;
  const int last = (min(row0 + S::kRows, n_flat) - 1) / a.group;  // last query of the workgroup
  const int behind = rq.len - rq.n;                            // tokens in front of the new ones (negative: some have no position)
  const int key_end = max(behind + last + 1, 0);
  const int key_all = behind + row0 / a.group + 1;             // the keys below are seen by every row
  const int unit_end = min((key_end + kUnit - 1) / kUnit, (split + 1) * a.split_units);
  if (a.n_splits > 1 && unit_end <= split * a.split_units) return;  // (the merge asks for no such split)

  Columns<S> s[S::kTiles];
  typedef T vec __attribute__((ext_vector_type(8), aligned(16)));
  vec raw[S::kTiles][S::kGroups][2];
#pragma unroll
  for (int t = 0; t < S::kTiles; ++t) {
    const int at = row0 + t * S::kTileRows + col, flat = min(at, n_flat - 1), token = flat / a.group, hq = head * a.group + flat % a.group;
    s[t].limit = at < n_flat ? behind + token + 1 : 0;
    const char* q = a.q + (rq.first + token) * a.q_stride + static_cast<int64_t>(hq) * D * sizeof(T);
#pragma unroll
    for (int g = 0; g < S::kGroups; ++g)
#pragma unroll
      for (int w = 0; w < 2; ++w) raw[t][g][w] = *reinterpret_cast<const vec*>(q + (g * kGroup + quarter * 16 + w * 8) * sizeof(T));
  }
  const int n_units = unit_end > unit0 ? (unit_end - unit0 + kWaves - 1) / kWaves : 0;  // of this wavefront
  // the blocks of the next 32 units, two lanes a unit; -1: not in the cache
  int ids = -1;
  const auto look_up = [&](int i0) {
    const int block = block_of_lane(i0);
    if (i0) entry = entry_of(block);
    const int64_t id = static_cast<int64_t>(entry) * a.page_blocks + block % a.page_blocks;
    ids = id >= 0 && id < a.n_blocks && block < (key_end + kTokens - 1) / kTokens ? static_cast<int>(id) : -1;
  };
  char* ring = lds + wave * L::kWave;
  const uint32_t ring_lds = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(MPIC_LDS_PTR(char, ring)));
  // load unit i of this wavefront into the next place of its ring; bit b of the result: block b is in the cache
  int ring_at = 0;  // of unit i to be staged
  auto stage = [&](int i) {
    if ((i & 31) == 0) look_up(i);
    const int id0 = __builtin_amdgcn_readlane(ids, 2 * i & 63), id1 = __builtin_amdgcn_readlane(ids, (2 * i & 63) + 1);
    const char* base = a.cache + static_cast<int64_t>(head) * B::kBytes;
    const int64_t pitch = static_cast<int64_t>(a.n_kv_heads) * B::kBytes;
    stage_unit<T, D>(base + max(id0, 0) * pitch, base + max(id1, 0) * pitch, lane, ring_lds + ring_at);
    ring_at = ring_at == (S::kRing - 1) * U::kBytes ? 0 : ring_at + U::kBytes;
    return (id0 >= 0 ? 1 : 0) | (id1 >= 0 ? 2 : 0);
  };
  int have = 0, have_next = 0;
  if (n_units > 0) have = stage(0);
  if (S::kRing > 2 && n_units > 1) have_next = stage(1);
#pragma unroll
  for (int t = 0; t < S::kTiles; ++t) {
    s[t].m = kLowest;
    s[t].l = 0.f;
    s[t].sums = f32x4{0};
#pragma unroll
    for (int g = 0; g < S::kLaneGroups; ++g) s[t].q_sum[g] = s[t].low[g] = 0.f, s[t].ones[g] = f32x4{0};
#pragma unroll
    for (int g = 0; g < S::kGroups; ++g) {
      const int lg = S::kNarrow ? 0 : g;
#pragma unroll
      for (int c = 0; c < 4; ++c) s[t].o[g][c] = f32x4{0};
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        f32x8 x = __builtin_convertvector(raw[t][g][w], f32x8);
        if (S::kNarrow && g != my_group) x = f32x8{0};
        s[t].q[g][w] = split_parts<S::kParts>(x);
#pragma unroll
        for (int e = 0; e < 8; ++e) s[t].q_sum[lg] += x[e];
      }
    }
#pragma unroll
    for (int g = 0; g < S::kLaneGroups; ++g) {
      s[t].q_sum[g] += __shfl_xor(s[t].q_sum[g], 16);
      s[t].q_sum[g] += __shfl_xor(s[t].q_sum[g], 32);
      s[t].q_sum[g] *= 1.f / S::kCode;
    }
    if (S::kFolded) {
      // a product of (scale, low) pairs with (-sum(q), sum(q) / 16): of one group per quarter, its three bf16 parts one after
      // the other; two quarters have nothing
      const float sum = quarter == 0 ? s[t].q_sum[0] : quarter == 1 ? s[t].q_sum[S::kLaneGroups - 1] : 0.f;
      f32x8 x = f32x8{0};
      float rest = sum;
#pragma unroll
      for (int i = 0; i < 3; ++i) {
        const float part = static_cast<float>(static_cast<__bf16>(rest));
        x[2 * i] = -16.f * part;
        x[2 * i + 1] = part;
        rest -= part;
      }
      s[t].q_pairs = __builtin_convertvector(x, bf16x8);
    }
  }
  const float factor = a.scale_log2 * S::kCode;
  int unit_at = 0;
  for (int i = 0; i < n_units; ++i) {
    // what was read of the unit that is loaded next has arrived (all of it has been used, but nothing else orders the two)
    MPIC_WAIT_LGKMCNT0();
    asm volatile("" ::: "memory");
    int have_last = 0;
    if (i + S::kRing - 1 < n_units) {
      have_last = stage(i + S::kRing - 1);
      MPIC_WAIT_VMCNT((S::kRing - 1) * U::kLoads);
    } else if (S::kRing > 2 && i + 1 < n_units) {
      MPIC_WAIT_VMCNT(U::kLoads);
    } else {
      MPIC_WAIT_VMCNT(0);
    }
    asm volatile("" ::: "memory");
    const int pos = (unit0 + i * kWaves) * kUnit;
    attend_unit(s, ring + unit_at, pos, have != 3 || pos + kUnit > key_all, have, lane, factor);
    unit_at = unit_at == (S::kRing - 1) * U::kBytes ? 0 : unit_at + U::kBytes;
    have = S::kRing > 2 ? have_next : have_last;
    have_next = have_last;
  }

#pragma unroll
  for (int t = 0; t < S::kTiles; ++t) {
    __syncthreads();  // (the ring has been read, or the tile in front)
    s[t].l += __shfl_xor(s[t].l, 16);
    s[t].l += __shfl_xor(s[t].l, 32);
    if (lane < S::kTileRows) {
      part_m[wave][col] = s[t].m;
      part_l[wave][col] = s[t].l;
    }
#pragma unroll
    for (int g = 0; g < S::kLaneGroups; ++g) {
      s[t].low[g] += __shfl_xor(s[t].low[g], 16);
      s[t].low[g] += __shfl_xor(s[t].low[g], 32);
      if (S::kFolded) s[t].low[g] += fmaf(8.f, s[t].sums[g & 1], s[t].sums[2 + (g & 1)]);
      const int group = S::kNarrow ? my_group : g;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        f32x4 o;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const float sum = S::kNarrow && my_group ? s[t].o[S::kGroups - 1][c][r] : s[t].o[g][c][r];
          o[c] = S::kExact ? sum + s[t].low[g] : fmaf(fmaf(-1.5f, s[t].ones[g][r], sum), S::kCode, s[t].low[g]);
        }
        *reinterpret_cast<f32x4*>(&part_o[wave][col][group * kGroup + quarter * 16 + 4 * r]) = o;
      }
    }
    __syncthreads();

    constexpr int kThreads = kWaves * 64 / S::kTileRows, kEach = D / kThreads;  // threads and values per row
    typedef float each __attribute__((ext_vector_type(kEach), aligned(16)));
    const int c = threadIdx.x / kThreads, d0 = threadIdx.x % kThreads * kEach, at = row0 + t * S::kTileRows + c;
    if (at < n_flat) {
      float top = part_m[0][c];
#pragma unroll
      for (int w = 1; w < kWaves; ++w) top = fmaxf(top, part_m[w][c]);
      float z = 0.f;
      each o = each{0};
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const float f = __builtin_amdgcn_exp2f(part_m[w][c] - top);
        z = fmaf(f, part_l[w][c], z);
        o += *reinterpret_cast<const each*>(&part_o[w][c][d0]) * f;
      }
      const bool none = z == 0.f;
      const float inv = none ? 0.f : 1.f / z, lse2 = none ? -INFINITY : top + log2f(z);
      o *= inv;
      const int64_t row = (rq.first + at / a.group) * a.n_q_heads + head * a.group + at % a.group;
      if (a.n_splits > 1) {
        const int64_t part = row * a.n_splits + split;
        if (d0 == 0) a.ws_lse[part] = lse2;
        if (!none) *reinterpret_cast<each*>(a.ws_o + part * D + d0) = o;
      } else {
        typedef T vec __attribute__((ext_vector_type(kEach), aligned(8)));
        *reinterpret_cast<vec*>(a.out + (row * D + d0) * sizeof(T)) = __builtin_convertvector(o, vec);
        if (a.lse && d0 == 0) a.lse[row] = lse2 * kLn2;
      }
    }
  }
}

// Output rows from the partial results of their splits: D / 4 threads hold four columns each, and kShares of them share the
// splits, in a fixed order.
template <typename T, int D, int kShares>
__global__ __launch_bounds__(256) void q4_merge_kernel(Q4AttnArgs a) {
  constexpr int kLanes = D / 4, kRows = 256 / kLanes / kShares;
  __shared__ __attribute__((aligned(16))) float sums[kShares][kRows][D];
  __shared__ float tops[kShares][kRows], zs[kShares][kRows];
  const Request rq = request_of(a, blockIdx.y);
  const int lane = threadIdx.x % kLanes, share = threadIdx.x / kLanes % kShares, mine = threadIdx.x / kLanes / kShares;
  const int64_t i = static_cast<int64_t>(blockIdx.x) * kRows + mine, n_rows = static_cast<int64_t>(rq.n) * a.n_q_heads;
  if (static_cast<int64_t>(blockIdx.x) * kRows >= n_rows) return;  // (the whole workgroup)
  const int64_t row = rq.first * a.n_q_heads + i;
  const float* part = a.ws_lse + row * a.n_splits;
  // splits that hold keys of this row
  const int keys = i < n_rows ? max(rq.len - rq.n + static_cast<int>(i / a.n_q_heads) + 1, 0) : 0;
  const int n_splits = keys > 0 ? min(((keys - 1) / kUnit) / a.split_units + 1, a.n_splits) : 0;
  // eight splits at a time: their loads do not wait for each other, nor an output for the log-sum-exp that says whether it
  // was written at all
  constexpr int kBatch = 8;
  float top = kLowest, z = 0.f;
  f32x4 o = f32x4{0};
  for (int s0 = share; s0 < n_splits; s0 += kBatch * kShares) {
    float lse[kBatch];
    f32x4 part_o[kBatch];
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      const int s = s0 + k * kShares, at = min(s, n_splits - 1);
      lse[k] = s < n_splits ? part[at] : -INFINITY;
      part_o[k] = *reinterpret_cast<const f32x4*>(a.ws_o + (row * a.n_splits + at) * D + 4 * lane);
    }
    float m = top;
#pragma unroll
    for (int k = 0; k < kBatch; ++k) m = fmaxf(m, lse[k]);
    const float f = __builtin_amdgcn_exp2f(top - m);
    top = m;
    z *= f;
    o *= f;
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      const float w = __builtin_amdgcn_exp2f(lse[k] - m);
      z += w;
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = lse[k] == -INFINITY ? o[e] : fmaf(part_o[k][e], w, o[e]);
    }
  }
  if (kShares > 1) {
    *reinterpret_cast<f32x4*>(&sums[share][mine][4 * lane]) = o;
    if (lane == 0) {
      tops[share][mine] = top;
      zs[share][mine] = z;
    }
    __syncthreads();
    if (share > 0) return;
#pragma unroll
    for (int k = 1; k < kShares; ++k) top = fmaxf(top, tops[k][mine]);
    z = 0.f;
    o = f32x4{0};
#pragma unroll
    for (int k = 0; k < kShares; ++k) {
      const float f = __builtin_amdgcn_exp2f(tops[k][mine] - top);
      z = fmaf(f, zs[k][mine], z);
      o += *reinterpret_cast<const f32x4*>(&sums[k][mine][4 * lane]) * f;
    }
  }
  if (i >= n_rows) return;
  const float inv = z == 0.f ? 0.f : 1.f / z;
  typedef T vec __attribute__((ext_vector_type(4)));
  *reinterpret_cast<vec*>(a.out + (row * D + 4 * lane) * sizeof(T)) = __builtin_convertvector(o * inv, vec);
  if (a.lse && lane == 0) a.lse[row] = z == 0.f ? -INFINITY : (top + log2f(z)) * kLn2;
}

// Rows of a workgroup and how the keys are cut.
//
// 8 rows where that is all there is.  Beyond that 16 or 32: a unit of 32 rows costs 1.3 times the instructions of one of 16, but
// takes longer from its first to its last, and only half as many wavefronts fit.  So 32 rows need a launch that fills the
// machine, (tiles of 16 rows) * (units of keys) over all kv heads and requests, and no more than a third of its tiles' rows may
// be without one: 9 500 of those units 19.9 us against 19.0 with 16 rows, 16 200 23.4 against 22.9, 22 800 24.0 against 25.5, 82 400
// 62.5 against 70.9, 410 000 220 against 257 (36 rows over 512 tokens 11 us against 8).
//
// 8 or 16 rows: splits of whole units for every wavefront, so that three workgroups a compute unit are there where the requests
// alone do not make them (four would fit with 8 rows, but smaller splits cost more: 4 requests of 19841 tokens 18.5 us
// against 17.6), and no less than two units a wavefront.  Lengths differ, and a launch is over when its longest split is:
// splits are cut down to 32 units as long as that makes no more than eight rounds of them.
// 32 rows: workgroups take longer, so their rounds count (two a compute unit): the number of splits with the least rounds *
// (units of a split + 16), 16 being what a workgroup and its share of the merge cost besides (2 requests of 16000 tokens with 256
// new ones 240 us; 10 % more by the rule above).
// Five units a wavefront stay in one piece: a further unit takes 0.9 us (4 requests of 128 tokens 4.5 us, of 256 5.4), the
// merge 2.7 and its launch 2.3 of the host.
struct Cut {
  int32_t rows;  // flattened rows of a workgroup
  int32_t n_splits, split_units;
  int64_t tiles;
};
Cut cut_of(const mpic_ctx* ctx, int32_t n_requests, int32_t max_q, int64_t max_len) {
  constexpr int64_t kWhole = 5 * kWaves, kLeast = 2 * kWaves, kRound = 768, kRounds = 8, kMost = 32;
  constexpr int64_t kRound32 = 512, kCost32 = 16, kSplits32 = 64, kLarge = 16384;
  const int64_t units = std::max<int64_t>(1, (max_len + kUnit - 1) / kUnit), flat = static_cast<int64_t>(max_q) * ctx->group;
  const int64_t tiles16 = (flat + 15) / 16, tiles32 = (flat + 31) / 32;
  const double work = static_cast<double>(tiles16 * ctx->cfg.n_kv_heads) * n_requests * units;
  Cut cut{};
  cut.rows = ctx->cfg.dtype != MPIC_BF16 ? 16 : flat <= 8 ? 8 : work < kLarge || 5 * tiles32 > 3 * tiles16 ? 16 : 32;
  cut.tiles = (flat + cut.rows - 1) / cut.rows;
  const int64_t lanes = cut.tiles * ctx->cfg.n_kv_heads * n_requests;
  const auto units_of = [&](int64_t splits) { return ((units + splits - 1) / splits + kWaves - 1) / kWaves * kWaves; };
  int64_t each = kWhole;
  if (units > kWhole && cut.rows == 32) {
    double best = INFINITY;
    for (int64_t splits = 1; splits <= kSplits32; ++splits) {
      const int64_t n = std::max(kLeast, units_of(splits)), used = (units + n - 1) / n;
      const double cost = static_cast<double>((lanes * used + kRound32 - 1) / kRound32) * (n + kCost32);
      if (cost >= best) continue;
      best = cost;
      each = n;
    }
  } else if (units > kWhole) {
    const auto of_rounds = [&](int64_t rounds) { return units_of(std::max<int64_t>(1, rounds * kRound / lanes)); };
    each = std::max(kLeast, std::min(of_rounds(1), std::max(kMost, of_rounds(kRounds))));
  }
  cut.split_units = static_cast<int32_t>(each);
  cut.n_splits = static_cast<int32_t>((units + each - 1) / each);
  return cut;
}
// (n_rows * n_q_heads: nothing derived from it passes 64 bits)
bool sizes_fit(const mpic_ctx* ctx, int32_t n_requests, int64_t n_rows, int32_t max_q, int64_t max_len) {
  return n_requests >= 0 && n_rows >= 0 && max_q >= 1 && max_len >= 0 && n_rows < INT32_MAX && n_rows * ctx->cfg.n_q_heads < int64_t{1} << 38 && max_len <= INT32_MAX - 64 &&
         static_cast<int64_t>(max_q) * ctx->group < INT32_MAX - 256;
}
// The grids of both launches hold them
bool launch_fits(const mpic_ctx* ctx, int32_t n_requests, int32_t max_q) {
  const int64_t tiles = (static_cast<int64_t>(max_q) * ctx->group + 7) / 8;
  return tiles * ctx->cfg.n_kv_heads <= INT32_MAX / (kWaves * 64) && static_cast<int64_t>(max_q) * ctx->cfg.n_q_heads <= INT32_MAX / 256 &&
         n_requests <= 65535;
}
int64_t workspace_of(const mpic_ctx* ctx, const Cut& cut, int64_t n_rows) {
  return cut.n_splits > 1 ? n_rows * ctx->cfg.n_q_heads * cut.n_splits * (ctx->cfg.head_dim + 1) * 4 : 0;
}

template <typename S, int kWavesPerSimd>
hipError_t launch_q4_attn(const Q4AttnArgs& a, dim3 grid, hipStream_t stream) {
  hipLaunchKernelGGL((q4_attn_kernel<S, kWavesPerSimd>), grid, dim3(kWaves * 64), AttnLds<S>::kBytes, stream, a);
  return hipGetLastError();
}
template <typename T, int D>
hipError_t launch_q4_merge(const Q4AttnArgs& a, int32_t n_requests, hipStream_t stream) {
  // a group of threads walks eight splits with one batch of loads: up to 8 splits one group a row, up to 16 two, then eight
  // (16384 rows of 8 splits: 28 us with eight groups a row, 10 with one)
  const auto go = [&](auto shares) {
    constexpr int kShares = decltype(shares)::value, kRows = 256 / (D / 4) / kShares;
    const int64_t rows = static_cast<int64_t>(a.max_q) * a.n_q_heads;
    hipLaunchKernelGGL((q4_merge_kernel<T, D, kShares>), dim3(static_cast<unsigned>((rows + kRows - 1) / kRows), n_requests), dim3(256), 0, stream, a);
  };
  if (a.n_splits <= 8)
    go(std::integral_constant<int, 1>{});
  else if (a.n_splits <= 16)
    go(std::integral_constant<int, 2>{});
  else
    go(std::integral_constant<int, 8>{});
  return hipGetLastError();
}

}  // namespace
}  // namespace mpic

extern "C" int mpic_q4_attn_workspace(const mpic_ctx* ctx, int32_t n_requests, int64_t n_rows, int32_t max_q, int64_t max_len,
                                      int64_t* bytes) {
  if (!ctx || !bytes || !mpic::sizes_fit(ctx, n_requests, n_rows, max_q, max_len)) return MPIC_ERR_INVALID;
  if (!mpic::launch_fits(ctx, n_requests, max_q)) return MPIC_ERR_UNSUPPORTED;
  *bytes = n_requests == 0 ? 0 : mpic::workspace_of(ctx, mpic::cut_of(ctx, n_requests, max_q, max_len), n_rows);
  return MPIC_OK;
}

extern "C" int mpic_q4_attn(mpic_ctx* ctx, const void* q, int64_t q_stride, int64_t n_rows, const int32_t* q_off, int32_t max_q,
                            const void* cache, int64_t cache_bytes, int64_t n_slots, const int32_t* page_table,
                            int64_t table_width, int32_t page_size, const int32_t* lens, int32_t n_requests, int64_t max_len, double softmax_scale,
                            void* out, float* lse, void* workspace, int64_t workspace_bytes, void* stream_) {
  using namespace mpic;
  if (!ctx) return MPIC_ERR_INVALID;
  const mpic_config& c = ctx->cfg;
  const int64_t elem = c.dtype == MPIC_F32 ? 4 : 2;
  const auto invalid = [&](const char* why) { return fail(ctx, MPIC_ERR_INVALID, why); };
  if (!sizes_fit(ctx, n_requests, n_rows, max_q, max_len)) return invalid("q4_attn: bad row, request or token count");
  if (!q_off && (n_rows != n_requests || max_q != 1)) return invalid("q4_attn: without q_off there is one query per request");
  if (page_size <= 0 || page_size % q4::kTokens) return invalid("q4_attn: page_size must be a positive multiple of 16");
  if (table_width < 0 || table_width > INT32_MAX || max_len > table_width * page_size) return invalid("q4_attn: page table narrower than max_len");
  if (n_slots < 0 || n_slots >= INT32_MAX) return invalid("q4_attn: bad slot count");
  // (16 log2(e) times it is an fp32 number that is neither zero, which a masked -inf would make no number, nor infinite)
  if (!(softmax_scale >= 0x1p-126 && softmax_scale <= 0x1p123)) return invalid("q4_attn: softmax_scale must be positive, 2^-126 to 2^123");
  if (q_stride < static_cast<int64_t>(c.n_q_heads) * c.head_dim || q_stride * elem % 16)
    return invalid("q4_attn: q_stride must hold a row and be a multiple of 16 bytes");
  if (cache_bytes < q4::cache_bytes(c.dtype == MPIC_F32, c.head_dim, c.n_kv_heads, n_slots)) return invalid("q4_attn: the cache is smaller than its slots");
  if (n_rows == 0 || n_requests == 0) return MPIC_OK;
  if (!q || !cache || !lens || !out || (max_len > 0 && !page_table)) return invalid("q4_attn: null buffer");
  if (max_len > 0 && n_slots == 0) return invalid("q4_attn: a cache without slots");
  if ((reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(cache) | reinterpret_cast<uintptr_t>(out) |
       reinterpret_cast<uintptr_t>(workspace)) & 15)
    return invalid("q4_attn: buffers must be 16-byte aligned");
  if (!launch_fits(ctx, n_requests, max_q))
    return fail(ctx, MPIC_ERR_UNSUPPORTED, "q4_attn: too many queries, heads or requests for one launch");
  const Cut cut = cut_of(ctx, n_requests, max_q, max_len);
  if (workspace_of(ctx, cut, n_rows) > (workspace ? workspace_bytes : 0)) return invalid("q4_attn: workspace too small");
  const int rc = bind_device(ctx);
  if (rc != MPIC_OK) return rc;
  Q4AttnArgs a{};
  a.q = static_cast<const char*>(q);
  a.cache = static_cast<const char*>(cache);
  a.q_off = q_off;
  a.table = page_table;
  a.lens = lens;
  a.out = static_cast<char*>(out);
  a.lse = lse;
  a.ws_o = static_cast<float*>(workspace);
  a.ws_lse = a.ws_o + n_rows * c.n_q_heads * cut.n_splits * c.head_dim;
  a.n_rows = n_rows;
  a.q_stride = q_stride * elem;
  a.table_width = max_len > 0 ? table_width : 0;  // (there may be no table then)
  a.n_blocks = static_cast<int32_t>((n_slots + q4::kTokens - 1) / q4::kTokens);
  a.page_blocks = page_size / q4::kTokens;
  a.max_q = max_q;
  a.max_len = static_cast<int32_t>(max_len);
  a.n_splits = cut.n_splits;
  a.split_units = cut.split_units;
  a.n_q_heads = c.n_q_heads;
  a.n_kv_heads = c.n_kv_heads;
  a.group = ctx->group;
  a.scale_log2 = static_cast<float>(softmax_scale * 1.4426950408889634);
  hipStream_t stream = static_cast<hipStream_t>(stream_);
  const dim3 grid(static_cast<unsigned>(cut.tiles * c.n_kv_heads), cut.n_splits, n_requests);
  if (c.dtype == MPIC_BF16 && cut.rows == 8)
    MPIC_HIP(ctx, (launch_q4_attn<Shape<__bf16, 128, true>, 4>(a, grid, stream)));
  else if (c.dtype == MPIC_BF16 && cut.rows == 16)
    MPIC_HIP(ctx, (launch_q4_attn<Shape<__bf16, 128, false>, 3>(a, grid, stream)));
  else if (c.dtype == MPIC_BF16)
    MPIC_HIP(ctx, (launch_q4_attn<Shape<__bf16, 128, false, 2>, 2>(a, grid, stream)));
  else if (c.head_dim == 128)
    MPIC_HIP(ctx, (launch_q4_attn<Shape<float, 128, false>, 3>(a, grid, stream)));
  else
    MPIC_HIP(ctx, (launch_q4_attn<Shape<float, 64, false>, 4>(a, grid, stream)));
  if (a.n_splits > 1) {
    if (c.dtype == MPIC_BF16)
      MPIC_HIP(ctx, (launch_q4_merge<__bf16, 128>(a, n_requests, stream)));
    else if (c.head_dim == 128)
      MPIC_HIP(ctx, (launch_q4_merge<float, 128>(a, n_requests, stream)));
    else
      MPIC_HIP(ctx, (launch_q4_merge<float, 64>(a, n_requests, stream)));
  }
  return MPIC_OK;
}
