// Attention over contexts held in 4 bits (gfx950).  Arguments and result: mpic_q4.h; layout of the cache: q4.h.
//
// With K_j = low + code * scale for every group of 64 values,
//   <q, K_j> = sum over groups of  scale_j * <q, code_j> + low_j * sum(q)
//   O        = sum_j (p_j scale_j) code_j + sum_j p_j low_j          (per group of columns)
// so both products run on the codes themselves: whole numbers below 16, exact in bf16.  A pair of codes becomes a pair of
// bf16 with one shift and one and-or, as 1 + code / 16 (the code in the upper mantissa bits of 1.0).  The ones are taken off
// again, in the first product by starting its accumulator at -sum(q), in the second by one more product with a matrix
// of ones, which sums the very weights (rounded) that met the codes.  There half the range of the codes goes too, 8 * scale
// moving to the lows with the unrounded weights: what the rounding of a weight is multiplied with is then at most
// 8 scales, not 15, and an output is off by what rounding the weights costs over a context in bf16.
//
// Transposed formulation: S^T = K Q^T, O^T = V^T P^T on 16x16x32 tiles whose columns are 16 flattened rows (query, head in
// the kv group).  A lane then holds the scores of its column for tokens 4g .. 4g + 3 of both blocks of a unit of 32 tokens,
// which is just what it has to hold of P^T for the second product: nothing crosses lanes, and since V lies in the cache
// by columns of four tokens, nothing goes through LDS either.  Softmax statistics are per lane; the reference point m of a
// column moves only when a score exceeds it by 2^8, the one case where lanes exchange it.
//
// A workgroup of four wavefronts takes a split of a request's keys for one kv head and 16 rows; its wavefronts take the
// units in turn and meet in LDS at the end.  Where the keys are cut into several splits, a second launch merges them.
// The kernel is bound by HBM bandwidth as long as enough loads are in flight: every wavefront has two units of LDS of its
// own, filled by direct global->LDS loads (five a unit, no registers, no barrier) while it works on the other one.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "common.h"
#include "mpic_q4.h"
#include "q4.h"
#include "wave_ops.h"

namespace mpic {
namespace {

using q4::Block;
using q4::kTokens;

constexpr int kWaves = 4;
constexpr int kUnit = 32;       // tokens a wavefront takes at a time: two blocks
constexpr int kCols = 16;       // flattened rows of a tile
constexpr float kSlack = 8.0f;  // a column's reference point may lag behind its greatest score by this much, log2 units

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
  int32_t n_blocks, page_blocks, max_q, max_len, n_splits, split_units, n_q_heads, n_kv_heads, group;
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

// Two codes of a word as two bf16: those in bits 4n.. and 16 + 4n..
template <bool kExact, int n>
__device__ inline uint32_t pair_of(uint32_t w) {
  if (kExact) {
    const float lo = static_cast<float>(w >> (4 * n) & 15u), hi = static_cast<float>(w >> (16 + 4 * n) & 15u);
    return __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, hi), __builtin_bit_cast(uint32_t, lo), 0x07060302u);
  }
  const uint32_t moved = n == 0 ? w << 3 : w >> (4 * n - 3);
  return (moved & 0x00780078u) | 0x3F803F80u;
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

template <typename T, int D>
struct Shape {
  using B = Block<T, D>;
  static constexpr bool kExact = std::is_same<T, float>::value;
  static constexpr int kParts = kExact ? 3 : 1;
  static constexpr int kGroups = B::kGroups;
  static constexpr int kWords = B::kLaneBytes / 4;
  static constexpr float kCode = kExact ? 1.f : 16.f;  // what a product with the codes has to be multiplied with
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
  typedef uint32_t words __attribute__((ext_vector_type(Shape<T, D>::kWords)));
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
__device__ inline void stage_1k(const char* base, uint32_t offset, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" : : "v"(offset), "s"(base), "s"(lds) : "memory", "m0");
}
__device__ inline void stage_2k(const char* base, uint32_t offset, uint32_t lds) {
  asm volatile(
      "s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1\n\tglobal_load_lds_dwordx4 %0, %1 offset:1024"
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

__device__ inline f32x4 mfma(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

// State of a column tile in one wavefront
template <typename T, int D>
struct Columns {
  using S = Shape<T, D>;
  Parts<S::kParts> q[S::kGroups][2];
  float q_sum[S::kGroups];
  f32x4 o[S::kGroups][4];  // O^T: lane (column, quarter g) holds columns 64 gr + 16 g + 4 r + tile of the output
  f32x4 ones[S::kGroups];  // sums of the rounded weights
  float low[S::kGroups];   // sum p * (low + 8 scale), F32: sum p * low; this lane's tokens
  float m, l;              // reference point (log2 units, the same in the lanes of a column), sum p of this lane's tokens
  int limit;               // positions 0 .. limit - 1 are seen
};

// One unit of 32 tokens.  kMasked: not every token is seen by every column (or a block is missing: bit of `have`).
template <typename T, int D, bool kMasked>
__device__ inline void attend_unit(Columns<T, D>& s, const char* unit, int pos, int have, int lane, float factor) {
  using S = Shape<T, D>;
  const int quarter = lane >> 4;
  float x[2][4];
#pragma unroll
  for (int b = 0; b < 2; ++b) {
    f32x4 sum = f32x4{0};
    const typename Held<T, D>::words words = codes_in<T, D, false>(unit, b, lane);
#pragma unroll
    for (int g = 0; g < S::kGroups; ++g) {
      const typename Held<T, D>::pairs pairs = pairs_in<T, D, false>(unit, b, g, quarter);
      const float start = S::kExact ? 0.f : -s.q_sum[g];
      f32x4 acc = {start, start, start, start};
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        const bf16x8 codes = keys_of<S::kExact>(words[2 * g + w]);
#pragma unroll
        for (int i = 0; i < S::kParts; ++i) acc = mfma(codes, s.q[g][w].p[i], acc);
      }
      const float base = s.q_sum[g] * (1.f / S::kCode);
#pragma unroll
      for (int r = 0; r < 4; ++r)
        sum[r] = fmaf(static_cast<float>(pairs[2 * r]), acc[r], fmaf(static_cast<float>(pairs[2 * r + 1]), base, sum[r]));
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const bool seen = !kMasked || ((have >> b & 1) && pos + kTokens * b + 4 * quarter + r < s.limit);
      x[b][r] = seen ? sum[r] : -INFINITY;
    }
  }
  float top = x[0][0];
#pragma unroll
  for (int i = 1; i < 8; ++i) top = fmaxf(top, x[i / 4][i % 4]);
  top *= factor;
  if (__any(top > s.m + kSlack)) {
    float m = fmaxf(s.m, top);
    m = fmaxf(m, __shfl_xor(m, 16));
    m = fmaxf(m, __shfl_xor(m, 32));
    const float f = m == -INFINITY ? 1.f : exp2f(s.m - m);
    s.m = m;
    s.l *= f;
#pragma unroll
    for (int g = 0; g < S::kGroups; ++g) {
      s.low[g] *= f;
      if (!S::kExact) s.ones[g] *= f;
#pragma unroll
      for (int c = 0; c < 4; ++c) s.o[g][c] *= f;
    }
  }
  const float m = s.m == -INFINITY ? 0.f : s.m;
  float p[2][4];
#pragma unroll
  for (int b = 0; b < 2; ++b)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      p[b][r] = __builtin_amdgcn_exp2f(fmaf(x[b][r], factor, -m));
      s.l += p[b][r];
    }
  const typename Held<T, D>::words v0 = codes_in<T, D, true>(unit, 0, lane), v1 = codes_in<T, D, true>(unit, 1, lane);
#pragma unroll
  for (int g = 0; g < S::kGroups; ++g) {
    f32x8 w;
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const typename Held<T, D>::pairs pairs = pairs_in<T, D, true>(unit, b, g, quarter);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        float scaled = p[b][r] * static_cast<float>(pairs[2 * r]);
        float low = p[b][r] * static_cast<float>(pairs[2 * r + 1]);
        if (kMasked && x[b][r] == -INFINITY) scaled = low = 0.f;  // (what is not seen may be no number)
        w[4 * b + (r & 1) * 2 + (r >> 1)] = scaled;               // tokens (0, 2), (1, 3)
        s.low[g] += S::kExact ? low : fmaf(8.f, scaled, low);
      }
    }
    const Parts<S::kParts> weights = split_parts<S::kParts>(w);
#pragma unroll
    for (int i = 0; i < S::kParts; ++i) {
      if (!S::kExact) {
        const u32x4 one = {0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u};
        s.ones[g] = mfma(__builtin_bit_cast(bf16x8, one), weights.p[i], s.ones[g]);
      }
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        s.o[g][2 * c] = mfma(values_of<S::kExact, 0>(v0[2 * g + c], v1[2 * g + c]), weights.p[i], s.o[g][2 * c]);
        s.o[g][2 * c + 1] = mfma(values_of<S::kExact, 1>(v0[2 * g + c], v1[2 * g + c]), weights.p[i], s.o[g][2 * c + 1]);
      }
    }
  }
}

// LDS: the units of every wavefront; at the end their partial results (rows of D + 4 floats, reference points, sums)
template <typename T, int D>
struct AttnLds {
  static constexpr int kRow = D + 4;
  static constexpr int kWave = 2 * Unit<T, D>::kBytes;
  static constexpr int kParts = kWaves * kCols * (kRow + 2) * 4;
  static constexpr int kBytes = kWaves * kWave > kParts ? kWaves * kWave : kParts;
  static_assert(kBytes <= 65536, "no opt-in needed");
};

template <typename T, int D>
__global__ __launch_bounds__(kWaves * 64, sizeof(T) == 2 ? 3 : 2) void q4_attn_kernel(Q4AttnArgs a) {
  using S = Shape<T, D>;
  using B = Block<T, D>;
  using L = AttnLds<T, D>;
  using U = Unit<T, D>;
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  typedef float PartRows[kCols][L::kRow];
  typedef float PartCols[kCols];
  PartRows* part_o = reinterpret_cast<PartRows*>(lds);
  PartCols* part_m = reinterpret_cast<PartCols*>(part_o + kWaves);
  PartCols* part_l = part_m + kWaves;
  const int lane = threadIdx.x & 63, col = lane & 15, quarter = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int split = blockIdx.x, head = blockIdx.y % a.n_kv_heads, b = blockIdx.z;
  const int row0 = static_cast<int>(blockIdx.y) / a.n_kv_heads * kCols;
  const Request rq = request_of(a, b);
  const int n_flat = rq.n * a.group;
  if (row0 >= n_flat) return;
  const int last = (min(row0 + kCols, n_flat) - 1) / a.group;  // last query of the tile
  const int behind = rq.len - rq.n;                            // tokens in front of the new ones (negative: some have no position)
  const int key_end = max(behind + last + 1, 0);
  const int key_all = behind + row0 / a.group + 1;             // the keys below are seen by every row

  Columns<T, D> s;
  const int flat = min(row0 + col, n_flat - 1), token = flat / a.group, hq = head * a.group + flat % a.group;
  s.limit = row0 + col < n_flat ? behind + token + 1 : 0;
  s.m = -INFINITY;
  s.l = 0.f;
  {
    const char* q = a.q + (rq.first + token) * a.q_stride + static_cast<int64_t>(hq) * D * sizeof(T);
#pragma unroll
    for (int g = 0; g < S::kGroups; ++g) {
      s.q_sum[g] = 0.f;
      s.low[g] = 0.f;
      s.ones[g] = f32x4{0};
#pragma unroll
      for (int c = 0; c < 4; ++c) s.o[g][c] = f32x4{0};
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        typedef T vec __attribute__((ext_vector_type(8), aligned(16)));
        f32x8 x = __builtin_convertvector(*reinterpret_cast<const vec*>(q + (g * q4::kGroup + quarter * 16 + w * 8) * sizeof(T)), f32x8);
        s.q[g][w] = split_parts<S::kParts>(x);
#pragma unroll
        for (int e = 0; e < 8; ++e) s.q_sum[g] += x[e];
      }
      s.q_sum[g] += __shfl_xor(s.q_sum[g], 16);
      s.q_sum[g] += __shfl_xor(s.q_sum[g], 32);
    }
  }
  const float factor = a.scale_log2 * S::kCode;
  const int unit_end = min((key_end + kUnit - 1) / kUnit, (split + 1) * a.split_units);
  const int unit0 = split * a.split_units + wave;
  const int n_units = unit_end > unit0 ? (unit_end - unit0 + kWaves - 1) / kWaves : 0;  // of this wavefront
  const int32_t* table = a.table + b * a.table_width;
  // blocks of the next 32 units, two lanes a unit; -1: not in the cache
  int ids = -1;
  auto look_up = [&](int i0) {
    const int block = 2 * (unit0 + (i0 + (lane >> 1)) * kWaves) + (lane & 1);
    ids = -1;
    if (block < (key_end + kTokens - 1) / kTokens) {
      const int64_t id = static_cast<int64_t>(table[block / a.page_blocks]) * a.page_blocks + block % a.page_blocks;
      if (id >= 0 && id < a.n_blocks) ids = static_cast<int>(id);
    }
  };
  char* ring = lds + wave * L::kWave;
  const uint32_t ring_lds = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(MPIC_LDS_PTR(char, ring)));
  // load unit i of this wavefront into its half of the ring; bit b of the result: block b is in the cache
  auto stage = [&](int i) {
    if ((i & 31) == 0) look_up(i);
    const int id0 = __builtin_amdgcn_readlane(ids, 2 * i & 63), id1 = __builtin_amdgcn_readlane(ids, (2 * i & 63) + 1);
    const char* base = a.cache + static_cast<int64_t>(head) * B::kBytes;
    const int64_t pitch = static_cast<int64_t>(a.n_kv_heads) * B::kBytes;
    stage_unit<T, D>(base + max(id0, 0) * pitch, base + max(id1, 0) * pitch, lane, ring_lds + (i & 1) * U::kBytes);
    return (id0 >= 0 ? 1 : 0) | (id1 >= 0 ? 2 : 0);
  };
  int have = 0;
  if (n_units > 0) have = stage(0);
  for (int i = 0; i < n_units; ++i) {
    int have_next = 0;
    if (i + 1 < n_units) {
      have_next = stage(i + 1);
      MPIC_WAIT_VMCNT(U::kLoads);
    } else {
      MPIC_WAIT_VMCNT(0);
    }
    asm volatile("" ::: "memory");
    const char* unit = ring + (i & 1) * U::kBytes;
    const int pos = (unit0 + i * kWaves) * kUnit;
    if (have == 3 && pos + kUnit <= key_all)
      attend_unit<T, D, false>(s, unit, pos, have, lane, factor);
    else
      attend_unit<T, D, true>(s, unit, pos, have, lane, factor);
    have = have_next;
  }
  __syncthreads();

  s.l += __shfl_xor(s.l, 16);
  s.l += __shfl_xor(s.l, 32);
  if (quarter == 0) {
    part_m[wave][col] = s.m;
    part_l[wave][col] = s.l;
  }
#pragma unroll
  for (int g = 0; g < S::kGroups; ++g) {
    s.low[g] += __shfl_xor(s.low[g], 16);
    s.low[g] += __shfl_xor(s.low[g], 32);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      f32x4 o;
#pragma unroll
      for (int c = 0; c < 4; ++c) o[c] = S::kExact ? s.o[g][c][r] + s.low[g] : fmaf(fmaf(-1.5f, s.ones[g][r], s.o[g][c][r]), S::kCode, s.low[g]);
      *reinterpret_cast<f32x4*>(&part_o[wave][col][g * q4::kGroup + quarter * 16 + 4 * r]) = o;
    }
  }
  __syncthreads();

  constexpr int kEach = D / 16;  // values of a row per thread
  const int c = threadIdx.x / 16, d0 = threadIdx.x % 16 * kEach;
  if (row0 + c >= n_flat) return;
  float top = part_m[0][c];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) top = fmaxf(top, part_m[w][c]);
  float z = 0.f, o[kEach] = {};
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    // (a wavefront that saw nothing, or nothing but what is no number, adds its sums as they are)
    const float f = part_m[w][c] == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(part_m[w][c] - top);
    z = fmaf(f, part_l[w][c], z);
#pragma unroll
    for (int e = 0; e < kEach; ++e) o[e] = fmaf(f, part_o[w][c][d0 + e], o[e]);
  }
  const bool none = z == 0.f;
  const float inv = none ? 0.f : 1.f / z, lse2 = none ? -INFINITY : (top == -INFINITY ? z : top + log2f(z));
  const int64_t row = (rq.first + (row0 + c) / a.group) * a.n_q_heads + head * a.group + (row0 + c) % a.group;
  if (a.n_splits > 1) {
    const int64_t at = row * a.n_splits + split;
    if (threadIdx.x % 16 == 0) a.ws_lse[at] = lse2;
    if (!none)
#pragma unroll
      for (int e = 0; e < kEach; e += 4) *reinterpret_cast<f32x4*>(a.ws_o + at * D + d0 + e) = f32x4{o[e] * inv, o[e + 1] * inv, o[e + 2] * inv, o[e + 3] * inv};
    return;
  }
  typedef T vec __attribute__((ext_vector_type(4)));
#pragma unroll
  for (int e = 0; e < kEach; e += 4)
    *reinterpret_cast<vec*>(a.out + (row * D + d0 + e) * sizeof(T)) =
        __builtin_convertvector((f32x4{o[e] * inv, o[e + 1] * inv, o[e + 2] * inv, o[e + 3] * inv}), vec);
  if (a.lse && threadIdx.x % 16 == 0) a.lse[row] = lse2 * 0.6931471805599453f;
}

// Output rows from the partial results of their splits.  A workgroup takes a row: D / 4 threads hold four columns each, and
// 256 / (D / 4) of them share the splits, in a fixed order.
template <typename T, int D>
__global__ __launch_bounds__(256) void q4_merge_kernel(Q4AttnArgs a) {
  constexpr int kLanes = D / 4, kShares = 256 / kLanes;
  __shared__ __attribute__((aligned(16))) float sums[kShares][D];
  __shared__ float tops[kShares], zs[kShares];
  const Request rq = request_of(a, blockIdx.y);
  const int64_t i = blockIdx.x;
  if (i >= static_cast<int64_t>(rq.n) * a.n_q_heads) return;  // (the whole workgroup)
  const int64_t row = rq.first * a.n_q_heads + i;
  const int lane = threadIdx.x % kLanes, share = threadIdx.x / kLanes;
  const float* part = a.ws_lse + row * a.n_splits;
  // every thread finds the greatest of its share's log-sum-exps; what is no number makes z no number
  float top = -INFINITY;
  for (int s = share; s < a.n_splits; s += kShares) top = fmaxf(top, part[s]);
  float z = 0.f;
  f32x4 o = f32x4{0};
#pragma unroll 4
  for (int s = share; s < a.n_splits; s += kShares) {
    const float lse = part[s];
    if (lse == -INFINITY) continue;  // (its output is not written)
    const float f = __builtin_amdgcn_exp2f(lse - (top == -INFINITY ? 0.f : top));
    z += f;
    o += *reinterpret_cast<const f32x4*>(a.ws_o + (row * a.n_splits + s) * D + 4 * lane) * f;
  }
  *reinterpret_cast<f32x4*>(&sums[share][4 * lane]) = o;
  if (lane == 0) {
    tops[share] = top;
    zs[share] = z;
  }
  __syncthreads();
  if (threadIdx.x >= kLanes) return;
  top = tops[0];
#pragma unroll
  for (int k = 1; k < kShares; ++k) top = fmaxf(top, tops[k]);
  z = 0.f;
  o = f32x4{0};
#pragma unroll
  for (int k = 0; k < kShares; ++k) {
    const float f = tops[k] == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(tops[k] - top);
    z = fmaf(f, zs[k], z);
    o += *reinterpret_cast<const f32x4*>(&sums[k][4 * lane]) * f;
  }
  const float inv = z == 0.f ? 0.f : 1.f / z;
  typedef T vec __attribute__((ext_vector_type(4)));
  *reinterpret_cast<vec*>(a.out + (row * D + 4 * lane) * sizeof(T)) = __builtin_convertvector(o * inv, vec);
  if (a.lse && lane == 0) a.lse[row] = z == 0.f ? -INFINITY : (top == -INFINITY ? z : top + log2f(z)) * 0.6931471805599453f;
}

// How the keys are cut: into splits of whole units for every wavefront, so that one round of workgroups covers the chip where
// the requests alone do not, but no less than two units a wavefront.  Lengths differ, and a launch is over when its longest
// split is: splits are cut down to 32 units as long as that makes no more than eight rounds of them.
struct Cut {
  int32_t n_splits, split_units;
};
Cut cut_of(const mpic_ctx* ctx, int32_t n_requests, int32_t max_q, int64_t max_len) {
  constexpr int64_t kRound = 1024, kRounds = 8, kLeast = 2 * kWaves, kMost = 32;
  const int64_t units = std::max<int64_t>(1, (max_len + kUnit - 1) / kUnit);
  const int64_t tiles = (static_cast<int64_t>(max_q) * ctx->group + kCols - 1) / kCols;
  const int64_t lanes = tiles * ctx->cfg.n_kv_heads * n_requests;
  const auto units_of = [&](int64_t workgroups) {  // a split's, for that many workgroups at most
    const int64_t splits = std::max<int64_t>(1, workgroups / lanes);
    return ((units + splits - 1) / splits + kWaves - 1) / kWaves * kWaves;
  };
  const int64_t each = std::max(kLeast, std::min(units_of(kRound), std::max(kMost, units_of(kRounds * kRound))));
  return Cut{static_cast<int32_t>((units + each - 1) / each), static_cast<int32_t>(each)};
}
bool sizes_fit(const mpic_ctx* ctx, int32_t n_requests, int64_t n_rows, int32_t max_q, int64_t max_len) {
  return n_requests >= 0 && n_rows >= 0 && max_q >= 1 && max_len >= 0 && n_rows < INT32_MAX && max_len <= INT32_MAX - 64 &&
         static_cast<int64_t>(max_q) * ctx->group < INT32_MAX - kCols;
}
int64_t workspace_of(const mpic_ctx* ctx, const Cut& cut, int64_t n_rows) {
  return cut.n_splits > 1 ? n_rows * ctx->cfg.n_q_heads * cut.n_splits * (ctx->cfg.head_dim + 1) * 4 : 0;
}

template <typename T, int D>
void launch_q4_attn(const Q4AttnArgs& a, dim3 grid, int32_t n_requests, hipStream_t stream) {
  hipLaunchKernelGGL((q4_attn_kernel<T, D>), grid, dim3(kWaves * 64), (AttnLds<T, D>::kBytes), stream, a);
  if (a.n_splits > 1) {
    hipLaunchKernelGGL((q4_merge_kernel<T, D>), dim3(static_cast<unsigned>(a.max_q) * a.n_q_heads, n_requests), dim3(256), 0, stream, a);
  }
}

}  // namespace
}  // namespace mpic

extern "C" int mpic_q4_attn_workspace(const mpic_ctx* ctx, int32_t n_requests, int64_t n_rows, int32_t max_q, int64_t max_len,
                                      int64_t* bytes) {
  if (!ctx || !bytes || !mpic::sizes_fit(ctx, n_requests, n_rows, max_q, max_len)) return MPIC_ERR_INVALID;
  *bytes = n_requests == 0 ? 0 : mpic::workspace_of(ctx, mpic::cut_of(ctx, n_requests, max_q, max_len), n_rows);
  return MPIC_OK;
}

extern "C" int mpic_q4_attn(mpic_ctx* ctx, const void* q, int64_t q_stride, int64_t n_rows, const int32_t* q_off, int32_t max_q,
                            const void* cache, int64_t n_slots, const int32_t* page_table, int64_t table_width,
                            int32_t page_size, const int32_t* lens, int32_t n_requests, int64_t max_len, double softmax_scale,
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
  if (!(softmax_scale > 0.0) || !std::isfinite(softmax_scale)) return invalid("q4_attn: softmax_scale must be finite and positive");
  if (q_stride < static_cast<int64_t>(c.n_q_heads) * c.head_dim || q_stride * elem % 16)
    return invalid("q4_attn: q_stride must hold a row and be a multiple of 16 bytes");
  if (n_rows == 0 || n_requests == 0) return MPIC_OK;
  if (!q || !cache || !lens || !out || (max_len > 0 && !page_table)) return invalid("q4_attn: null buffer");
  if (max_len > 0 && n_slots == 0) return invalid("q4_attn: a cache without slots");
  if ((reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(cache) | reinterpret_cast<uintptr_t>(out) |
       reinterpret_cast<uintptr_t>(workspace)) & 15)
    return invalid("q4_attn: buffers must be 16-byte aligned");
  const Cut cut = cut_of(ctx, n_requests, max_q, max_len);
  if (workspace_of(ctx, cut, n_rows) > (workspace ? workspace_bytes : 0)) return invalid("q4_attn: workspace too small");
  const int64_t tiles = (static_cast<int64_t>(max_q) * ctx->group + kCols - 1) / kCols;
  if (tiles * c.n_kv_heads > 65535 || n_requests > 65535)
    return fail(ctx, MPIC_ERR_UNSUPPORTED, "q4_attn: too many queries, heads or requests for one launch");
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
  a.table_width = table_width;
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
  const dim3 grid(cut.n_splits, static_cast<unsigned>(tiles * c.n_kv_heads), n_requests);
  if (c.dtype == MPIC_BF16)
    launch_q4_attn<__bf16, 128>(a, grid, n_requests, stream);
  else if (c.head_dim == 128)
    launch_q4_attn<float, 128>(a, grid, n_requests, stream);
  else
    launch_q4_attn<float, 64>(a, grid, n_requests, stream);
  MPIC_HIP(ctx, hipGetLastError());
  return MPIC_OK;
}
