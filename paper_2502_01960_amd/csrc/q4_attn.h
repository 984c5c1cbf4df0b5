// What the kernels of attention over a cache in 4 bits share: arguments, requests, codes as matrix operands.
#pragma once

#include <algorithm>

#include "common.h"
#include "mpic_q4.h"
#include "q4.h"
#include "wave_ops.h"

namespace mpic {
namespace q4 {

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
  int32_t split_units, split_least, split_step;  // see units_of_split
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

// Units of a request's splits.  In launches of many rows that are one round of workgroups a shorter request has shorter
// splits, as many as the longest one where split_least and whole steps allow it: all end about together.  Otherwise
// (split_least = 0) all splits are as long, and shorter requests have fewer; with few rows the first table entries are asked for
// before the length is known.
__device__ inline int units_of_split(const Q4AttnArgs& a, const Request& r) {
  if (a.split_least == 0) return a.split_units;
  const int units = (r.len + kUnit - 1) / kUnit, each = (units + a.n_splits - 1) / a.n_splits;
  return max((each + a.split_step - 1) / a.split_step * a.split_step, a.split_least);
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

// Many rows per kv head (bf16): a launch whose workgroups take kManyRows flattened rows each; splits are multiples of
// kManyUnits units.
constexpr int kManyRows = 128;
constexpr int kManyUnits = 2;
hipError_t launch_q4_attn_many(const Q4AttnArgs& a, dim3 grid, hipStream_t stream);

}  // namespace q4
}  // namespace mpic
