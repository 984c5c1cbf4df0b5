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

// What a lane holds of a block: codes, and the pairs of its four tokens
template <typename T, int D>
struct Held {
  typedef uint32_t words __attribute__((ext_vector_type(Shape<T, D>::kWords)));
  typedef T pairs __attribute__((ext_vector_type(8)));  // scale, low of four tokens
  words k, v;
  pairs kp[Shape<T, D>::kGroups], vp[Shape<T, D>::kGroups];
};
template <typename T, int D>
__device__ inline Held<T, D> load_block(const char* block, int lane) {
  using B = Block<T, D>;
  using H = Held<T, D>;
  H h;
  h.k = *reinterpret_cast<const typename H::words*>(block + ((lane & 15) * 4 + (lane >> 4)) * B::kLaneBytes);
  h.v = *reinterpret_cast<const typename H::words*>(block + B::kV + lane * B::kLaneBytes);
#pragma unroll
  for (int g = 0; g < B::kGroups; ++g) {
    h.kp[g] = *reinterpret_cast<const typename H::pairs*>(block + B::kKPairs + (g * kTokens + 4 * (lane >> 4)) * B::kPair);
    h.vp[g] = *reinterpret_cast<const typename H::pairs*>(block + B::kVPairs + (g * kTokens + 4 * (lane >> 4)) * B::kPair);
  }
  return h;
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
__device__ inline void attend_unit(Columns<T, D>& s, const Held<T, D> (&h)[2], int pos, int have, int quarter, float factor) {
  using S = Shape<T, D>;
  float x[2][4];
#pragma unroll
  for (int b = 0; b < 2; ++b) {
    f32x4 sum = f32x4{0};
#pragma unroll
    for (int g = 0; g < S::kGroups; ++g) {
      const float start = S::kExact ? 0.f : -s.q_sum[g];
      f32x4 acc = {start, start, start, start};
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        const bf16x8 codes = keys_of<S::kExact>(h[b].k[2 * g + w]);
#pragma unroll
        for (int i = 0; i < S::kParts; ++i) acc = mfma(codes, s.q[g][w].p[i], acc);
      }
      const float base = s.q_sum[g] * (1.f / S::kCode);
#pragma unroll
      for (int r = 0; r < 4; ++r)
        sum[r] = fmaf(static_cast<float>(h[b].kp[g][2 * r]), acc[r], fmaf(static_cast<float>(h[b].kp[g][2 * r + 1]), base, sum[r]));
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
#pragma unroll
  for (int g = 0; g < S::kGroups; ++g) {
    f32x8 w;
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        float scaled = p[b][r] * static_cast<float>(h[b].vp[g][2 * r]);
        float low = p[b][r] * static_cast<float>(h[b].vp[g][2 * r + 1]);
        if (kMasked && x[b][r] == -INFINITY) scaled = low = 0.f;  // (what is not seen may be no number)
        w[4 * b + (r & 1) * 2 + (r >> 1)] = scaled;               // tokens (0, 2), (1, 3)
        s.low[g] += S::kExact ? low : fmaf(8.f, scaled, low);
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
        s.o[g][2 * c] = mfma(values_of<S::kExact, 0>(h[0].v[2 * g + c], h[1].v[2 * g + c]), weights.p[i], s.o[g][2 * c]);
        s.o[g][2 * c + 1] = mfma(values_of<S::kExact, 1>(h[0].v[2 * g + c], h[1].v[2 * g + c]), weights.p[i], s.o[g][2 * c + 1]);
      }
    }
  }
}

template <typename T, int D>
__global__ __launch_bounds__(kWaves * 64) void q4_attn_kernel(Q4AttnArgs a) {
  using S = Shape<T, D>;
  using B = Block<T, D>;
  constexpr int kRow = D + 4;  // floats of a row of partial outputs in LDS
  __shared__ __attribute__((aligned(16))) float part_o[kWaves][kCols][kRow];
  __shared__ float part_m[kWaves][kCols], part_l[kWaves][kCols];
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
  auto fetch = [&](int i, Held<T, D>(&h)[2], int* have) {
    *have = 0;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int id = __builtin_amdgcn_readlane(ids, (2 * i & 63) + k);
      *have |= (id >= 0) << k;
      h[k] = load_block<T, D>(a.cache + (static_cast<int64_t>(max(id, 0)) * a.n_kv_heads + head) * B::kBytes, lane);
    }
  };
  for (int i = 0; i < n_units; ++i) {
    if ((i & 31) == 0) look_up(i);
    Held<T, D> h[2];
    int have;
    fetch(i, h, &have);
    const int pos = (unit0 + i * kWaves) * kUnit;
    if (have == 3 && pos + kUnit <= key_all)
      attend_unit<T, D, false>(s, h, pos, have, quarter, factor);
    else
      attend_unit<T, D, true>(s, h, pos, have, quarter, factor);
  }

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

// Output rows from the partial results of their splits: D / 4 threads a row, the splits in their order.
template <typename T, int D>
__global__ __launch_bounds__(256) void q4_merge_kernel(Q4AttnArgs a) {
  constexpr int kLanes = D / 4;
  const Request rq = request_of(a, blockIdx.y);
  const int64_t i = static_cast<int64_t>(blockIdx.x) * (256 / kLanes) + threadIdx.x / kLanes;
  if (i >= static_cast<int64_t>(rq.n) * a.n_q_heads) return;
  const int64_t row = rq.first * a.n_q_heads + i;
  const int d0 = threadIdx.x % kLanes * 4;
  const float* part = a.ws_lse + row * a.n_splits;
  float top = -INFINITY;
  bool nan = false;
  for (int s = 0; s < a.n_splits; ++s) {
    top = fmaxf(top, part[s]);
    nan |= part[s] != part[s];
  }
  float z = 0.f;
  f32x4 o = f32x4{0};
  if (top != -INFINITY)
    for (int s = 0; s < a.n_splits; ++s) {
      if (part[s] == -INFINITY) continue;
      const float f = __builtin_amdgcn_exp2f(part[s] - top);
      z += f;
      o += *reinterpret_cast<const f32x4*>(a.ws_o + (row * a.n_splits + s) * D + d0) * f;
    }
  const float inv = z == 0.f ? 0.f : 1.f / z;
  o = nan ? f32x4{NAN, NAN, NAN, NAN} : o * inv;
  typedef T vec __attribute__((ext_vector_type(4)));
  *reinterpret_cast<vec*>(a.out + (row * D + d0) * sizeof(T)) = __builtin_convertvector(o, vec);
  if (a.lse && d0 == 0) a.lse[row] = nan ? NAN : z == 0.f ? -INFINITY : (top + log2f(z)) * 0.6931471805599453f;
}

// How the keys are cut: into splits of whole units for every wavefront, so that the launch has some 1024 workgroups
// (four a compute unit) where the requests alone do not supply them, but no less than two units a wavefront.
struct Cut {
  int32_t n_splits, split_units;
};
Cut cut_of(const mpic_ctx* ctx, int32_t n_requests, int32_t max_q, int64_t max_len) {
  constexpr int64_t kWorkgroups = 1024, kLeast = 2 * kWaves;
  const int64_t units = std::max<int64_t>(1, (max_len + kUnit - 1) / kUnit);
  const int64_t tiles = (static_cast<int64_t>(max_q) * ctx->group + kCols - 1) / kCols;
  const int64_t lanes = tiles * ctx->cfg.n_kv_heads * n_requests;
  const int64_t want = std::min(std::max<int64_t>(1, kWorkgroups / lanes), (units + kLeast - 1) / kLeast);
  const int64_t each = ((units + want - 1) / want + kWaves - 1) / kWaves * kWaves;
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
  hipLaunchKernelGGL((q4_attn_kernel<T, D>), grid, dim3(kWaves * 64), 0, stream, a);
  if (a.n_splits > 1) {
    const int64_t rows = static_cast<int64_t>(a.max_q) * a.n_q_heads, each = 256 / (D / 4);
    hipLaunchKernelGGL((q4_merge_kernel<T, D>), dim3(static_cast<unsigned>((rows + each - 1) / each), n_requests), dim3(256), 0, stream, a);
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
