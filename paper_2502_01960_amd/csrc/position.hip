// Fresh rows on their way into a context: norms of the query and key heads and the rotation to the rows' positions,
// on one or several axes, in one pass (gfx950).
//
//   y = x * rsqrt(mean(x^2) + eps) * w,   pair i of y turned by pos[axis(i)] * theta^(-2i/D)
//
// The kernel reads and writes every row once and is bound by HBM bandwidth (some 10 operations per value).  Angles:
// the turn per position of pair i is a 64-bit fraction F_i = theta^(-2i/D) / 2 pi * 2^64 from the host; pos * F_i
// modulo 2^64 is the angle modulo a full turn, exact to 2^-33 of a turn for any int32 position, where an fp32 product is off
// by 5e-3 radians at 75K tokens already.  Its two leading bits are the quadrant, the rest goes through the Taylor
// series of sine and cosine on [-pi/4, pi/4] (next terms below 2e-9).
#include <algorithm>
#include <cfloat>
#include <cmath>

#include "common.h"
#include "wave_ops.h"
#include "mpic_q4.h"

namespace mpic {
namespace {

constexpr int kMaxPairs = 64;

struct PositionArgs {
  const void* q;
  const void* k;
  void* q_out;
  void* k_out;
  const void* q_weight;
  const void* k_weight;
  const int32_t* pos;
  int64_t n_rows, q_stride, k_stride, q_out_stride, k_out_stride;  // strides in elements
  int32_t n_q_heads, n_heads;                                      // query heads, query and key heads
  float eps;
  uint64_t axis_bits[2];        // two bits a pair
  uint64_t turn[kMaxPairs];     // F_i
};

__device__ inline void sincos_turn(uint64_t phase, float* s, float* c) {
  const uint32_t top = static_cast<uint32_t>(phase >> 32);
  const uint32_t quadrant = (top + 0x20000000u) >> 30;
  const float x = static_cast<float>(static_cast<int32_t>(top - (quadrant << 30))) * (6.283185307179586f / 4294967296.f);
  const float u = x * x;
  const float sx = x * fmaf(u, fmaf(u, fmaf(u, fmaf(u, 1.f / 362880.f, -1.f / 5040.f), 1.f / 120.f), -1.f / 6.f), 1.f);
  const float cx = fmaf(u, fmaf(u, fmaf(u, fmaf(u, fmaf(u, -1.f / 3628800.f, 1.f / 40320.f), -1.f / 720.f), 1.f / 24.f), -0.5f), 1.f);
  const float a = quadrant & 1 ? cx : sx, b = quadrant & 1 ? sx : cx;
  *s = quadrant & 2 ? -a : a;
  *c = (quadrant + 1) & 2 ? -b : b;
}

// One wavefront per row and part: its lanes hold the heads of the part, kLanes lanes a head, each with 16 bytes of the
// head's first half and 16 of its second (rotate-half pairs lie in one lane then, neighbouring pairs in any case).  What
// depends on the row and the pair only, the sines and cosines, is computed once for all heads of the part.  Rows are read with
// streaming loads (7680 rows of 32 heads 31.0 -> 28.3 us, 4.45 TB/s) and stored the ordinary way for whoever reads them next.
template <typename T, int D, bool kInterleaved, bool kNorm>
__global__ __launch_bounds__(256) void position_kernel(PositionArgs a, int heads_per_part) {
  constexpr int V = 16 / sizeof(T);  // values per 16 bytes
  constexpr int kLanes = D / (2 * V);
  constexpr int kHeads = 64 / kLanes;  // heads a wavefront takes at a time
  typedef T vec __attribute__((ext_vector_type(V)));
  typedef float fvec __attribute__((ext_vector_type(V)));
  const int lane = threadIdx.x & 63;
  const int64_t row = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6);
  if (row >= a.n_rows) return;
  const int part = lane % kLanes, sub = lane / kLanes;

  float sn[V], cs[V];
#pragma unroll
  for (int e = 0; e < V; ++e) {
    // pair of values 2 e', 2 e' + 1 of the lane's two runs, or of value e of both
    const int pair = kInterleaved ? (e < V / 2 ? part * (V / 2) + e : D / 4 + part * (V / 2) + e - V / 2) : part * V + e;
    const int axis = static_cast<int>(a.axis_bits[pair >> 5] >> (2 * (pair & 31))) & 3;
    const int32_t p = a.pos[axis * a.n_rows + row];
    sincos_turn(static_cast<uint64_t>(static_cast<int64_t>(p)) * a.turn[pair], &sn[e], &cs[e]);
  }
  const int first = blockIdx.y * heads_per_part, last = min(first + heads_per_part, a.n_heads);
  for (int h0 = first; h0 < last; h0 += kHeads) {
    const int h = h0 + sub;
    const bool is_q = h < a.n_q_heads;
    const int hh = is_q ? h : h - a.n_q_heads;
    if (h >= last) continue;  // (whole heads leave: the lanes of a head agree)
    const T* src = static_cast<const T*>(is_q ? a.q : a.k) + row * (is_q ? a.q_stride : a.k_stride) + hh * D;
    T* dst = static_cast<T*>(is_q ? a.q_out : a.k_out) + row * (is_q ? a.q_out_stride : a.k_out_stride) + hh * D;
    fvec lo = __builtin_convertvector(__builtin_nontemporal_load(reinterpret_cast<const vec*>(src + part * V)), fvec);
    fvec hi = __builtin_convertvector(__builtin_nontemporal_load(reinterpret_cast<const vec*>(src + D / 2 + part * V)), fvec);
    if (kNorm) {
      float sq = 0.f;
#pragma unroll
      for (int e = 0; e < V; ++e) sq = fmaf(lo[e], lo[e], fmaf(hi[e], hi[e], sq));
#pragma unroll
      for (int off = kLanes / 2; off > 0; off >>= 1) sq += __shfl_xor(sq, off);
      const float r = 1.f / sqrtf(sq * (1.f / D) + a.eps);
      const T* w = static_cast<const T*>(is_q ? a.q_weight : a.k_weight);
      lo *= r;
      hi *= r;
      if (w) {
        lo *= __builtin_convertvector(*reinterpret_cast<const vec*>(w + part * V), fvec);
        hi *= __builtin_convertvector(*reinterpret_cast<const vec*>(w + D / 2 + part * V), fvec);
      }
    }
    fvec olo, ohi;
    if (kInterleaved) {
#pragma unroll
      for (int e = 0; e < V / 2; ++e) {
        olo[2 * e] = lo[2 * e] * cs[e] - lo[2 * e + 1] * sn[e];
        olo[2 * e + 1] = lo[2 * e] * sn[e] + lo[2 * e + 1] * cs[e];
        ohi[2 * e] = hi[2 * e] * cs[V / 2 + e] - hi[2 * e + 1] * sn[V / 2 + e];
        ohi[2 * e + 1] = hi[2 * e] * sn[V / 2 + e] + hi[2 * e + 1] * cs[V / 2 + e];
      }
    } else {
#pragma unroll
      for (int e = 0; e < V; ++e) {
        olo[e] = lo[e] * cs[e] - hi[e] * sn[e];
        ohi[e] = lo[e] * sn[e] + hi[e] * cs[e];
      }
    }
    *reinterpret_cast<vec*>(dst + part * V) = __builtin_convertvector(olo, vec);
    *reinterpret_cast<vec*>(dst + D / 2 + part * V) = __builtin_convertvector(ohi, vec);
  }
}

// Workgroups and heads of a wavefront.  Few rows: their heads are spread over more wavefronts.
struct Spread {
  int64_t blocks, parts;
  int heads;
};
Spread spread_of(int64_t n_rows, int64_t n_heads, int head_bytes) {
  const int at_a_time = 64 / (head_bytes / 32);
  const int64_t blocks = (n_rows + 3) / 4, steps = (n_heads + at_a_time - 1) / at_a_time;
  const int64_t per_part = blocks >= 1024 ? steps : 1;
  return {blocks, (steps + per_part - 1) / per_part, static_cast<int>(per_part * at_a_time)};
}

template <typename T, int D>
void launch_position(const PositionArgs& a, bool interleaved, bool norm, hipStream_t stream) {
  const Spread s = spread_of(a.n_rows, a.n_heads, D * static_cast<int>(sizeof(T)));
  const dim3 grid(static_cast<unsigned>(s.blocks), static_cast<unsigned>(s.parts));
  const int heads = s.heads;
  auto go = [&](auto i, auto n) {
    hipLaunchKernelGGL((position_kernel<T, D, decltype(i)::value, decltype(n)::value>), grid, dim3(256), 0, stream, a, heads);
  };
  auto with_norm = [&](auto i) {
    if (norm)
      go(i, std::true_type{});
    else
      go(i, std::false_type{});
  };
  if (interleaved)
    with_norm(std::true_type{});
  else
    with_norm(std::false_type{});
}

bool misaligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) != 0; }

}  // namespace
}  // namespace mpic

extern "C" int mpic_position_rows(mpic_ctx* ctx, const void* q, int64_t q_stride, const void* k, int64_t k_stride,
                                  int64_t n_rows, const int32_t* pos, int32_t n_axes, const int32_t* pair_axis,
                                  const void* q_weight, const void* k_weight, double eps, void* q_out,
                                  int64_t q_out_stride, void* k_out, int64_t k_out_stride, void* stream_) {
  using namespace mpic;
  if (!ctx) return MPIC_ERR_INVALID;
  const mpic_config& c = ctx->cfg;
  const int half = c.head_dim / 2;
  const int64_t unit = c.dtype == MPIC_F32 ? 4 : 8;
  if (n_rows < 0 || n_rows >= INT32_MAX) return fail(ctx, MPIC_ERR_INVALID, "position_rows: bad row count");
  if (n_axes < 1 || n_axes > 4) return fail(ctx, MPIC_ERR_INVALID, "position_rows: n_axes must be 1 to 4");
  if (!std::isfinite(eps)) return fail(ctx, MPIC_ERR_INVALID, "position_rows: eps must be finite");
  if (eps < 0 && (q_weight || k_weight)) return fail(ctx, MPIC_ERR_INVALID, "position_rows: weights without norms (eps < 0)");
  PositionArgs a{};
  if (pair_axis)
    for (int i = 0; i < half; ++i) {
      if (pair_axis[i] < 0 || pair_axis[i] >= n_axes) return fail(ctx, MPIC_ERR_INVALID, "position_rows: pair_axis names no axis");
      a.axis_bits[i >> 5] |= static_cast<uint64_t>(pair_axis[i]) << (2 * (i & 31));
    }
  const int64_t q_row = static_cast<int64_t>(c.n_q_heads) * c.head_dim, k_row = static_cast<int64_t>(c.n_kv_heads) * c.head_dim;
  if (q_stride < q_row || q_out_stride < q_row || k_stride < k_row || k_out_stride < k_row ||
      q_stride % unit || q_out_stride % unit || k_stride % unit || k_out_stride % unit)
    return fail(ctx, MPIC_ERR_INVALID, "position_rows: strides must hold a row and be multiples of 16 bytes");
  if (n_rows == 0) return MPIC_OK;
  if (!q || !k || !pos || !q_out || !k_out) return fail(ctx, MPIC_ERR_INVALID, "position_rows: null buffer");
  if (misaligned(q) || misaligned(k) || misaligned(q_out) || misaligned(k_out) || misaligned(q_weight) || misaligned(k_weight))
    return fail(ctx, MPIC_ERR_INVALID, "position_rows: buffers must be 16-byte aligned");
  if ((q == q_out && q_stride != q_out_stride) || (k == k_out && k_stride != k_out_stride))
    return fail(ctx, MPIC_ERR_INVALID, "position_rows: rows positioned in place must keep their stride");
  // (threads of a launch, its second dimension, head counts in the kernel)
  const int64_t n_heads = static_cast<int64_t>(c.n_q_heads) + c.n_kv_heads;
  if (n_rows > INT32_MAX / 64 || n_heads > INT32_MAX / 128 || spread_of(n_rows, n_heads, c.head_dim * (c.dtype == MPIC_F32 ? 4 : 2)).parts > 65535)
    return fail(ctx, MPIC_ERR_UNSUPPORTED, "position_rows: too many rows or heads for one launch");
  const int rc = bind_device(ctx);
  if (rc != MPIC_OK) return rc;
  if (!ctx->turns_known) {
    for (int i = 0; i < half; ++i) {
      // positions are whole numbers, so whole turns per position can go
      const long double per = std::pow(static_cast<long double>(c.rope_theta), -2.0L * i / c.head_dim) / 6.283185307179586476925286766559L;
      ctx->turns[i] = static_cast<uint64_t>((per - std::floor(per)) * 18446744073709551616.0L);
    }
    ctx->turns_known = true;
  }
  for (int i = 0; i < half; ++i) a.turn[i] = ctx->turns[i];
  a.q = q;
  a.k = k;
  a.q_out = q_out;
  a.k_out = k_out;
  a.q_weight = q_weight;
  a.k_weight = k_weight;
  a.pos = pos;
  a.n_rows = n_rows;
  a.q_stride = q_stride;
  a.k_stride = k_stride;
  a.q_out_stride = q_out_stride;
  a.k_out_stride = k_out_stride;
  a.n_q_heads = c.n_q_heads;
  a.n_heads = c.n_q_heads + c.n_kv_heads;
  a.eps = eps > 0 ? std::max(static_cast<float>(eps), FLT_MIN) : 0.f;  // (zeros stay zeros however small it is)
  hipStream_t stream = static_cast<hipStream_t>(stream_);
  const bool norm = eps >= 0, inter = c.rope_interleaved != 0;
  if (c.dtype == MPIC_BF16)
    launch_position<__bf16, 128>(a, inter, norm, stream);
  else if (c.head_dim == 128)
    launch_position<float, 128>(a, inter, norm, stream);
  else
    launch_position<float, 64>(a, inter, norm, stream);
  MPIC_HIP(ctx, hipGetLastError());
  return MPIC_OK;
}
