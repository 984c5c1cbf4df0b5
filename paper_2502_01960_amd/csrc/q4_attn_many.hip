// Attention over contexts held in 4 bits, large launches of many rows per kv head (gfx950, bf16): a prompt in chunks, the
// questions of a next turn over long contexts.  Formulas and formulation as in q4_attn.hip; other work bounds it: 4 D flops per
// row and key for D bytes of codes a key make it a matter of the matrix cores and of the vector instructions around them.
//
// A workgroup of four wavefronts takes 128 flattened rows (query, head in the kv group), 32 each, and walks the keys 64 at a
// time.  Every wavefront turns one of the four blocks of 16 tokens into matrix operands for all: K codes into bf16 pairs (exact,
// scales and lows are applied to the scores: 4 operations a score), V into its values, rounded to bf16 as they would be
// read back (two and a half operations a value once, where scaling the weights takes 7 per row and key).  Weights go in as two
// bf16 parts: with V rounded too, one part (623 TFLOP/s instead of 520) makes the error 1.6 times that of rounding the
// output, two make it 1.35, as with few rows.  The operands
// lie in LDS in the order in which lanes fetch them, in two buffers: one barrier per 64 keys, and the codes of the next 64 are
// loaded meanwhile.
//
// A token whose V holds what is no number (or reaches the end of the range) is made one whose score is no number, and its V zero:
// in the products a weight of zero would not keep it from rows that do not see it.  Slots that were never written may hold
// anything; they are treated the same, and no row sees their scores.
#include "q4_attn.h"

namespace mpic {
namespace q4 {
namespace {

constexpr int D = 128;
using B = Block<__bf16, D>;
constexpr int kWaves = 4;
constexpr int kStep = kWaves * kTokens;  // keys of a step
constexpr int kRowTiles = 2;             // of 16 rows, a wavefront
static_assert(kManyRows == kWaves * kRowTiles * 16 && kStep == kManyUnits * kUnit, "");

// A buffer: K operands [block][group, half][lane], V operands [block pair][group, column of four][lane], K pairs [block][group][token]
constexpr int kKeys = kWaves * 4 * 1024;
constexpr int kBuffer = 2 * kKeys + kWaves * B::kPairs;
constexpr int kLds = 2 * kBuffer;

typedef __bf16 pairs8 __attribute__((ext_vector_type(8)));

// Do the values of a group fit bf16?  (false also where one of the two is no number)
__device__ inline bool in_range(float scale, float low) { return fabsf(low) + 16.f * fabsf(scale) < 3.38e38f; }

// A block in registers of the wavefront that prepares it
struct Raw {
  u32x4 k, v;
  pairs8 vp[2];      // scale, low of the lane's four tokens, per group
  uint32_t kp, vp1;  // lanes 0 .. 31: the pairs of token lane % 16 and group lane / 16
  bool have;
};

__global__ __launch_bounds__(kWaves * 64, 2) void q4_attn_many_kernel(Q4AttnArgs a) {
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  const int lane = threadIdx.x & 63, col = lane & 15, quarter = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int head = blockIdx.x % a.n_kv_heads, split = blockIdx.y, b = blockIdx.z;
  const int row0 = static_cast<int>(blockIdx.x / a.n_kv_heads) * kManyRows;
  const Request rq = request_of(a, b);
  const int n_flat = rq.n * a.group;
  if (row0 >= n_flat) return;
  const int behind = rq.len - rq.n;
  const int key_end = max(behind + (min(row0 + kManyRows, n_flat) - 1) / a.group + 1, 0);  // of the workgroup
  const int64_t each = static_cast<int64_t>(units_of_split(a, rq)) * kUnit;
  const int64_t from = split * each;  // keys of the split
  const int first = static_cast<int>(min(from, static_cast<int64_t>(key_end))), end = static_cast<int>(min(from + each, static_cast<int64_t>(key_end)));
  if (a.n_splits > 1 && end <= first) return;  // (the merge asks for no such split)
  const int n_steps = end > first ? (end - first + kStep - 1) / kStep : 0;
  // of this wavefront: rows, keys that some of them see, keys that all of them see
  const int my_row0 = row0 + wave * kRowTiles * 16, my_last = min(my_row0 + kRowTiles * 16, n_flat) - 1;
  const int my_end = my_row0 < n_flat ? min(end, behind + my_last / a.group + 1) : first;
  const int my_all = behind + my_row0 / a.group + 1;

  bf16x8 q[kRowTiles][2][2];
  float q_sum[kRowTiles][2], m[kRowTiles], l[kRowTiles];  // (q_sum: a sixteenth)
  f32x4 o[kRowTiles][8];
  int limit[kRowTiles];
#pragma unroll
  for (int t = 0; t < kRowTiles; ++t) {
    const int at = my_row0 + 16 * t + col, flat = min(at, n_flat - 1), token = flat / a.group;
    limit[t] = at < n_flat ? behind + token + 1 : 0;
    const __bf16* src = reinterpret_cast<const __bf16*>(a.q + (rq.first + token) * a.q_stride) + static_cast<int64_t>(head * a.group + flat % a.group) * D;
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      q_sum[t][g] = 0.f;
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        q[t][g][w] = *reinterpret_cast<const bf16x8*>(src + g * kGroup + quarter * 16 + w * 8);
        const f32x8 x = __builtin_convertvector(q[t][g][w], f32x8);
#pragma unroll
        for (int e = 0; e < 8; ++e) q_sum[t][g] += x[e];
      }
      q_sum[t][g] += __shfl_xor(q_sum[t][g], 16);
      q_sum[t][g] += __shfl_xor(q_sum[t][g], 32);
    }
    q_sum[t][0] *= 0.0625f;
    q_sum[t][1] *= 0.0625f;
    m[t] = kLowest;
    l[t] = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) o[t][i] = f32x4{0};
  }
  const float factor = a.scale_log2 * 16.f;

  const int32_t* table = a.table + b * a.table_width;
  // blocks of this wavefront's next 64 steps, one a lane; -1: not in the cache
  int ids = -1;
  const auto look_up = [&](int step0) {
    const int64_t block = first / kTokens + static_cast<int64_t>(step0 + lane) * kWaves + wave;
    ids = -1;
    if (block * kTokens < end) {
      const int n = static_cast<int>(block);
      const int64_t id = static_cast<int64_t>(table[n / a.page_blocks]) * a.page_blocks + n % a.page_blocks;
      if (id >= 0 && id < a.n_blocks) ids = static_cast<int>(id);
    }
  };
  const auto load = [&](int step) {
    Raw r;
    if ((step & 63) == 0) look_up(step);
    const int64_t id = __builtin_amdgcn_readlane(ids, step & 63);
    r.have = id >= 0;
    const char* p = a.cache + ((r.have ? id : 0) * a.n_kv_heads + head) * B::kBytes;
    r.k = *reinterpret_cast<const u32x4*>(p + lane * 16);
    r.v = *reinterpret_cast<const u32x4*>(p + B::kV + lane * 16);
#pragma unroll
    for (int g = 0; g < 2; ++g) r.vp[g] = *reinterpret_cast<const pairs8*>(p + B::kVPairs + (g * kTokens + 4 * quarter) * 4);
    r.kp = *reinterpret_cast<const uint32_t*>(p + B::kKPairs + (lane & 31) * 4);
    r.vp1 = *reinterpret_cast<const uint32_t*>(p + B::kVPairs + (lane & 31) * 4);
    return r;
  };
  // this wavefront's block into a buffer
  const auto prepare = [&](const Raw& r, char* buffer) {
#pragma unroll
    for (int w = 0; w < 4; ++w) *reinterpret_cast<bf16x8*>(buffer + (wave * 4 + w) * 1024 + lane * 16) = keys_of<false>(r.k[w]);
    // (of a block that is not in the cache block 0 stands here; its scores are masked)
    char* values = buffer + kKeys + (wave >> 1) * 8 * 1024 + lane * 16 + (wave & 1) * 8;
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      float scale[4], low[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        scale[i] = static_cast<float>(r.vp[g][2 * i]);
        low[i] = static_cast<float>(r.vp[g][2 * i + 1]);
        if (!in_range(scale[i], low[i])) scale[i] = low[i] = 0.f;
      }
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        uint32_t nibbles = r.v[2 * g + c / 2] >> (4 * (c & 1)) & 0x0F0F0F0Fu;
        asm("" : "+v"(nibbles));  // (bytes, which are converted in one instruction each)
        f32x4 x;
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = fmaf(static_cast<float>(nibbles >> (8 * i) & 255u), scale[i], low[i]);
        *reinterpret_cast<bf16x4*>(values + (g * 4 + c) * 1024) = __builtin_convertvector(x, bf16x4);
      }
    }
    if (lane < 32) {
      // (0x7FFF in both halves is no number: the pair of a token whose V is none, in either of its groups)
      const bool nan = !in_range(__builtin_bit_cast(float, r.vp1 << 16), __builtin_bit_cast(float, r.vp1 & 0xFFFF0000u));
      const bool any = __builtin_amdgcn_ballot_w64(nan) >> (lane & 15) & 0x10001u;
      *reinterpret_cast<uint32_t*>(buffer + 2 * kKeys + wave * B::kPairs + lane * 4) = any ? 0x7FFF7FFFu : r.kp;
    }
  };
  const auto attend = [&](const char* buffer, int pos, uint32_t have) {
    float x[kRowTiles][kWaves][4];
#pragma unroll
    for (int k = 0; k < kWaves; ++k) {
      bf16x8 keys[4];
      float scale[2][4], low[2][4];
#pragma unroll
      for (int w = 0; w < 4; ++w) keys[w] = *reinterpret_cast<const bf16x8*>(buffer + (k * 4 + w) * 1024 + lane * 16);
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        const pairs8 p = *reinterpret_cast<const pairs8*>(buffer + 2 * kKeys + k * B::kPairs + (g * kTokens + 4 * quarter) * 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          scale[g][i] = static_cast<float>(p[2 * i]);
          // the ones in the codes' operands come off here: (low - 16 scale) sum(q)
          low[g][i] = fmaf(-16.f, scale[g][i], static_cast<float>(p[2 * i + 1]));
        }
      }
#pragma unroll
      for (int t = 0; t < kRowTiles; ++t) {
        f32x4 sum[2];
#pragma unroll
        for (int g = 0; g < 2; ++g) {
          sum[g] = mfma(keys[2 * g], q[t][g][0], f32x4{0});
          sum[g] = mfma(keys[2 * g + 1], q[t][g][1], sum[g]);
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          x[t][k][r] = fmaf(scale[1][r], sum[1][r],
                            fmaf(scale[0][r], sum[0][r], fmaf(low[1][r], q_sum[t][1], low[0][r] * q_sum[t][0])));
        }
      }
    }
    if (have != 15 || pos + kStep > my_all) {  // not every row sees every key
#pragma unroll
      for (int t = 0; t < kRowTiles; ++t)
#pragma unroll
        for (int k = 0; k < kWaves; ++k)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const bool seen = (have >> k & 1) && pos + kTokens * k + 4 * quarter + r < limit[t];
            x[t][k][r] = seen ? x[t][k][r] : -INFINITY;
          }
    }
    bf16x8 p[kRowTiles][2][2];  // weights in two parts
#pragma unroll
    for (int t = 0; t < kRowTiles; ++t) {
      float top = x[t][0][0];
#pragma unroll
      for (int i = 1; i < 4 * kWaves; ++i) top = fmaxf(top, x[t][i / 4][i % 4]);
      top *= factor;
      if (__any(top > m[t] + kSlack)) {
        float n = fmaxf(m[t], top);
        n = fmaxf(n, __shfl_xor(n, 16));
        n = fmaxf(n, __shfl_xor(n, 32));
        const float f = __builtin_amdgcn_exp2f(m[t] - n);
        m[t] = n;
        l[t] *= f;
#pragma unroll
        for (int i = 0; i < 8; ++i) o[t][i] *= f;
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        f32x8 w;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          w[i] = __builtin_amdgcn_exp2f(fmaf(x[t][2 * h + i / 4][i % 4], factor, -m[t]));
          l[t] += w[i];
        }
        p[t][h][0] = __builtin_convertvector(w, bf16x8);
        p[t][h][1] = __builtin_convertvector(w - __builtin_convertvector(p[t][h][0], f32x8), bf16x8);
      }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const bf16x8 values = *reinterpret_cast<const bf16x8*>(buffer + kKeys + (h * 8 + i) * 1024 + lane * 16);
#pragma unroll
        for (int t = 0; t < kRowTiles; ++t) o[t][i] = mfma(values, p[t][h][0], mfma(values, p[t][h][1], o[t][i]));
      }
  };

  __shared__ uint32_t have_block[2][kWaves];
  Raw raw;
  if (n_steps > 0) raw = load(0);
  for (int s = 0; s < n_steps; ++s) {
    char* buffer = lds + (s & 1) * kBuffer;
    // the buffer was read two steps ago, in front of the barrier of the step between
    prepare(raw, buffer);
    if (lane == 0) have_block[s & 1][wave] = raw.have;
    if (s + 1 < n_steps) raw = load(s + 1);
    __syncthreads();
    uint32_t have = 0;
#pragma unroll
    for (int k = 0; k < kWaves; ++k) have |= have_block[s & 1][k] << k;
    have = __builtin_amdgcn_readfirstlane(have);
    const int pos = first + s * kStep;
    if (pos < my_end) attend(buffer, pos, have);
  }

#pragma unroll
  for (int t = 0; t < kRowTiles; ++t) {
    float z = l[t];
    z += __shfl_xor(z, 16);
    z += __shfl_xor(z, 32);
    const int at = my_row0 + 16 * t + col;
    if (at >= n_flat) continue;
    const bool none = z == 0.f;
    const float inv = none ? 0.f : 1.f / z, lse2 = none ? -INFINITY : m[t] + log2f(z);
    const int64_t row = (rq.first + at / a.group) * a.n_q_heads + head * a.group + at % a.group;
    const int64_t part = row * a.n_splits + split;
    if (quarter == 0) {
      if (a.n_splits > 1)
        a.ws_lse[part] = lse2;
      else if (a.lse)
        a.lse[row] = lse2 * kLn2;
    }
#pragma unroll
    for (int g = 0; g < 2; ++g)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const f32x4 x = f32x4{o[t][4 * g][r], o[t][4 * g + 1][r], o[t][4 * g + 2][r], o[t][4 * g + 3][r]} * inv;
        const int d0 = g * kGroup + quarter * 16 + 4 * r;
        if (a.n_splits > 1)
          *reinterpret_cast<f32x4*>(a.ws_o + part * D + d0) = x;
        else
          *reinterpret_cast<bf16x4*>(a.out + (row * D + d0) * 2) = __builtin_convertvector(x, bf16x4);
      }
  }
}

LdsOptIn opt_in;

}  // namespace

hipError_t launch_q4_attn_many(const Q4AttnArgs& a, dim3 grid, hipStream_t stream) {
  int dev = -1;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  e = opt_in.ensure(dev, [] {
    return hipFuncSetAttribute(reinterpret_cast<const void*>(q4_attn_many_kernel), hipFuncAttributeMaxDynamicSharedMemorySize, kLds);
  });
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(q4_attn_many_kernel, grid, dim3(kWaves * 64), kLds, stream, a);
  return hipGetLastError();
}

}  // namespace q4
}  // namespace mpic
