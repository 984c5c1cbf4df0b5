// Writing rows into a cache held in 4 bits and reading them back (gfx950).  The format is described in mpic_q4.h, its
// layout in q4.h.
//
// Both kernels move every byte once, 2 * D values of 2 or 4 bytes on one side and D bytes of codes on the other, and are
// bound by HBM bandwidth.  A wavefront takes 16 rows of one head and either their keys or their values, with the lanes
// arranged as the codes are: its 64 lanes hold the codes of 16 tokens, and what a group of 64 values shares is found by
// exchanges between 4 lanes (K) or 16 (V).
#include "common.h"
#include "mpic_q4.h"
#include "q4.h"

namespace mpic {
namespace {

using q4::Block;
using q4::kGroup;
using q4::kTokens;

typedef float f32x4 __attribute__((ext_vector_type(4)));

struct RowsArgs {
  const char* k;  // rows (read or written)
  const char* v;
  char* cache;
  const int32_t* slots;
  int64_t n_rows, n_slots, k_stride, v_stride;  // strides in bytes
  int32_t n_heads;
};

// Slot of a row, -1 for rows that are left out
__device__ inline int slot_of(const RowsArgs& a, int64_t row) {
  if (row >= a.n_rows) return -1;
  const int64_t s = a.slots ? a.slots[row] : row;
  return s >= 0 && s < a.n_slots ? static_cast<int>(s) : -1;
}

template <typename T, int D>
__device__ inline char* block_of(const RowsArgs& a, int slot, int head) {
  return a.cache + (static_cast<int64_t>(slot >> 4) * a.n_heads + head) * Block<T, D>::kBytes;
}

// What a group's values share.  `nan`: one of them is no number.
struct Coding {
  float low, scale, inv;
};
template <typename T>
__device__ inline Coding coding_of(float low, float high, bool nan) {
  const float range = high - low;
  if (nan || !(range < INFINITY)) return Coding{NAN, NAN, 0.f};  // (infinities and ranges beyond fp32 alike)
  const float scale = static_cast<float>(static_cast<T>(range / 15.f));
  if (!(scale >= q4::kLeastScale)) return Coding{low, 0.f, 0.f};
  return Coding{low, scale, 1.f / scale};
}

// The whole number nearest to (x - low) / scale, halves upwards.  The product with the reciprocal is off by some 2^-22 at
// most, so the candidate is off by one at most, and the remainder d - code * scale (exact: both are multiples of the
// smaller one's last place, and it is no larger than about a scale) tells on which side of a border the value lies.
__device__ inline uint32_t code_of(float x, const Coding& c) {
  const float d = x - c.low;
  float code = floorf(fmaf(d, c.inv, 0.5f));
  const float e = fmaf(-code, c.scale, d), half = 0.5f * c.scale;
  code += e >= half ? 1.f : 0.f;
  code -= e < -half ? 1.f : 0.f;
  return c.inv == 0.f ? 0u : min(static_cast<uint32_t>(static_cast<int32_t>(code)), 15u);
}

// n values of T at p as floats (n * sizeof(T) bytes, 8 or 16 byte units)
template <typename T, int N>
__device__ inline void load_values(const char* p, float (&x)[N]) {
  typedef T vec __attribute__((ext_vector_type(N), aligned(8)));
  const vec v = *reinterpret_cast<const vec*>(p);
#pragma unroll
  for (int e = 0; e < N; ++e) x[e] = static_cast<float>(v[e]);
}
template <typename T, int N>
__device__ inline void store_values(char* p, const float (&x)[N]) {
  typedef T vec __attribute__((ext_vector_type(N), aligned(8)));
  vec v;
#pragma unroll
  for (int e = 0; e < N; ++e) v[e] = static_cast<T>(x[e]);
  *reinterpret_cast<vec*>(p) = v;
}
template <typename T>
struct Pair {
  T scale, low;
};

template <typename T, int D>
__device__ inline void write_keys(const RowsArgs& a, int64_t row0, int head, int lane) {
  using B = Block<T, D>;
  const int t = lane & 15, c = lane >> 4;
  const int slot = slot_of(a, row0 + t);
  // rows that are left out take part in the exchanges (with zeros) and store nothing
  char* block = block_of<T, D>(a, max(slot, 0), head);
  uint32_t words[B::kGroups * 2];
#pragma unroll
  for (int g = 0; g < B::kGroups; ++g) {
    float x[16] = {};
    if (slot >= 0) load_values<T, 16>(a.k + (row0 + t) * a.k_stride + (head * D + g * kGroup + 16 * c) * sizeof(T), x);
    float low = x[0], high = x[0];
    bool nan = false;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      low = fminf(low, x[e]);
      high = fmaxf(high, x[e]);
      nan |= x[e] != x[e];
    }
#pragma unroll
    for (int off = 16; off < 64; off <<= 1) {
      low = fminf(low, __shfl_xor(low, off));
      high = fmaxf(high, __shfl_xor(high, off));
    }
    nan = (__ballot(nan) >> t & 0x0001000100010001ull) != 0;
    const Coding code = coding_of<T>(low, high, nan);
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      uint32_t word = 0;
#pragma unroll
      for (int n = 0; n < 4; ++n)
        word |= code_of(x[8 * w + 2 * n], code) << (4 * n) | code_of(x[8 * w + 2 * n + 1], code) << (16 + 4 * n);
      words[2 * g + w] = word;
    }
    if (slot >= 0 && c == 0)
      reinterpret_cast<Pair<T>*>(block + B::kKPairs)[g * kTokens + (slot & 15)] = Pair<T>{static_cast<T>(code.scale), static_cast<T>(code.low)};
  }
  if (slot < 0) return;
  uint32_t* dst = reinterpret_cast<uint32_t*>(block + (c * kTokens + (slot & 15)) * B::kLaneBytes);
#pragma unroll
  for (int w = 0; w < B::kGroups * 2; ++w) dst[w] = words[w];
}

template <typename T, int D>
__device__ inline void write_values(const RowsArgs& a, int64_t row0, int head, int lane) {
  using B = Block<T, D>;
  const int i = lane & 15, quad = lane >> 4;
  int slot[4];
  uint32_t words[B::kGroups * 2] = {};
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const int64_t row = row0 + 4 * quad + r;
    slot[r] = slot_of(a, row);
#pragma unroll
    for (int g = 0; g < B::kGroups; ++g) {
      float x[4] = {};
      if (slot[r] >= 0) load_values<T, 4>(a.v + row * a.v_stride + (head * D + g * kGroup + 4 * i) * sizeof(T), x);
      float low = fminf(fminf(x[0], x[1]), fminf(x[2], x[3])), high = fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3]));
      bool nan = x[0] != x[0] || x[1] != x[1] || x[2] != x[2] || x[3] != x[3];
#pragma unroll
      for (int off = 1; off < 16; off <<= 1) {
        low = fminf(low, __shfl_xor(low, off));
        high = fmaxf(high, __shfl_xor(high, off));
      }
      nan = (__ballot(nan) >> (16 * quad) & 0xffffull) != 0;
      const Coding code = coding_of<T>(low, high, nan);
#pragma unroll
      for (int e = 0; e < 4; ++e) words[2 * g + e / 2] |= code_of(x[e], code) << (8 * r + 4 * (e & 1));
      if (slot[r] >= 0 && i == 0)
        reinterpret_cast<Pair<T>*>(block_of<T, D>(a, slot[r], head) + B::kVPairs)[g * kTokens + (slot[r] & 15)] =
            Pair<T>{static_cast<T>(code.scale), static_cast<T>(code.low)};
    }
  }
  // four rows that fill a quad of slots go out as words, any others byte by byte
  const bool whole = slot[0] >= 0 && (slot[0] & 3) == 0 && slot[1] == slot[0] + 1 && slot[2] == slot[0] + 2 && slot[3] == slot[0] + 3;
  if (whole) {
    char* at = block_of<T, D>(a, slot[0], head) + B::kV + ((slot[0] & 12) * 4 + i) * B::kLaneBytes;
#pragma unroll
    for (int w = 0; w < B::kGroups * 2; ++w) reinterpret_cast<uint32_t*>(at)[w] = words[w];
    return;
  }
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    if (slot[r] < 0) continue;
    char* at = block_of<T, D>(a, slot[r], head) + B::kV + ((slot[r] & 12) * 4 + i) * B::kLaneBytes + (slot[r] & 3);
#pragma unroll
    for (int w = 0; w < B::kGroups * 2; ++w) at[4 * w] = static_cast<char>(words[w] >> (8 * r));
  }
}

// A wavefront's 16 rows, and their keys or values of a head: grid (four tiles of rows, head and part)
struct Item {
  int64_t row0;
  int head;
  bool values;
};
__device__ inline bool item_of(const RowsArgs& a, Item* item) {
  item->row0 = (static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6)) * kTokens;
  item->head = blockIdx.y >> 1;
  item->values = blockIdx.y & 1;
  return item->row0 < a.n_rows;
}

template <typename T, int D>
__global__ __launch_bounds__(256) void q4_write_kernel(RowsArgs a) {
  Item item;
  if (!item_of(a, &item)) return;
  const int lane = threadIdx.x & 63;
  if (item.values)
    write_values<T, D>(a, item.row0, item.head, lane);
  else
    write_keys<T, D>(a, item.row0, item.head, lane);
}

template <typename T, int D>
__global__ __launch_bounds__(256) void q4_read_kernel(RowsArgs a) {
  using B = Block<T, D>;
  Item item;
  if (!item_of(a, &item)) return;
  const int lane = threadIdx.x & 63;
  if (!item.values) {
    const int t = lane & 15, c = lane >> 4;
    const int slot = slot_of(a, item.row0 + t);
    if (slot < 0) return;
    const char* block = block_of<T, D>(a, slot, item.head);
    const uint32_t* src = reinterpret_cast<const uint32_t*>(block + (c * kTokens + (slot & 15)) * B::kLaneBytes);
    char* dst = const_cast<char*>(a.k) + (item.row0 + t) * a.k_stride + (item.head * D + 16 * c) * sizeof(T);
#pragma unroll
    for (int g = 0; g < B::kGroups; ++g) {
      const Pair<T> p = reinterpret_cast<const Pair<T>*>(block + B::kKPairs)[g * kTokens + (slot & 15)];
      float x[16];
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const uint32_t code = src[2 * g + e / 8] >> (4 * (e % 8 / 2) + 16 * (e & 1)) & 15;
        x[e] = fmaf(static_cast<float>(code), static_cast<float>(p.scale), static_cast<float>(p.low));
      }
      store_values<T, 16>(dst + g * kGroup * sizeof(T), x);
    }
    return;
  }
  const int i = lane & 15, quad = lane >> 4;
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const int64_t row = item.row0 + 4 * quad + r;
    const int slot = slot_of(a, row);
    if (slot < 0) continue;
    const char* block = block_of<T, D>(a, slot, item.head);
    const uint32_t* src = reinterpret_cast<const uint32_t*>(block + B::kV + ((slot & 12) * 4 + i) * B::kLaneBytes);
    char* dst = const_cast<char*>(a.v) + row * a.v_stride + (item.head * D + 4 * i) * sizeof(T);
#pragma unroll
    for (int g = 0; g < B::kGroups; ++g) {
      const Pair<T> p = reinterpret_cast<const Pair<T>*>(block + B::kVPairs)[g * kTokens + (slot & 15)];
      float x[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t code = src[2 * g + e / 2] >> (8 * (slot & 3) + 4 * (e & 1)) & 15;
        x[e] = fmaf(static_cast<float>(code), static_cast<float>(p.scale), static_cast<float>(p.low));
      }
      store_values<T, 4>(dst + g * kGroup * sizeof(T), x);
    }
  }
}

constexpr int kMaxGridY = 65535;

// Checks shared by both directions; fills *a and sets *go if there is anything to do.
int rows_args(mpic_ctx* ctx, const char* what, const void* k, int64_t k_stride, const void* v, int64_t v_stride, int64_t n_rows,
              const int32_t* slots, const void* cache, int64_t cache_bytes, int64_t n_slots, RowsArgs* a, bool* go) {
  const mpic_config& c = ctx->cfg;
  const auto invalid = [&](const char* why) { return fail(ctx, MPIC_ERR_INVALID, std::string(what) + ": " + why); };
  const int64_t elem = c.dtype == MPIC_F32 ? 4 : 2, row = static_cast<int64_t>(c.n_kv_heads) * c.head_dim;
  *go = false;
  if (n_rows < 0 || n_rows >= INT32_MAX) return invalid("bad row count");
  if (n_slots < 0 || n_slots >= INT32_MAX) return invalid("bad slot count");
  if (k_stride < row || v_stride < row || k_stride * elem % 16 || v_stride * elem % 16)
    return invalid("strides must hold a row and be multiples of 16 bytes");
  if (!slots && n_rows > n_slots) return invalid("more rows than slots");
  if (cache_bytes < q4::cache_bytes(c.dtype == MPIC_F32, c.head_dim, c.n_kv_heads, n_slots)) return invalid("the cache is smaller than its slots");
  if (n_rows == 0 || n_slots == 0) return MPIC_OK;  // (no row has a slot)
  if (!k || !v || !cache) return invalid("null buffer");
  if ((reinterpret_cast<uintptr_t>(k) | reinterpret_cast<uintptr_t>(v) | reinterpret_cast<uintptr_t>(cache)) & 15)
    return invalid("buffers must be 16-byte aligned");
  if (2 * static_cast<int64_t>(c.n_kv_heads) > kMaxGridY) return fail(ctx, MPIC_ERR_UNSUPPORTED, std::string(what) + ": too many heads");
  const int rc = bind_device(ctx);
  if (rc != MPIC_OK) return rc;
  a->k = static_cast<const char*>(k);
  a->v = static_cast<const char*>(v);
  a->cache = static_cast<char*>(const_cast<void*>(cache));
  a->slots = slots;
  a->n_rows = n_rows;
  a->n_slots = n_slots;
  a->k_stride = k_stride * elem;
  a->v_stride = v_stride * elem;
  a->n_heads = c.n_kv_heads;
  *go = true;
  return MPIC_OK;
}

}  // namespace
}  // namespace mpic

extern "C" int mpic_q4_bytes(const mpic_ctx* ctx, int64_t n_slots, int64_t* bytes) {
  if (!ctx || !bytes || n_slots < 0 || n_slots >= INT32_MAX) return MPIC_ERR_INVALID;
  const mpic_config& c = ctx->cfg;
  *bytes = mpic::q4::cache_bytes(c.dtype == MPIC_F32, c.head_dim, c.n_kv_heads, n_slots);
  return MPIC_OK;
}

#define MPIC_Q4_ROWS(kernel, args, stream)                                                                          \
  do {                                                                                                              \
    const dim3 grid(static_cast<unsigned>((args.n_rows + 63) / 64), 2 * args.n_heads);                              \
    if (ctx->cfg.dtype == MPIC_BF16)                                                                                \
      hipLaunchKernelGGL((mpic::kernel<__bf16, 128>), grid, dim3(256), 0, stream, args);                            \
    else if (ctx->cfg.head_dim == 128)                                                                              \
      hipLaunchKernelGGL((mpic::kernel<float, 128>), grid, dim3(256), 0, stream, args);                             \
    else                                                                                                            \
      hipLaunchKernelGGL((mpic::kernel<float, 64>), grid, dim3(256), 0, stream, args);                              \
    MPIC_HIP(ctx, hipGetLastError());                                                                               \
  } while (0)

extern "C" int mpic_q4_write(mpic_ctx* ctx, const void* k, int64_t k_stride, const void* v, int64_t v_stride, int64_t n_rows,
                             const int32_t* slots, void* cache, int64_t cache_bytes, int64_t n_slots, void* stream) {
  if (!ctx) return MPIC_ERR_INVALID;
  mpic::RowsArgs a{};
  bool go;
  const int rc = mpic::rows_args(ctx, "q4_write", k, k_stride, v, v_stride, n_rows, slots, cache, cache_bytes, n_slots, &a, &go);
  if (rc != MPIC_OK || !go) return rc;
  MPIC_Q4_ROWS(q4_write_kernel, a, static_cast<hipStream_t>(stream));
  return MPIC_OK;
}

extern "C" int mpic_q4_read(mpic_ctx* ctx, const void* cache, int64_t cache_bytes, int64_t n_slots, const int32_t* slots,
                            int64_t n_rows, void* k, int64_t k_stride, void* v, int64_t v_stride, void* stream) {
  if (!ctx) return MPIC_ERR_INVALID;
  mpic::RowsArgs a{};
  bool go;
  const int rc = mpic::rows_args(ctx, "q4_read", k, k_stride, v, v_stride, n_rows, slots, cache, cache_bytes, n_slots, &a, &go);
  if (rc != MPIC_OK || !go) return rc;
  MPIC_Q4_ROWS(q4_read_kernel, a, static_cast<hipStream_t>(stream));
  return MPIC_OK;
}
