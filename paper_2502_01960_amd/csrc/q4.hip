// Writing rows into a cache held in 4 bits and reading them back (gfx950).  The format is described in mpic_q4.h, its
// layout in q4.h.
//
// Both kernels move every byte once, 2 * D values of 2 or 4 bytes on one side and D bytes of codes on the other, and are
// bound by HBM bandwidth.  A wavefront takes 16 rows of one head and either their keys or their values, with the lanes
// arranged as the codes are: its 64 lanes hold the codes of 16 tokens, and what a group of 64 values shares is found by
// exchanges between 4 lanes (K) or 16 (V).  Rows come and go with streaming loads and stores (79360 rows of 4 heads, written and
// read back: 83 us, 92 with ordinary ones); codes are stored the ordinary way, streaming stores take 15 us more.  Writing
// takes 49 us of that (4.3 TB/s; 520 vector instructions a wavefront keep it above the 44 of a copy), reading 34 (6.1 TB/s).
// Rows in slots without order touch some eight lines each for their 144 bytes: 65536 of them 83 and 65 us, in pages 42 and 29.
#include "common.h"
#include "mpic_q4.h"
#include "q4.h"

namespace mpic {
namespace {

using q4::Block;
using q4::kGroup;
using q4::kTokens;

struct RowsArgs {
  const char* k;  // rows (read or written)
  const char* v;
  char* cache;
  const int32_t* slots;
  int64_t n_rows, n_slots, k_stride, v_stride;  // strides in bytes
  uint32_t n_heads;
};

template <typename T>
struct Pair {
  T scale, low;
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

// Minimum and maximum as single instructions (fminf and fmaxf make a second one of every operand that may be a signalling
// NaN; what is no number is looked for separately).
__device__ inline float min3(float a, float b, float c) {
  float r;
  asm("v_min3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}
__device__ inline float max3(float a, float b, float c) {
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}
struct Range {
  float low, high;
};
// *nan: one of the values is no number
template <int N>
__device__ inline Range range_of(const float (&x)[N], bool* nan) {
  Range r = {x[0], x[0]};
#pragma unroll
  for (int e = 0; e < N; e += 2) {
    r.low = min3(r.low, x[e], x[e + 1]);
    r.high = max3(r.high, x[e], x[e + 1]);
    *nan |= __builtin_isunordered(x[e], x[e + 1]);
  }
  return r;
}
// over lanes l, l ^ 16, l ^ 32, l ^ 48 (a swap of two copies leaves the one half's values in one, the other's in the other)
__device__ inline Range range_across_quarters(Range r) {
  auto both = [](float x, bool rows, float* y) {
    const unsigned u = __builtin_bit_cast(unsigned, x);
    const auto p = rows ? __builtin_amdgcn_permlane16_swap(u, u, false, false) : __builtin_amdgcn_permlane32_swap(u, u, false, false);
    const unsigned p0 = p[0], p1 = p[1];
    y[0] = __builtin_bit_cast(float, p0);
    y[1] = __builtin_bit_cast(float, p1);
  };
#pragma unroll
  for (int step = 0; step < 2; ++step) {
    float l[2], h[2];
    both(r.low, step == 0, l);
    both(r.high, step == 0, h);
    r.low = min3(l[0], l[0], l[1]);
    r.high = max3(h[0], h[0], h[1]);
  }
  return r;
}
// over the sixteen lanes of a row, for four ranges: rotations by 8, 4, 2 and 1, interleaved so that no instruction follows
// within two of the one whose result it fetches from other lanes
#define MPIC_STEP(n)                                                        \
  "v_min_f32_dpp %0, %0, %0 row_ror:" #n " row_mask:0xf bank_mask:0xf\n\t" \
  "v_max_f32_dpp %4, %4, %4 row_ror:" #n " row_mask:0xf bank_mask:0xf\n\t" \
  "v_min_f32_dpp %1, %1, %1 row_ror:" #n " row_mask:0xf bank_mask:0xf\n\t" \
  "v_max_f32_dpp %5, %5, %5 row_ror:" #n " row_mask:0xf bank_mask:0xf\n\t" \
  "v_min_f32_dpp %2, %2, %2 row_ror:" #n " row_mask:0xf bank_mask:0xf\n\t" \
  "v_max_f32_dpp %6, %6, %6 row_ror:" #n " row_mask:0xf bank_mask:0xf\n\t" \
  "v_min_f32_dpp %3, %3, %3 row_ror:" #n " row_mask:0xf bank_mask:0xf\n\t" \
  "v_max_f32_dpp %7, %7, %7 row_ror:" #n " row_mask:0xf bank_mask:0xf\n\t"
__device__ inline void ranges_across_row(Range (&r)[4]) {
  asm("s_nop 1\n\t" MPIC_STEP(8) MPIC_STEP(4) MPIC_STEP(2) MPIC_STEP(1) "s_nop 0"
      : "+v"(r[0].low), "+v"(r[1].low), "+v"(r[2].low), "+v"(r[3].low), "+v"(r[0].high), "+v"(r[1].high), "+v"(r[2].high), "+v"(r[3].high));
}
#undef MPIC_STEP

// What a group's values share.  range / 15 by the product with RN(1/15) and one step of the remainder, which rounds it
// correctly; the reciprocal of the scale is a little too large (see code_of).
struct Coding {
  float low, scale, inv;
};
// Sets *odd if a group is flat or its range is not finite (0 / 0 and inf - inf come out as no number).
template <typename T, int N>
__device__ inline void codings_of(const Range (&r)[N], Coding (&c)[N], bool* odd) {
  constexpr float kFifteenth = 1.f / 15.f;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const float range = r[i].high - r[i].low;
    float q = range * kFifteenth;
    q = fmaf(fmaf(-15.f, q, range), kFifteenth, q);
    c[i].low = r[i].low;
    c[i].scale = static_cast<float>(static_cast<T>(q));
    c[i].inv = __builtin_amdgcn_rcpf(c[i].scale) * (1.f + 0x1p-20f);
    *odd |= !(c[i].scale >= q4::kLeastScale);
  }
}
// What such groups get, and groups with a value that is no number: `nan` of any of the `lanes` that share the group
__device__ inline void settle(Coding* c, bool nan, uint64_t lanes) {
  if ((__ballot(nan) & lanes) || c->scale != c->scale)
    *c = Coding{NAN, NAN, 0.f};
  else if (!(c->scale >= q4::kLeastScale))
    *c = Coding{c->low, 0.f, 0.f};
}

// The whole number nearest to (x - low) / scale, halves upwards.  The candidate is the product with the reciprocal, rounded by
// an addition that leaves it in the last bits of a float.  The reciprocal is 2^-20 too large, more than it can be off: so
// quotients halfway between two codes, which are common where values have few bits, go up as they should, and the
// only candidates that are wrong are one too large, for quotients within 2^-16 below a border.  The remainder
// e = d - code * scale is exact (both are multiples of the smaller one's last place, and it is no larger than about a scale)
// and tells those; `check` collects them, and a wavefront that has any (or a group that is flat or not finite) is done
// once more with care.  The greatest value gets 15: rounding the scale makes its quotient 15.06 at most.
constexpr float kWhole = 8388608.f;  // 2^23
struct Codes {
  uint32_t word;
  bool check;
  // Codes go in from the last nibble of a word to the first.  What the float's other bits add to the word is the same for
  // every code and comes off at the end.
  template <bool kSure>
  __device__ inline void push(float x, const Coding& c) {
    const float d = x - c.low;
    const float t = fmaf(d, c.inv, kWhole);
    const float e = fmaf(kWhole - t, c.scale, d);
    const bool over = e < -0.5f * c.scale;
    if (!kSure) {
      check |= over;
      word = (word << 4) + __builtin_bit_cast(uint32_t, t);
    } else {
      word = word << 4 | (c.inv == 0.f ? 0u : static_cast<uint32_t>(static_cast<int>(t - kWhole) - (over ? 1 : 0)));
    }
  }
  static constexpr uint32_t kRest = 0xFB000000u;  // sum of 0x4B000000 << 4 n, n = 0 .. 7, modulo 2^32
  template <bool kSure>
  __device__ inline uint32_t done() const { return kSure ? word : word - kRest; }
};

// N values of T, kept as they are in memory: bf16 values take half the registers of floats, and are widened where they are
// needed, once for the range and once for the codes (more wavefronts fit a SIMD)
template <typename T, int N>
struct Values {
  typedef T vec __attribute__((ext_vector_type(N), aligned(8)));
  typedef uint32_t bits __attribute__((ext_vector_type(N * sizeof(T) / 4)));
  bits raw;
  __device__ inline void load(const char* p) { raw = __builtin_bit_cast(bits, __builtin_nontemporal_load(reinterpret_cast<const vec*>(p))); }
  __device__ inline void widen(float (&x)[N]) const {
    const vec v = __builtin_bit_cast(vec, raw);
#pragma unroll
    for (int e = 0; e < N; ++e) x[e] = static_cast<float>(v[e]);
  }
  // what was widened before is not kept
  __device__ inline void forget() {
    if (sizeof(T) == 2)
#pragma unroll
      for (int i = 0; i < static_cast<int>(N * sizeof(T) / 4); ++i) {
        uint32_t u = raw[i];
        asm volatile("" : "+v"(u));
        raw[i] = u;
      }
  }
};
template <typename T, int N>
__device__ inline void store_values(char* p, const float (&x)[N]) {
  typedef T vec __attribute__((ext_vector_type(N), aligned(8)));
  vec v;
#pragma unroll
  for (int e = 0; e < N; ++e) v[e] = static_cast<T>(x[e]);
  __builtin_nontemporal_store(v, reinterpret_cast<vec*>(p));
}

// Codes and codings of a lane's keys: `row` its values of the first group.  kSure: without a doubt, values read again; returns
// whether that has to be done in this wavefront.
template <typename T, int D, bool kSure>
__device__ inline bool encode_keys(const char* row, int t, Pair<T> (&pairs)[Block<T, D>::kGroups], uint32_t (&words)[Block<T, D>::kGroups * 2]) {
  constexpr int kGroups = Block<T, D>::kGroups;
  Values<T, 16> v[kGroups];
#pragma unroll
  for (int g = 0; g < kGroups; ++g) v[g].load(row + g * kGroup * sizeof(T));
  Range range[kGroups];
  float x[16];
  bool check = false, nan[kGroups] = {};
#pragma unroll
  for (int g = 0; g < kGroups; ++g) {
    v[g].widen(x);
    range[g] = range_across_quarters(range_of(x, kSure ? &nan[g] : &check));
    v[g].forget();
  }
  Coding code[kGroups];
  codings_of<T>(range, code, &check);
#pragma unroll
  for (int g = 0; g < kGroups; ++g) {
    __builtin_amdgcn_sched_barrier(0);  // (a group after the other: fewer registers, more wavefronts)
    if (kSure) settle(&code[g], nan[g], 0x0001000100010001ull << t);
    pairs[g] = Pair<T>{static_cast<T>(code[g].scale), static_cast<T>(code[g].low)};
    v[g].widen(x);
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      Codes codes = {0, check};
#pragma unroll
      for (int n = 7; n >= 0; --n) codes.push<kSure>(x[8 * w + (n < 4 ? 2 * n : 2 * n - 7)], code[g]);
      words[2 * g + w] = codes.done<kSure>();
      check = codes.check;
    }
  }
  return __any(check);
}

template <typename T, int D>
__device__ inline void write_keys(const RowsArgs& a, int64_t row0, int head, int lane) {
  using B = Block<T, D>;
  const int t = lane & 15, c = lane >> 4;
  const int slot = slot_of(a, row0 + t);
  // rows that are left out take part in the exchanges (with a row that is there) and store nothing
  const char* row = a.k + min(row0 + t, a.n_rows - 1) * a.k_stride + (head * D + 16 * c) * sizeof(T);
  Pair<T> pairs[B::kGroups];
  uint32_t words[B::kGroups * 2];
  if (encode_keys<T, D, false>(row, t, pairs, words)) encode_keys<T, D, true>(row, t, pairs, words);
  char* block = block_of<T, D>(a, max(slot, 0), head);
  if (slot >= 0 && c == 0)
#pragma unroll
    for (int g = 0; g < B::kGroups; ++g)
      reinterpret_cast<Pair<T>*>(block + B::kKPairs)[g * kTokens + (slot & 15)] = pairs[g];
  if (slot < 0) return;
  uint32_t* dst = reinterpret_cast<uint32_t*>(block + (c * kTokens + (slot & 15)) * B::kLaneBytes);
#pragma unroll
  for (int w = 0; w < B::kGroups * 2; ++w) dst[w] = words[w];
}

// The same of the values of four rows
template <typename T, int D, bool kSure>
__device__ inline bool encode_values(const char* const (&row)[4], int quad, Pair<T> (&pairs)[Block<T, D>::kGroups][4],
                                     uint32_t (&words)[Block<T, D>::kGroups * 2]) {
  constexpr int kGroups = Block<T, D>::kGroups;
  Values<T, 4> v[kGroups][4];
#pragma unroll
  for (int r = 0; r < 4; ++r)
#pragma unroll
    for (int g = 0; g < kGroups; ++g) v[g][r].load(row[r] + g * kGroup * sizeof(T));
  bool check = false;
#pragma unroll
  for (int g = 0; g < kGroups; ++g) {
    __builtin_amdgcn_sched_barrier(0);
    float x[4][4];
    Range range[4];
    bool nan[4] = {};
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      v[g][r].widen(x[r]);
      range[r] = range_of(x[r], kSure ? &nan[r] : &check);
    }
    ranges_across_row(range);
    Coding code[4];
    codings_of<T>(range, code, &check);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      if (kSure) settle(&code[r], nan[r], 0xffffull << (16 * quad));
      pairs[g][r] = Pair<T>{static_cast<T>(code[r].scale), static_cast<T>(code[r].low)};
    }
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      Codes codes = {0, check};
#pragma unroll
      for (int n = 7; n >= 0; --n) codes.push<kSure>(x[n / 2][2 * w + n % 2], code[n / 2]);
      words[2 * g + w] = codes.done<kSure>();
      check = codes.check;
    }
  }
  return __any(check);
}

template <typename T, int D>
__device__ inline void write_values(const RowsArgs& a, int64_t row0, int head, int lane) {
  using B = Block<T, D>;
  const int i = lane & 15, quad = lane >> 4;
  const char* row[4];
  int slot[4];
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const int64_t n = row0 + 4 * quad + r;
    slot[r] = slot_of(a, n);
    row[r] = a.v + min(n, a.n_rows - 1) * a.v_stride + (head * D + 4 * i) * sizeof(T);
  }
  Pair<T> pairs[B::kGroups][4];
  uint32_t words[B::kGroups * 2];
  if (encode_values<T, D, false>(row, quad, pairs, words)) encode_values<T, D, true>(row, quad, pairs, words);
  if (i == 0)
#pragma unroll
    for (int r = 0; r < 4; ++r)
      if (slot[r] >= 0)
#pragma unroll
        for (int g = 0; g < B::kGroups; ++g)
          reinterpret_cast<Pair<T>*>(block_of<T, D>(a, slot[r], head) + B::kVPairs)[g * kTokens + (slot[r] & 15)] = pairs[g][r];
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

// A wavefront's 16 rows, and their keys or values of a head.  Heads come first, so that whole rows are read and written by
// neighbouring wavefronts.
struct Item {
  int64_t row0;
  int head;
  bool values;
};
__device__ inline bool item_of(const RowsArgs& a, Item* item) {
  const uint32_t n = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), th = n / a.n_heads;
  item->head = static_cast<int>(n % a.n_heads);
  item->values = th & 1;
  item->row0 = static_cast<int64_t>(th >> 1) * kTokens;
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

// Checks shared by both directions; fills *a and sets *go if there is anything to do.
int rows_args(mpic_ctx* ctx, const char* what, const void* k, int64_t k_stride, const void* v, int64_t v_stride, int64_t n_rows,
              const int32_t* slots, const void* cache, int64_t cache_bytes, int64_t n_slots, RowsArgs* a, bool* go) {
  const mpic_config& c = ctx->cfg;
  const auto invalid = [&](const char* why) { return fail(ctx, MPIC_ERR_INVALID, what, why); };
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
  if ((n_rows + kTokens - 1) / kTokens * c.n_kv_heads * 2 > INT32_MAX / 64)  // (wavefronts; threads of a launch)
    return fail(ctx, MPIC_ERR_UNSUPPORTED, what, "too many rows and heads for one launch");
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
  const int64_t need = mpic::q4::cache_bytes(c.dtype == MPIC_F32, c.head_dim, c.n_kv_heads, n_slots);
  if (need == INT64_MAX) return MPIC_ERR_UNSUPPORTED;
  *bytes = need;
  return MPIC_OK;
}

#define MPIC_Q4_ROWS(kernel, args, stream)                                                                          \
  do {                                                                                                              \
    const dim3 grid(static_cast<unsigned>(((args.n_rows + mpic::kTokens - 1) / mpic::kTokens * args.n_heads * 2 + 3) / 4)); \
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
