// Layout of a cache held in 4 bits, shared by the kernels that write, read and attend it.
//
// 16 slots and one kv head make a block; blocks lie slot group after slot group, inside it head after head.  A block holds
//   K codes   [4 quarters][16 tokens][D / 8 bytes]   quarter c of a token: per group of 64 values the 16 values 16c .. 16c + 15
//   V codes   [4 token quads][16 columns][D / 8 bytes]  column i of tokens 4g .. 4g + 3: per group the values 4i .. 4i + 3
//   K pairs   [D / 64 groups][16 tokens] (scale, low)
//   V pairs   the same
// so that lane after lane of a wavefront reads D / 8 bytes after D / 8 bytes, of K and of V, and finds there what a 16x16x32
// matrix instruction takes from that lane: of K eight neighbouring values of one token, of V (whose tokens are the summed
// dimension) four tokens of one column.  Nothing is transposed on the way.
// A K word holds 8 neighbouring values, value 2n in bits 4n.. and value 2n + 1 in bits 16 + 4n..; a V word holds two
// columns of four tokens, token r in byte r, the even column in its low half.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace mpic {
namespace q4 {

constexpr int kTokens = 16;  // slots of a block
constexpr int kGroup = 64;   // values that share a scale and a minimum
constexpr float kLeastScale = 7.888609052210118e-31f;  // 2^-100

template <typename T, int D>
struct Block {
  static constexpr int kGroups = D / kGroup;
  static constexpr int kLaneBytes = D / 8;  // codes of a lane: of one token (K), of four (V)
  static constexpr int kCodes = 64 * kLaneBytes;
  static constexpr int kPair = 2 * sizeof(T);
  static constexpr int kPairs = kGroups * kTokens * kPair;
  static constexpr int kV = kCodes;  // offsets
  static constexpr int kKPairs = 2 * kCodes;
  static constexpr int kVPairs = kKPairs + kPairs;
  static constexpr int kBytes = kVPairs + kPairs;
};

inline int64_t block_bytes(bool f32, int head_dim) {
  return f32 ? (head_dim == 128 ? Block<float, 128>::kBytes : Block<float, 64>::kBytes) : Block<__bf16, 128>::kBytes;
}
// INT64_MAX (which no cache has) for what 64 bits do not hold
inline int64_t cache_bytes(bool f32, int head_dim, int n_kv_heads, int64_t n_slots) {
  int64_t bytes = (n_slots + kTokens - 1) / kTokens;
  if (__builtin_mul_overflow(bytes, static_cast<int64_t>(n_kv_heads), &bytes) || __builtin_mul_overflow(bytes, block_bytes(f32, head_dim), &bytes)) return INT64_MAX;
  return bytes;
}

}  // namespace q4
}  // namespace mpic
