// kv4.h -- the 4-bit cache: where a (page, kv head) block keeps its codes and scales, and the
// conversions from and to bf16.
//
// The d values of a token's K or V row of one kv head form blocks of 32.  A block holds a scale
// 2^s, stored as the byte s + 127, and 32 codes of 4 bits in e2m1 (0, 1/2, 1, 3/2, 2, 3, 4, 6 and
// their negatives).  s is the least with max|x| <= 7 * 2^s: up to 7, the largest code 6 is no
// further off than half a step of its binade.  A code times its scale has 2 significant bits,
// so it is exact in bf16, and gfx950 converts two codes with their scale in one instruction, both
// ways, to nearest with ties to even; the byte 255 (a block that is not finite) converts to NaN.
//
// The codes lie in the order in which lanes feed the MFMAs, so that a wave reads a page's K (or V)
// codes as 64 contiguous pieces of d / 8 bytes, lane l the l-th, and nothing passes through LDS:
//   K  lane l: slot l % 16, entries [d/4 (l/16), + d/4)   (A operand of S^T = K Q^T, 16 keys)
//   V  lane l: slots 4 (l/16) .. + 3, d/16 entries from d/16 (l%16) of each, slot after slot (the 4
//      keys whose probabilities the lane holds after S^T, so A operand of O^T += V^T P^T)
// with a byte's lower half the lower entry.  Block bytes: K codes 8 d, V codes 8 d, K scales
// [d/32][16 slots], V scales [4 quads][d/32][4 slots].  17 d bytes: 17 lines of 128 at d = 128.
#pragma once

#include "tide_device.h"

namespace tide {

template <int D>
struct Kv4 {
  static constexpr int kBlock = kv4_block_bytes(D);
  static constexpr int kLane = D / 8;      // code bytes of a lane (K or V of a page)
  static constexpr int kWords = D / 32;    // the same in 32-bit words
  static constexpr int kVCodes = 8 * D;
  static constexpr int kKScales = 16 * D;
  static constexpr int kVScales = 16 * D + D / 2;
  static constexpr int kSpan = D / 16;     // entries of a V slot in a lane
  static constexpr int kBlocks = D / 32;   // scale blocks of a row
  static constexpr int kVLanes = 32 / kSpan;  // lanes (of 16) of one V scale block
  // the scale byte of lane's K codes, and the 4 of its V codes, from the block's start
  static __device__ __forceinline__ int k_scale(int lane) {
    return kKScales + 16 * ((lane >> 4) * (D / 4) / 32) + (lane & 15);
  }
  static __device__ __forceinline__ int v_scale(int lane) {
    return kVScales + 4 * ((lane >> 4) * kBlocks + (lane & 15) / kVLanes);
  }
  // A row as 16 pieces of kSpan entries: the bytes of piece r of slot `slot` in K's and in V's codes, and
  // the scale byte of K's (V's: v_scale of the lane 16 (slot / 4) + r, its byte slot % 4)
  static __device__ __forceinline__ int k_word(int r, int slot) {
    return ((r >> 2) * 16 + slot) * kLane + (r & 3) * (kLane / 4);
  }
  static __device__ __forceinline__ int k_byte(int r, int slot) { return kKScales + 16 * (r / kVLanes) + slot; }
  static __device__ __forceinline__ int v_word(int r, int slot) {
    return kVCodes + ((slot >> 2) * 16 + r) * kLane + (slot & 3) * (kLane / 4);
  }
};

// A scale byte as the factor that the conversions take.
__device__ __forceinline__ float kv4_factor(uint32_t byte) { return __builtin_bit_cast(float, byte << 23); }

// Codes 2 kSel and 2 kSel + 1 of a word as a packed bf16 pair.
template <int kSel>
__device__ __forceinline__ uint32_t kv4_pair(uint32_t codes, float factor) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, factor, kSel));
}

// The 8 codes of a word, as a lane's bf16 operand.
__device__ __forceinline__ bf16x8 kv4_octet(uint32_t codes, float factor) {
  const u32x4 x = {kv4_pair<0>(codes, factor), kv4_pair<1>(codes, factor), kv4_pair<2>(codes, factor),
                   kv4_pair<3>(codes, factor)};
  return as_bf16x8(x);
}

// Writes the codes of a packed bf16 pair as byte kSel of a word.
template <int kSel>
__device__ __forceinline__ uint32_t kv4_put(uint32_t codes, uint32_t pair, float factor) {
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, __builtin_bit_cast(bf16x2, pair), factor, kSel);
}

// Codes of 8 bf16 values (4 packed pairs).
__device__ __forceinline__ uint32_t kv4_codes(u32x4 x, float factor) {
  uint32_t c = kv4_put<0>(0u, x[0], factor);
  c = kv4_put<1>(c, x[1], factor);
  c = kv4_put<2>(c, x[2], factor);
  return kv4_put<3>(c, x[3], factor);
}

// Largest magnitude of packed bf16 pairs, as bits (they order like the values; inf and NaN last).
__device__ __forceinline__ uint32_t kv4_max(uint32_t m, uint32_t pair) {
  return max(m, max(pair & 0x7FFFu, (pair >> 16) & 0x7FFFu));
}

// The scale byte of a block whose largest magnitude has these bf16 bits.
__device__ __forceinline__ uint32_t kv4_scale_byte(uint32_t amax) {
  const int b = (int)(amax >> 7) - 2 + ((amax & 0x7F) > 0x60 ? 1 : 0);
  return amax >= 0x7F80u ? 255u : (uint32_t)min(max(b, 7), 252);
}

}  // namespace tide
