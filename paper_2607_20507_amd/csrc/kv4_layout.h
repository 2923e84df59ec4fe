// The 4-bit KV cache: element values, scales and byte order of one (page, kv
// head) block, 16 tokens x hd dims of K or of V.
//
// A token's head vector is held in blocks of 32 consecutive dims.  A block has
// a scale 2^E, E the smallest integer >= -126 with max |x| <= 6 2^E, stored as
// the byte E + 127 (255: the block held an infinity or a NaN and reads back as
// NaN), and 32 codes: sign bit 8, magnitude codes 0..7 for 0, 0.5, 1, 1.5, 2,
// 3, 4, 6, the nearest to x 2^-E with ties to the even code.  Every value held
// is exactly a bf16 number: reading it back rounds nothing.  (E is the
// smallest that clips no value: the largest error in a block is half a step.)
//
// A block is 8 hd bytes of codes, then hd / 2 scale bytes; dims in the order
// of the attention kernel's matrix operands:
//  * K, token k, dim d, with s = d / 32, g = d / 8 % 4, h = k / 4 % 2,
//    j = k % 4 + 4 (k / 8): 4-byte unit s of lane unit (h, g, j) holds dims
//    32 s + 8 g .. + 7 of the token, low nibbles first.  Lane units are ordered
//    ((h 4 + g) 8 + j) for hd = 128 (16 bytes each) and ((g 8 + j) 2 + h) for
//    hd = 64 (8 bytes), so that a lane's load is 16 bytes in both.  The scale
//    of (k, s): byte (j 2 + h) hd / 32 + s.
//  * V, token k, dim d, with b = d / 32, i = d % 16: byte
//    16 ((b / 2 * 2 + k / 8) 16 + i) + 8 (b % 2) + k % 8, low nibble dim
//    32 b + i, high nibble dim 32 b + 16 + i (both of one token: tokens never
//    share a byte, so rows of one call may be appended by different threads).
//    The scale of (k, b): byte (k / 8 * hd / 32 + b) 8 + k % 8.
#pragma once

#include <stddef.h>
#include <stdint.h>

namespace spec {

#define SPEC_HD __host__ __device__ __forceinline__

SPEC_HD constexpr int kv4_code_bytes(int hd) { return 8 * hd; }
SPEC_HD constexpr int kv4_block_bytes(int hd) { return 8 * hd + hd / 2; }

// Byte of the 4-byte unit that holds dims 32 s + 8 g .. + 7 of token k's key.
SPEC_HD int kv4_k_unit(int k, int s, int g, int hd) {
  const int h = (k >> 2) & 1, j = (k & 3) + 4 * (k >> 3);
  return (hd == 128 ? ((h * 4 + g) * 8 + j) * 16 : ((g * 8 + j) * 2 + h) * 8) + 4 * s;
}
SPEC_HD int kv4_k_scale(int k, int s, int hd) {
  const int h = (k >> 2) & 1, j = (k & 3) + 4 * (k >> 3);
  return kv4_code_bytes(hd) + (j * 2 + h) * (hd >> 5) + s;
}
// Byte of dims 32 b + i and 32 b + 16 + i (i < 16) of token k's value vector.
SPEC_HD int kv4_v_byte(int k, int b, int i) {
  return (((b >> 1) * 2 + (k >> 3)) * 16 + i) * 16 + 8 * (b & 1) + (k & 7);
}
SPEC_HD int kv4_v_scale(int k, int b, int hd) {
  return kv4_code_bytes(hd) + ((k >> 3) * (hd >> 5) + b) * 8 + (k & 7);
}

// Scale byte of a block whose largest magnitude is m: the exponent field less
// 2, one more where the fraction exceeds 1.5 (6 2^E = 1.5 2^(E + 2)), at
// least 1; 255 for an infinity or a NaN.
SPEC_HD uint32_t kv4_scale_of(uint32_t m_bits) {
  const uint32_t ex = (m_bits >> 23) & 255u;
  if (ex == 255u) return 255u;
  const int e = static_cast<int>(ex) - 2 + ((m_bits & 0x7FFFFFu) > 0x400000u ? 1 : 0);
  return static_cast<uint32_t>(e < 1 ? 1 : e);
}

#undef SPEC_HD

}  // namespace spec
