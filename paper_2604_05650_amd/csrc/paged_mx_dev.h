// The paged cache in 4 bits as the kernels see it: blocks, table, ring and plan are those of the cache in 8 bits
// (paged_dev.h), a complete block is in e2m1 with a power of two per 32 values.
//
// A block of a kv head is 4 KiB of keys, 4 KiB of values and 256 bytes of scale exponents for each, in the order in
// which a wave's lanes take operands of 32x32 matrix instructions: lane l = 32 h + m reads the 16 bytes (32 codes)
// at 32 m + 16 h of a KiB, and the four exponents at 4 l.
//   keys    KiB 2 a + t: tokens 32 t + m, channels 64 a + 32 h .. +31; a scale per token and those 32 channels,
//           byte 2 t + a of the lane's four
//   values  KiB c: channel 32 c + m, of the block's 64 tokens those with bit 2 equal to h, in ascending order, which
//           are the rows of the lane's scores; a scale per channel and those 32 tokens, byte c of the lane's four
// An even code is the low half of its byte.
#pragma once

#include "paged_dev.h"

namespace lvspec {

constexpr int kPage4Bytes = kPageTokens * 64;      // keys or values of one head
constexpr int kScale4Bytes = 256;

// Eight e2m1 times a scale as bf16 (exact: of the scales that a cache holds none leaves bf16's range).
LVS_DEV u32x4 widen4(uint32_t x, float scale) {
  auto two = [&](auto which) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, scale, decltype(which)::value));
  };
  return u32x4{two(std::integral_constant<int, 0>{}), two(std::integral_constant<int, 1>{}),
               two(std::integral_constant<int, 2>{}), two(std::integral_constant<int, 3>{})};
}

// Scale i of a dword of four exponents.
template <int I>
LVS_DEV float scale4(uint32_t x) {
  const uint32_t e = I == 0 ? x << 23 : I == 1 ? x << 15 : I == 2 ? x << 7 : x >> 1;
  return __builtin_bit_cast(float, e & 0x7f800000u);
}

}  // namespace lvspec
