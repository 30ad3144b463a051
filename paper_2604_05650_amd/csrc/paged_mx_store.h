// Complete blocks of the paged cache in 4 bits (paged_mx_dev.h): rounding and layout.
//
// Keys are rounded where they are, eight channels of a token in a dword, and go to memory from there; the largest
// magnitudes of values, whose groups run over tokens, and their codes, which lie by channel, go through LDS.  A row is read
// once and a block written once: bound by memory as in 8 bits, of whose blocks these are half.
#pragma once

#include "paged_mx_dev.h"
#include "paged_store.h"

namespace lvspec {

namespace {

// The scale of 32 values from the bits of their largest magnitude: the smallest power of two s >= 2^-60 with
// max |x| <= 7 s, at which no value is further from its code's than half a step (codes end at 6, the next would be 8).
// A value that is not finite makes its whole group NaN: e2m1 has none of its own.
struct Scale4 {
  uint32_t byte;           // exponent + 127; 255: NaN
  float s;
  uint32_t keep;           // mask of the codes: all, or none of a NaN group
  bool top;                // s = 2^126: magnitudes to 3 s, since 4 s is beyond binary32
  LVS_DEV explicit Scale4(uint32_t m) {
    const int e = max((int)(m >> 7) - 127 - 2 + ((m & 0x7fu) > 0x60u ? 1 : 0), -60);      // 7 = 1.75 * 2^2
    const bool nan = m >= 0x7f80u;
    byte = nan ? 255u : (uint32_t)(e + 127);
    s = __builtin_bit_cast(float, (uint32_t)(e + 127) << 23);
    keep = nan ? 0u : 0xffffffffu;
    top = e >= 126;
  }
};

// Codes of 4 (6) become 3 (5).
LVS_DEV uint32_t below4(uint32_t codes) {
  const uint32_t y = (codes & 0x77777777u) ^ 0x66666666u;                  // 0 where it is 6
  return codes - (((0x88888888u - y) >> 3) & 0x11111111u);
}

typedef uint16_t pair16 __attribute__((ext_vector_type(2)));
LVS_DEV uint32_t max_pairs(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(pair16, a), __builtin_bit_cast(pair16, b)));
}

struct Pool4 {
  typedef __bf16 bf16x2s __attribute__((ext_vector_type(2)));
  // (a value, not an element: of elements of a vector this compiler casts the first)
  static LVS_DEV bf16x2s as_pair(uint32_t x) { return __builtin_bit_cast(bf16x2s, x); }
  struct Scratch {
    __align__(16) uint8_t turn[16 * 272];        // values' codes: a channel in 32 bytes, eight in 272
    __align__(16) uint32_t max[4][2][16][4];     // largest magnitudes of a wave's tokens: half, chunk of 8 channels
    __align__(16) uint8_t scale[kScale4Bytes];
  };

  // Thread (q, c) = (tid / 16, tid % 16) holds chunk c of rows 4q .. 4q+3.
  static LVS_DEV bool store(const u32x4 (&x)[4], bool values, uint8_t* pool, void* scale, int64_t at, Scratch& s) {
    uint8_t* dst = pool + at * kPage4Bytes;
    __syncthreads();                       // (the scratch of a block before this one has been read)
    if (values)
      store_values(x, dst, s);
    else
      store_keys(x, dst, s);
    __syncthreads();
    const int tid = threadIdx.x;
    if (values)
      *reinterpret_cast<u32x4*>(dst + tid * 16) =
          *reinterpret_cast<const u32x4*>(s.turn + (tid >> 4) * 272 + (tid & 15) * 16);
    if (tid < kScale4Bytes / 4)
      reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(scale) + at * kScale4Bytes)[tid] =
          reinterpret_cast<const uint32_t*>(s.scale)[tid];
    return false;
  }
  static LVS_DEV void mend(uint8_t*, int64_t) {}

  // four chunks in a row are a group
  static LVS_DEV void store_keys(const u32x4 (&x)[4], uint8_t* dst, Scratch& s) {
    const int tid = threadIdx.x, q = tid >> 4, c = tid & 15;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t m = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) m = max_pairs(m, x[i][j] & 0x7fff7fffu);
      m = max(m & 0xffffu, m >> 16);
      m = max(m, dpp_move<0xB1, 0xf>(0u, m));
      m = max(m, dpp_move<0x4E, 0xf>(0u, m));
      const Scale4 f(m);
      uint32_t codes = 0;
      codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, as_pair(x[i][0]), f.s, 0);
      codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, as_pair(x[i][1]), f.s, 1);
      codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, as_pair(x[i][2]), f.s, 2);
      codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, as_pair(x[i][3]), f.s, 3);
      codes = (f.top ? below4(codes) : codes) & f.keep;
      const int token = 4 * q + i;
      *reinterpret_cast<uint32_t*>(dst + (c >> 3) * 2048 + token * 32 + (c & 7) * 4) = codes;
      if ((c & 3) == 0)
        s.scale[((c >> 2) & 1) * 128 + (token & 31) * 4 + 2 * (token >> 5) + (c >> 3)] = (uint8_t)f.byte;
    }
  }

  // Rows 4q .. 4q+3 are tokens of half q % 2, in order the 4 (q / 2)-th and on.
  static LVS_DEV void store_values(const u32x4 (&x)[4], uint8_t* dst, Scratch& s) {
    const int tid = threadIdx.x, q = tid >> 4, c = tid & 15, half = q & 1;
    u32x4 m;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      uint32_t y = x[0][j] & 0x7fff7fffu;
#pragma unroll
      for (int i = 1; i < 4; ++i) y = max_pairs(y, x[i][j] & 0x7fff7fffu);
      m[j] = max_pairs(y, (uint32_t)__shfl_xor((int)y, 32, 64));            // (q and q + 2)
    }
    if ((tid & 32) == 0) *reinterpret_cast<u32x4*>(s.max[tid >> 6][half][c]) = m;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const u32x4 y = *reinterpret_cast<const u32x4*>(s.max[w][half][c]);
#pragma unroll
      for (int j = 0; j < 4; ++j) m[j] = max_pairs(m[j], y[j]);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      auto value = [&](int i) { return j & 1 ? bf16_hi(x[i][j >> 1]) : bf16_lo(x[i][j >> 1]); };
      const Scale4 f(j & 1 ? m[j >> 1] >> 16 : m[j >> 1] & 0xffffu);
      uint32_t codes = 0;
      codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, value(0), value(1), f.s, 0);
      codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, value(2), value(3), f.s, 1);
      codes = (f.top ? below4(codes) : codes) & f.keep;
      *reinterpret_cast<uint16_t*>(s.turn + c * 272 + j * 32 + half * 16 + (q >> 1) * 2) = (uint16_t)codes;
      const int channel = 8 * c + j;
      if (tid < 32) s.scale[half * 128 + (channel & 31) * 4 + (channel >> 5)] = (uint8_t)f.byte;
    }
  }
};

}  // namespace

}  // namespace lvspec
