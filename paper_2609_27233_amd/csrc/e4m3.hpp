// Cached features in 8 bits: e4m3 values (sign, 4 bits of exponent, 3 of the
// fraction, largest 448, no infinities) under one power of two for each entry
// and head (gfx950).
//
// A float format loses nothing to a scale that is only a power of two (a row's
// largest value lands anywhere in the upper binade of 17), and a power of two
// costs nothing: quantising is one exact product and the conversion's own
// rounding, and reading back is the conversion alone, which takes the exponent
// with it.  The exponent goes by the row as it comes in, before it is turned:
// its bits do not depend on how a rotation rounds.  With M = max|x| (times the
// rotation's scale where that is above 1), 2^(e+8) >= M, and a turned pair is
// at most sqrt 2 M <= 362 x 2^e, below 448 x 2^e.
#pragma once

#include "common.hpp"

namespace sm {

// Exponents kept: bf16 holds 2^-9 x 2^-100 and 448 x 2^119 exactly.
constexpr int kExpBias = 127, kLeastExp = -100, kMostExp = 119;
constexpr float kMostE4m3 = 448.f;

// Byte of the least e with most <= 2^(e + 8), for most >= 0.
__device__ __forceinline__ int exp_byte(float most) {
  const uint32_t b = __float_as_uint(most);
  const int up = (int)(b >> 23) - 127 + ((b & 0x7fffffu) != 0);  // (a subnormal: far below the least)
  return min(max(up - 8, kLeastExp), kMostExp) + kExpBias;
}

__device__ __forceinline__ float exp_scale(int byte) { return __uint_as_float((uint32_t)byte << 23); }     // 2^(byte - 127)
__device__ __forceinline__ float exp_inverse(int byte) { return __uint_as_float((uint32_t)(254 - byte) << 23); }

// Four quotients -> four e4m3 values, the first in the low byte (to nearest,
// ties to even; NaN and infinities become NaN).
__device__ __forceinline__ uint32_t pack_e4m3(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
  return (uint32_t)w;
}
// Under the largest exponent a finite quotient may be above 448: the largest value then.
__device__ __forceinline__ float in_e4m3(float z) {
  const float size = fabsf(z);
  return size > kMostE4m3 && size < INFINITY ? copysignf(kMostE4m3, z) : z;
}

// Four e4m3 values times 2^(scale's exponent) -> two pairs of bf16, exact.
__device__ __forceinline__ uint32_t e4m3_lo(uint32_t w, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, false));
}
__device__ __forceinline__ uint32_t e4m3_hi(uint32_t w, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, true));
}
// Eight (two words) -> 16 bytes of bf16.
__device__ __forceinline__ u32x4_t e4m3_to_bf16(uint32_t a, uint32_t b, float scale) {
  return u32x4_t{e4m3_lo(a, scale), e4m3_hi(a, scale), e4m3_lo(b, scale), e4m3_hi(b, scale)};
}

typedef uint16_t u16x2_t __attribute__((ext_vector_type(2)));

// Largest |feature| of 16 bytes of bf16, as bf16's bits.  (Without its sign it
// ascends as the 16-bit integer: two features to an instruction.)
__device__ __forceinline__ uint32_t largest_bits(u32x4_t v) {
  u16x2_t m = __builtin_bit_cast(u16x2_t, v[0] & 0x7fff7fffu);
#pragma unroll
  for (int i = 1; i < 4; ++i) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2_t, v[i] & 0x7fff7fffu));
  return max((uint32_t)m[0], (uint32_t)m[1]);
}
// A row whose largest feature passes these bits (2^126) has an infinity or NaN
// in it, which its maximum leaves out, or the largest exponent, under which a
// feature may have to be cut to 448.
constexpr uint32_t kPlainBits = 0x7e80u;
__device__ __forceinline__ float largest(u32x4_t v) {
  uint32_t most = largest_bits(v);
  if (most >= 0x7f80u) {
    most = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t x = v[i / 2] >> (16 * (i % 2)) & 0x7fffu;
      if (x < 0x7f80u) most = max(most, x);
    }
  }
  return __uint_as_float(most << 16);
}

template <int CTRL>
__device__ __forceinline__ uint32_t dpp_bits(uint32_t v) {
  return __float_as_uint(dpp_f32<CTRL>(__uint_as_float(v)));
}
// Maximum (of values >= 0, by their bits) over the lanes of a head, 8 features
// each: 16 neighbours, or 8 where the head has 64.
__device__ __forceinline__ uint32_t head_max(uint32_t v, bool wide) {
  v = max(v, dpp_bits<kDppXor1>(v));
  v = max(v, dpp_bits<kDppXor2>(v));
  v = max(v, dpp_bits<kDppHalfMirror>(v));
  const uint32_t both = max(v, dpp_bits<kDppMirror>(v));
  return wide ? both : v;
}

// Bytes i of four words: in[r] byte d -> out[d] byte r.
__device__ __forceinline__ void transpose4(const uint32_t (&in)[4], uint32_t (&out)[4]) {
  const uint32_t a = __builtin_amdgcn_perm(in[1], in[0], 0x05010400u), b = __builtin_amdgcn_perm(in[1], in[0], 0x07030602u);
  const uint32_t c = __builtin_amdgcn_perm(in[3], in[2], 0x05010400u), d = __builtin_amdgcn_perm(in[3], in[2], 0x07030602u);
  out[0] = __builtin_amdgcn_perm(c, a, 0x05040100u);
  out[1] = __builtin_amdgcn_perm(c, a, 0x07060302u);
  out[2] = __builtin_amdgcn_perm(d, b, 0x05040100u);
  out[3] = __builtin_amdgcn_perm(d, b, 0x07060302u);
}

// Exponent bytes of an e4m3 pool: behind its values, [num_blocks][num_kv_heads][block_size].
template <typename P>
static inline P *pool_exps(P *pool, int64_t num_blocks, int heads, int bs, int D) {
  return pool + num_blocks * heads * bs * D;
}

}  // namespace sm
