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

// A quotient as e4m3 takes it: above 448 (only under the largest exponent) the
// largest value, an infinity NaN.
__device__ __forceinline__ float in_e4m3(float z) {
  const float size = fabsf(z);
  return size <= kMostE4m3 ? z : size < INFINITY ? copysignf(kMostE4m3, z) : NAN;
}

// Four quotients -> four e4m3 values, the first in the low byte (to nearest, ties to even).
__device__ __forceinline__ uint32_t pack_e4m3(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(in_e4m3(a), in_e4m3(b), 0, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(in_e4m3(c), in_e4m3(d), w, true);
  return (uint32_t)w;
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

// Largest |feature| of 16 bytes of bf16, infinities and NaN left out.
__device__ __forceinline__ float largest(const float (&f)[8]) {
  float m = fmaxf(fmaxf(fabsf(f[0]), fabsf(f[1])), fmaxf(fabsf(f[2]), fabsf(f[3])));  // (fmaxf leaves NaN out)
  m = fmaxf(m, fmaxf(fmaxf(fabsf(f[4]), fabsf(f[5])), fmaxf(fabsf(f[6]), fabsf(f[7]))));
  if (m == INFINITY) {
    m = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) m = fabsf(f[e]) < INFINITY ? fmaxf(m, fabsf(f[e])) : m;
  }
  return m >= 0.f ? m : 0.f;  // (nothing but NaN)
}

// Maximum over the 8 or 16 neighbouring lanes of a head (8 features each).
template <int LANES>
__device__ __forceinline__ float head_max(float v) {
  v = fmaxf(v, dpp_f32<kDppXor1>(v));
  v = fmaxf(v, dpp_f32<kDppXor2>(v));
  v = fmaxf(v, dpp_f32<kDppHalfMirror>(v));
  if constexpr (LANES == 16) v = fmaxf(v, dpp_f32<kDppMirror>(v));
  return v;
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
