// 16 bytes of fp32 or bf16 features as floats (gfx950).
#pragma once

#include "common.hpp"

namespace sm {

// The address of row `row` (no rows: none).
static inline const void *row_at(const void *p, int64_t row, int64_t stride, int es) {
  return p ? (const char *)p + row * stride * es : nullptr;
}
static inline void *row_at(void *p, int64_t row, int64_t stride, int es) {
  return p ? (char *)p + row * stride * es : nullptr;
}

template <typename T> struct Vec16;
template <> struct Vec16<float> {
  static constexpr int N = 4;
  static constexpr uint32_t kMinusInf = 0xff800000u, kLowest = 0xff7fffffu;  // as 32-bit words
  static __device__ __forceinline__ void open(u32x4_t v, float *f) {
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(v[i]);
  }
  static __device__ __forceinline__ u32x4_t close(const float *f) {
    return u32x4_t{__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])};
  }
};
template <> struct Vec16<uint16_t> {
  static constexpr int N = 8;
  static constexpr uint32_t kMinusInf = 0xff80ff80u, kLowest = 0xff7fff7fu;
  static __device__ __forceinline__ void open(u32x4_t v, float *f) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = __uint_as_float(v[i] << 16);
      f[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ u32x4_t close(const float *f) {
    return u32x4_t{pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7])};
  }
};

}  // namespace sm
