// Rotary positions of rows of heads, and a layer's projected rows on their
// way into the paged cache (gfx950): rotary, kv_write_rotary.
//
// Every feature pair of a head is turned by position x frequency; the angles
// of a row are the same for all its heads.  Both calls read and write each
// row once and are bound by that traffic.  A workgroup takes a tile of rows
// and a range of heads: it forms the tile's cosines and sines in LDS (angle
// and reduction in double precision, then fp32), and turns 16 bytes of each
// half of a pair per thread.
//
// K rows go to token-major pages 16 bytes at a time.  V pages are dim-major,
// so V is transposed in registers: 8 rows (fp32: 4) that fill an aligned
// group of a page's slots become 16-byte stores.  Tiles are cut where such
// groups begin, so a prompt's rows are stored whole wherever its sequence
// starts in the batch; single rows (a decode step) are stored an element at
// a time, which the layout of the pages asks for.
#include <cmath>

#include "cache_meta.hpp"

namespace sm {

constexpr int kRotThreads = 256;
constexpr int kTileRows = 16;
constexpr int kMaxPairs = 128;

// One stream of rows of heads: [rows][heads][D] with a row stride.
struct Rows {
  const void *in;
  void *out;
  int64_t in_stride, out_stride;
  int heads;
};

struct RopeArgs {
  double turns[kMaxPairs];  // frequency / 2 pi: turns per position
  const int32_t *pos;
  int rows, R, sign;        // sign -1: transposed
  float scale;
  FastDiv per_head;         // units of a head: R / (2 VEC) turned pairs and (D - R) / VEC copies (scalar: R / 2 and D - R)
};

// Cosine and sine of the tile's rows, [row][pair]: the angle in turns is
// reduced to [-1/2, 1/2] in double precision.
__device__ __forceinline__ void fill_angles(const RopeArgs &a, int r0, int nr, float2 *cs) {
  const int P = a.R / 2;
  for (int u = threadIdx.x; u < nr * P; u += kRotThreads) {
    const int r = u / P, j = u - r * P;
    const double t = a.turns[j] * (double)a.pos[r0 + r];
    const float x = 2.f * (float)(t - rint(t));
    float s, c;
    sincospif(x, &s, &c);
    cs[u] = make_float2(a.scale * c, a.sign * a.scale * s);
  }
}

template <typename T> struct Vec;  // 16 bytes of T as floats
template <> struct Vec<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void open(u32x4_t v, float (&f)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(v[i]);
  }
  static __device__ __forceinline__ u32x4_t close(const float (&f)[4]) {
    return u32x4_t{__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])};
  }
};
template <> struct Vec<uint16_t> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void open(u32x4_t v, float (&f)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = __uint_as_float(v[i] << 16);
      f[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ u32x4_t close(const float (&f)[8]) {
    return u32x4_t{pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7])};
  }
};

__device__ __forceinline__ float2 turned(float a, float b, float2 cs) {
  return make_float2(a * cs.x - b * cs.y, a * cs.y + b * cs.x);
}

// Unit `j` of a head at `in` to `out`, cs: the row's cosines and sines.
// WIDE: a unit moves 16 bytes (half layout: of each half); else one pair or
// one feature.
template <typename T, bool HALF, bool WIDE>
__device__ __forceinline__ void turn_unit(const T *in, T *out, int j, int R, const float2 *cs) {
  if constexpr (WIDE) {
    constexpr int N = Vec<T>::N;
    const int turning = HALF ? R / (2 * N) : R / N;
    if (j >= turning) {  // behind the turned part
      const int at = R + (j - turning) * N;
      *(u32x4_t *)(out + at) = *(const u32x4_t *)(in + at);
    } else if constexpr (HALF) {
      float a[N], b[N];
      Vec<T>::open(*(const u32x4_t *)(in + j * N), a);
      Vec<T>::open(*(const u32x4_t *)(in + R / 2 + j * N), b);
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const float2 t = turned(a[e], b[e], cs[j * N + e]);
        a[e] = t.x;
        b[e] = t.y;
      }
      *(u32x4_t *)(out + j * N) = Vec<T>::close(a);
      *(u32x4_t *)(out + R / 2 + j * N) = Vec<T>::close(b);
    } else {
      float a[N];
      Vec<T>::open(*(const u32x4_t *)(in + j * N), a);
#pragma unroll
      for (int e = 0; e < N; e += 2) {
        const float2 t = turned(a[e], a[e + 1], cs[(j * N + e) / 2]);
        a[e] = t.x;
        a[e + 1] = t.y;
      }
      *(u32x4_t *)(out + j * N) = Vec<T>::close(a);
    }
  } else {
    if (j >= R / 2) {
      out[R / 2 + j] = in[R / 2 + j];
      return;
    }
    const int i0 = HALF ? j : 2 * j, i1 = HALF ? j + R / 2 : 2 * j + 1;
    const float2 t = turned(Elem<T>::load(in + i0), Elem<T>::load(in + i1), cs[j]);
    out[i0] = Elem<T>::to_store(t.x);
    out[i1] = Elem<T>::to_store(t.y);
  }
}

template <typename T, bool HALF, bool WIDE>
__global__ __launch_bounds__(kRotThreads) void rotary_kernel(RopeArgs a, Rows x, int D, int heads_per) {
  extern __shared__ float2 cs[];  // [rows of a tile][R / 2]
  const int r0 = blockIdx.x * kTileRows, nr = min(kTileRows, a.rows - r0);
  const int h0 = blockIdx.y * heads_per, nh = min(heads_per, x.heads - h0);
  fill_angles(a, r0, nr, cs);
  __syncthreads();
  const int per = a.per_head.d;
  const T *in = (const T *)x.in + (int64_t)r0 * x.in_stride + (int64_t)h0 * D;
  T *out = (T *)x.out + (int64_t)r0 * x.out_stride + (int64_t)h0 * D;
  for (int u = threadIdx.x; u < nr * nh * per; u += kRotThreads) {
    const int hr = fdiv(u, a.per_head), j = u - hr * per, r = hr / nh, h = hr - r * nh;
    turn_unit<T, HALF, WIDE>(in + r * x.in_stride + h * D, out + r * x.out_stride + h * D, j, a.R, cs + r * (a.R / 2));
  }
}

// ---------------------------------------------------------------------------
// kv_write_rotary

struct WriteArgs {
  Rows q, k, v;
  const int32_t *slots;
  void *k_pool, *v_pool;
  int32_t *err;
  int bs_log2, dh_log2, num_slots;
};

// Whether row r begins a group: rows that fill consecutive slots of one
// aligned group of VEC slots.
template <int VEC>
__device__ __forceinline__ bool begins_group(const int32_t *slots, int r) {
  const int s = slots[r];
  return r == 0 || s < 0 || s % VEC == 0 || slots[r - 1] != s - 1;
}

// Rows of a tile: from the first row at or past `r` (at most VEC - 1 further,
// the last row of a run aside) that begins a group.
template <int VEC>
__device__ __forceinline__ int tile_begin(const int32_t *slots, int r, int rows) {
  while (r < rows && !begins_group<VEC>(slots, r)) ++r;
  return min(r, rows);
}

template <typename T, bool HALF, bool WIDE>
__global__ __launch_bounds__(kRotThreads) void kv_write_kernel(RopeArgs a, WriteArgs w, int heads_per) {
  constexpr int VEC = 16 / sizeof(T);
  constexpr int kMost = kTileRows + VEC;
  extern __shared__ float2 cs[];
  __shared__ int slot[kMost], bounds[2];
  const int t = threadIdx.x, D = 1 << w.dh_log2, bs = 1 << w.bs_log2;
  if (t < 2) bounds[t] = tile_begin<VEC>(w.slots, (int)min((int64_t)a.rows, ((int64_t)blockIdx.x + t) * kTileRows), a.rows);
  __syncthreads();
  const int r0 = bounds[0], nr = bounds[1] - r0;
  const int h0 = blockIdx.y * heads_per, h1 = min(h0 + heads_per, w.q.heads + 2 * w.k.heads);
  if (t < nr) {
    const int s = w.slots[r0 + t];
    if (s < -1 || s >= w.num_slots) {
      if (h0 == 0) set_err(w.err, SM_ERR_EINVAL);
      slot[t] = -1;
    } else {
      slot[t] = s;
    }
  }
  const bool turns = h0 < w.q.heads + w.k.heads;
  if (turns) fill_angles(a, r0, nr, cs);
  __syncthreads();
  const int per = a.per_head.d;
  // q: this range's heads below q.heads
  {
    const int nh = min(h1, w.q.heads) - h0;
    const T *in = (const T *)w.q.in + (int64_t)r0 * w.q.in_stride + (int64_t)h0 * D;
    T *out = (T *)w.q.out + (int64_t)r0 * w.q.out_stride + (int64_t)h0 * D;
    for (int u = t; nh > 0 && u < nr * nh * per; u += kRotThreads) {
      const int hr = fdiv(u, a.per_head), j = u - hr * per, r = hr / nh, h = hr - r * nh;
      turn_unit<T, HALF, WIDE>(in + r * w.q.in_stride + h * D, out + r * w.q.out_stride + h * D, j, a.R,
                               cs + r * (a.R / 2));
    }
  }
  // k
  {
    const int g0 = max(h0 - w.q.heads, 0), nh = min(h1 - w.q.heads, w.k.heads) - g0;
    const T *in = (const T *)w.k.in + (int64_t)r0 * w.k.in_stride;
    for (int u = t; nh > 0 && u < nr * nh * per; u += kRotThreads) {
      const int hr = fdiv(u, a.per_head), j = u - hr * per, r = hr / nh, h = g0 + hr - r * nh;
      const int s = slot[r];
      if (s < 0) continue;
      T *out = (T *)w.k_pool + ((((int64_t)(s >> w.bs_log2) * w.k.heads + h) << w.bs_log2) + (s & (bs - 1))) * D;
      turn_unit<T, HALF, WIDE>(in + r * w.k.in_stride + h * D, out, j, a.R, cs + r * (a.R / 2));
    }
  }
  // v
  {
    const int g0 = max(h0 - w.q.heads - w.k.heads, 0), nh = h1 - w.q.heads - w.k.heads - g0;
    const T *in = (const T *)w.v.in + (int64_t)r0 * w.v.in_stride;
    for (int u = t; nh > 0 && u < nr * nh * D; u += kRotThreads) {
      const int d = u & (D - 1), hr = u >> w.dh_log2, r = hr / nh, h = g0 + hr - r * nh;
      const int s = slot[r];
      if (s < 0) continue;
      T *out = (T *)w.v_pool + (((((int64_t)(s >> w.bs_log2) * w.k.heads + h) << w.dh_log2) + d) << w.bs_log2) +
               (s & (bs - 1));
      *out = in[r * w.v.in_stride + h * D + d];
    }
  }
}

}  // namespace sm

using namespace sm;

static bool rope_ok(const sm_rope_params *p, int head_dim) {
  if (!p || p->rot_dim < 2 || (p->rot_dim & 1) || p->rot_dim > head_dim) return false;
  if (p->layout != SM_ROPE_HALF && p->layout != SM_ROPE_INTERLEAVED) return false;
  if (!(p->theta > 0.f) || !std::isfinite(p->theta) || !std::isfinite(p->attn_scale)) return false;
  if (p->scaling == SM_ROPE_PLAIN) return true;
  if (p->scaling < 0 || p->scaling > SM_ROPE_RAMP || !(p->factor > 0.f) || !std::isfinite(p->factor)) return false;
  if (p->scaling == SM_ROPE_LINEAR) return true;
  return p->low > 0.f && p->high > p->low && std::isfinite(p->high) && p->context > 0.f && std::isfinite(p->context) &&
         (p->scaling != SM_ROPE_RAMP || p->theta > 1.f);
}

// Frequencies in turns per position, on the host in double precision.
static void set_turns(const sm_rope_params *p, RopeArgs *a) {
  constexpr double two_pi = 6.283185307179586476925286766559;
  const int P = p->rot_dim / 2;
  const double ln_theta = std::log((double)p->theta), s = p->factor;
  const auto pair_of = [&](double t) { return p->rot_dim * std::log(p->context / (two_pi * t)) / (2 * ln_theta); };
  double j0 = 0, span = 1;
  if (p->scaling == SM_ROPE_RAMP) {
    j0 = std::fmax(std::floor(pair_of(p->high)), 0.0);
    span = std::fmax(std::fmin(std::ceil(pair_of(p->low)), p->rot_dim - 1.0) - j0, 0.001);
  }
  for (int j = 0; j < P; ++j) {
    double w = std::exp(-ln_theta * j / P) / two_pi;  // turns per position
    if (p->scaling == SM_ROPE_LINEAR) {
      w /= s;
    } else if (p->scaling == SM_ROPE_BANDS) {
      const double u = std::fmin(std::fmax((p->context * w - p->low) / ((double)p->high - p->low), 0.0), 1.0);
      w = u * w + (1 - u) * w / s;
    } else if (p->scaling == SM_ROPE_RAMP) {
      const double v = std::fmin(std::fmax((j - j0) / span, 0.0), 1.0);
      w = v * w / s + (1 - v) * w;
    }
    a->turns[j] = w;
  }
}

static bool wide_rows(const void *p, int64_t stride, size_t es) {
  return (uintptr_t)p % 16 == 0 && stride * es % 16 == 0;
}

static RopeArgs rope_args(const sm_rope_params *p, const int32_t *pos, int rows, int D, size_t es, bool wide,
                          int transpose) {
  RopeArgs a;
  set_turns(p, &a);
  a.pos = pos;
  a.rows = rows;
  a.R = p->rot_dim;
  a.sign = transpose ? -1 : 1;
  a.scale = p->attn_scale;
  const int vec = 16 / (int)es;
  a.per_head = make_fastdiv((uint32_t)(!wide ? p->rot_dim / 2 + D - p->rot_dim
                                              : (p->layout == SM_ROPE_HALF ? p->rot_dim / (2 * vec) : p->rot_dim / vec) +
                                                    (D - p->rot_dim) / vec));
  return a;
}

static bool wide_head(const sm_rope_params *p, int D, size_t es) {
  const int vec = 16 / (int)es;
  return D % vec == 0 && p->rot_dim % (2 * vec) == 0;
}

// Heads per workgroup: enough workgroups for the device where there are few rows.
static int heads_per_wg(int heads, int64_t tiles) {
  int per = heads;
  while (per > 1 && tiles * ((heads + per - 1) / per) < 512) per = (per + 1) / 2;
  return per;
}

template <typename T>
static void launch_rotary(const RopeArgs &a, const Rows &x, int D, bool half, bool wide, hipStream_t stream) {
  const int64_t tiles = ((int64_t)a.rows + kTileRows - 1) / kTileRows;
  const int per = heads_per_wg(x.heads, tiles);
  const dim3 grid((unsigned)tiles, (x.heads + per - 1) / per);
  const size_t lds = kTileRows * (a.R / 2) * sizeof(float2);
  const auto kernel = half ? (wide ? rotary_kernel<T, true, true> : rotary_kernel<T, true, false>)
                           : (wide ? rotary_kernel<T, false, true> : rotary_kernel<T, false, false>);
  hipLaunchKernelGGL(kernel, grid, dim3(kRotThreads), lds, stream, a, x, D, per);
}

SM_API sm_status sm_rotary(const void *x, int64_t x_stride, const int32_t *pos, int rows, int heads, int head_dim,
                           const sm_rope_params *p, int transpose, sm_dtype dt, void *out, int64_t out_stride,
                           hipStream_t stream) {
  if (dt != SM_F32 && dt != SM_BF16) return SM_EINVAL;
  if (rows < 0 || heads < 1 || heads > 1024 || head_dim < 2 || head_dim > 2 * kMaxPairs || !rope_ok(p, head_dim))
    return SM_EINVAL;
  const int64_t width = (int64_t)heads * head_dim;
  if (x_stride < width || out_stride < width || (transpose != 0 && transpose != 1)) return SM_EINVAL;
  if (rows == 0) return SM_OK;
  if (!x || !pos || !out) return SM_EINVAL;
  const size_t es = dt == SM_BF16 ? 2 : 4;
  const bool wide = wide_head(p, head_dim, es) && wide_rows(x, x_stride, es) && wide_rows(out, out_stride, es);
  const RopeArgs a = rope_args(p, pos, rows, head_dim, es, wide, transpose);
  const Rows r{x, out, x_stride, out_stride, heads};
  if (dt == SM_BF16) launch_rotary<uint16_t>(a, r, head_dim, p->layout == SM_ROPE_HALF, wide, stream);
  else launch_rotary<float>(a, r, head_dim, p->layout == SM_ROPE_HALF, wide, stream);
  return hipGetLastError() == hipSuccess ? SM_OK : SM_EHIP;
}

template <typename T>
static void launch_write(const RopeArgs &a, const WriteArgs &w, bool half, bool wide, hipStream_t stream) {
  const int64_t tiles = ((int64_t)a.rows + kTileRows - 1) / kTileRows;
  const int heads = w.q.heads + 2 * w.k.heads, per = heads_per_wg(heads, tiles);
  const dim3 grid((unsigned)tiles, (heads + per - 1) / per);
  const size_t lds = (kTileRows + 16 / sizeof(T)) * (a.R / 2) * sizeof(float2);
  const auto kernel = half ? (wide ? kv_write_kernel<T, true, true> : kv_write_kernel<T, true, false>)
                           : (wide ? kv_write_kernel<T, false, true> : kv_write_kernel<T, false, false>);
  hipLaunchKernelGGL(kernel, grid, dim3(kRotThreads), lds, stream, a, w, per);
}

SM_API sm_status sm_kv_write_rotary(const sm_paged_cache *c, const int32_t *pos, const int32_t *slots, int rows,
                                    const void *q, int64_t q_stride, int num_q_heads, const void *k, int64_t k_stride,
                                    const void *v, int64_t v_stride, const sm_rope_params *p, void *q_out,
                                    int64_t q_out_stride, hipStream_t stream) {
  CacheArgs ca;
  if (!cache_ok(c, ca) || rows < 0 || num_q_heads < 0 || num_q_heads > 1024 || c->num_kv_heads > 1024) return SM_EINVAL;
  if ((int64_t)c->num_blocks * c->block_size > INT32_MAX || !rope_ok(p, c->head_dim)) return SM_EINVAL;
  const int D = c->head_dim;
  const int64_t kv_width = (int64_t)c->num_kv_heads * D, q_width = (int64_t)num_q_heads * D;
  if (k_stride < kv_width || v_stride < kv_width) return SM_EINVAL;
  if (num_q_heads > 0 && (q_stride < q_width || q_out_stride < q_width)) return SM_EINVAL;
  if (rows == 0) return SM_OK;
  if (!pos || !slots || !k || !v || (num_q_heads > 0 && (!q || !q_out))) return SM_EINVAL;
  const size_t es = c->dtype == SM_BF16 ? 2 : 4;
  const bool wide = wide_head(p, D, es) && wide_rows(k, k_stride, es) && wide_rows(v, v_stride, es) &&
                    wide_rows(c->k_pool, 0, es) && wide_rows(c->v_pool, 0, es) &&
                    (num_q_heads == 0 || (wide_rows(q, q_stride, es) && wide_rows(q_out, q_out_stride, es)));
  const RopeArgs a = rope_args(p, pos, rows, D, es, wide, 0);
  WriteArgs w{Rows{q, q_out, q_stride, q_out_stride, num_q_heads}, Rows{k, nullptr, k_stride, 0, c->num_kv_heads},
              Rows{v, nullptr, v_stride, 0, c->num_kv_heads}, slots, c->k_pool, c->v_pool, c->err, ca.bs_log2,
              ca.dh_log2, c->num_blocks * c->block_size};
  if (c->dtype == SM_BF16) launch_write<uint16_t>(a, w, p->layout == SM_ROPE_HALF, wide, stream);
  else launch_write<float>(a, w, p->layout == SM_ROPE_HALF, wide, stream);
  return hipGetLastError() == hipSuccess ? SM_OK : SM_EHIP;
}
