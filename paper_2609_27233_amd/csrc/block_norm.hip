// The residual stream past one block with the norms around it (gfx950):
//   h_out = h + scale gate norm_post(y),  n_out = norm_pre(h_out).
//
// Each row is read and written once: the row's features stay in registers
// (fp32) between the norms, so both norms, the gate and the sum cost no
// traffic beyond h, y, h_out and n_out, which bound the call: 39,328 bf16 rows
// of 4096 take 220 us (5.9 TB/s; a plain copy of 1 GiB reaches 5.1), with a
// norm behind y and a gate 228.  Few rows are bound by the loads' latency and
// the sums' barriers: 16 rows of 4096 2.6 and 3.4 us.  LayerNorm takes its
// mean first and sums squares of the differences from registers.
//
// A row is held by 8 threads to 1024, two 16-byte chunks each, so that its
// loads are all in flight at once and short rows fill a wave.  One chunk each
// (twice the threads) is faster without a norm behind y (39,328 rows of 4096
// 218 us) and for few rows, but has more waves wait for each sum where there
// are two (265 us); four are slower for all but rows of 16,384 (16 rows of
// 4096 4.1 us).  Rows that 16 bytes do not divide are read by the same chunks
// at the alignment they have, the last one by features (16,384 rows of 4095 bf16
// features 120 us, of 4096 93).
#include <algorithm>
#include <cmath>

#include "vec16.hpp"

namespace sm {

// A norm's kind: kNone leaves the row as it is.
enum { kNone = -1 };

struct NormArgs {
  const void *h, *y, *gate;
  const void *g_post, *b_post, *g_pre, *b_pre;
  void *h_out, *n_out;
  int64_t sh, sy, sg, sho, sno;
  int rows, d, post, pre;
  float scale, eps_post, eps_pre, inv_d;
};

// Sum over the TPR threads that hold a row; `red`: a float for each of their waves.
template <int TPR>
__device__ __forceinline__ float row_sum(float v, float *red) {
  if constexpr (TPR < 64) {
    v += dpp_f32<kDppXor1>(v);
    v += dpp_f32<kDppXor2>(v);
    v += dpp_f32<kDppHalfMirror>(v);
    if constexpr (TPR == 32) {
      v += dpp_f32<kDppMirror>(v);
      float a, b;
      swap16(v, a, b);
      v = a + b;
    }
  } else {
    v = wave_sum(v);
  }
  if constexpr (TPR > 64) {
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.f;
#pragma unroll
    for (int i = 0; i < TPR / 64; ++i) v += red[i];
  }
  return v;
}

// 16 bytes of features.  WHOLE: every chunk of a row is 16-byte aligned and
// within it; else at any address, and cut at feature d.
template <typename T, bool WHOLE>
struct Chunk {
  static constexpr int VEC = Vec16<T>::N;
  float f[VEC];
  static __device__ __forceinline__ u32x4_t load(const void *row, int64_t offset, int at, int d) {
    const T *p = (const T *)row + offset + at;
    u32x4_t v;
    if (WHOLE) {
      v = *(const u32x4_t *)p;
    } else if (at + VEC <= d) {
      __builtin_memcpy(&v, p, 16);
    } else {  // whole words, and for bf16 a half
      const int n = (d - at) * (int)sizeof(T);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint32_t x = 0;
        if (4 * i + 4 <= n) __builtin_memcpy(&x, (const char *)p + 4 * i, 4);
        else if (4 * i < n) x = *(const uint16_t *)((const char *)p + 4 * i);
        v[i] = x;
      }
    }
    return v;
  }
  __device__ __forceinline__ void store(void *row, int64_t offset, int at, int d) const {
    T *p = (T *)row + offset + at;
    const u32x4_t v = Vec16<T>::close(f);
    if (WHOLE) {
      *(u32x4_t *)p = v;
    } else if (at + VEC <= d) {
      __builtin_memcpy(p, &v, 16);
    } else {
      const int n = (d - at) * (int)sizeof(T);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t x = v[i];
        if (4 * i + 4 <= n) __builtin_memcpy((char *)p + 4 * i, &x, 4);
        else if (4 * i < n) *(uint16_t *)((char *)p + 4 * i) = (uint16_t)x;
      }
    }
  }
};

// Whether a row's gate, gain and bias are on their way before they are used.
// Aligned rows gain by it (16,384 fp32 rows of 2048 with both norms and a gate
// 94 us, 102 without; 16 bf16 rows of 4096 3.5 and 4.0); workgroups of 1024
// threads, of which a compute unit then holds one and not two, lose (8192
// bf16 rows of 16,384 245 and 209), and so do unaligned rows (16,384 rows of
// 2049 78 and 66).
template <bool WHOLE, int TPR>
constexpr bool kEarly = WHOLE && TPR < 1024;

// x <- norm(x), the row spread over TPR threads, NV chunks a thread.
template <typename T, bool WHOLE, int NV, int TPR>
__device__ __forceinline__ void norm_row(Chunk<T, WHOLE> (&x)[NV], int kind, float eps, const void *gain, const void *bias,
                                         int d, float inv_d, int at0, float *red) {
  constexpr int VEC = Vec16<T>::N, STEP = TPR * VEC;
  u32x4_t gains[NV], biases[NV];
  const auto load = [&](int v) {
    const int at = at0 + v * STEP;
    if (at >= d) return;
    if (gain) gains[v] = Chunk<T, WHOLE>::load(gain, 0, at, d);
    if (bias) biases[v] = Chunk<T, WHOLE>::load(bias, 0, at, d);
  };
  if (kEarly<WHOLE, TPR>)
#pragma unroll
    for (int v = 0; v < NV; ++v) load(v);
  if (kind == SM_NORM_LAYER) {
    float s = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int e = 0; e < VEC; ++e) s += x[v].f[e];  // (features past d are zeros)
    const float mean = row_sum<TPR>(s, red) * inv_d;
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int e = 0; e < VEC; ++e)
        if (at0 + v * STEP + (WHOLE ? 0 : e) < d) x[v].f[e] -= mean;
  }
  float q = 0.f;
#pragma unroll
  for (int v = 0; v < NV; ++v)
#pragma unroll
    for (int e = 0; e < VEC; ++e) q += x[v].f[e] * x[v].f[e];
  // (the hardware's root is off by a unit, the product with 1 / d rounded to fp32
  // by one more: the sum passes up to 40 roundings.  The root is for normal
  // numbers: an epsilon of 0 may leave less)
  const float m = row_sum<TPR>(q, red) * inv_d + eps, inv = m < 1.2e-38f ? 1.f / sqrtf(m) : __builtin_amdgcn_rsqf(m);
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int at = at0 + v * STEP;
    if (at >= d) continue;
    if (!kEarly<WHOLE, TPR>) load(v);
    float g[VEC], b[VEC];
    if (gain) Vec16<T>::open(gains[v], g);
    if (bias) Vec16<T>::open(biases[v], b);
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      float n = x[v].f[e] * inv;
      if (gain) n *= g[e];
      if (bias) n += b[e];
      x[v].f[e] = n;
    }
  }
}

constexpr int wg_threads(int tpr) { return tpr <= 64 ? 256 : tpr; }

// TPR threads hold a row, NV chunks each.
template <typename T, bool WHOLE, int NV, int TPR>
__global__ __launch_bounds__(wg_threads(TPR)) void block_norm_kernel(NormArgs a) {
  constexpr int RPW = wg_threads(TPR) / TPR;  // rows per workgroup
  constexpr int VEC = Vec16<T>::N, STEP = TPR * VEC;
  __shared__ float red[TPR > 64 ? TPR / 64 : 1];  // (several waves to a row: one row per workgroup)
  const int64_t row = (int64_t)blockIdx.x * RPW + threadIdx.x / TPR;
  const bool there = row < a.rows;
  const int64_t r = there ? row : a.rows - 1;  // (all lanes take part in the sums)
  const int at0 = threadIdx.x % TPR * VEC;
  u32x4_t hv[NV], yv[NV], gates[NV];
  const auto load = [&](u32x4_t (&to)[NV], int v, const void *p, int64_t stride) {
    to[v] = u32x4_t{0, 0, 0, 0};
    if (p && at0 + v * STEP < a.d) to[v] = Chunk<T, WHOLE>::load(p, r * stride, at0 + v * STEP, a.d);
  };
  if constexpr (kEarly<WHOLE, TPR>) {  // (in the order of their use)
#pragma unroll
    for (int v = 0; v < NV; ++v) load(yv, v, a.y, a.sy);
#pragma unroll
    for (int v = 0; v < NV; ++v) load(hv, v, a.h, a.sh);
#pragma unroll
    for (int v = 0; v < NV; ++v) load(gates, v, a.gate, a.sg);
  } else {
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int at = at0 + v * STEP;
      hv[v] = yv[v] = u32x4_t{0, 0, 0, 0};
      if (at < a.d) {
        hv[v] = Chunk<T, WHOLE>::load(a.h, r * a.sh, at, a.d);
        if (a.y) yv[v] = Chunk<T, WHOLE>::load(a.y, r * a.sy, at, a.d);
      }
    }
  }
  Chunk<T, WHOLE> h[NV], y[NV];
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    Vec16<T>::open(hv[v], h[v].f);
    Vec16<T>::open(yv[v], y[v].f);
  }
  if (a.y) {
    if (a.post != kNone) norm_row<T, WHOLE, NV, TPR>(y, a.post, a.eps_post, a.g_post, a.b_post, a.d, a.inv_d, at0, red);
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int at = at0 + v * STEP;
      if (at >= a.d) continue;
      if (!kEarly<WHOLE, TPR>) load(gates, v, a.gate, a.sg);
      float g[VEC];
      if (a.gate) Vec16<T>::open(gates[v], g);
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const float t = a.gate ? y[v].f[e] * g[e] : y[v].f[e];
        h[v].f[e] += a.scale * t;
      }
    }
  }
  if (a.h_out && there)
#pragma unroll
    for (int v = 0; v < NV; ++v)
      if (at0 + v * STEP < a.d) h[v].store(a.h_out, r * a.sho, at0 + v * STEP, a.d);
  if (!a.n_out) return;
  norm_row<T, WHOLE, NV, TPR>(h, a.pre, a.eps_pre, a.g_pre, a.b_pre, a.d, a.inv_d, at0, red);
  if (there)
#pragma unroll
    for (int v = 0; v < NV; ++v)
      if (at0 + v * STEP < a.d) h[v].store(a.n_out, r * a.sno, at0 + v * STEP, a.d);
}

template <typename T, bool WHOLE, int NV, int TPR>
static void launch(const NormArgs &a, hipStream_t stream) {
  constexpr int RPW = wg_threads(TPR) / TPR;
  hipLaunchKernelGGL((block_norm_kernel<T, WHOLE, NV, TPR>), dim3((unsigned)(((int64_t)a.rows + RPW - 1) / RPW)),
                     dim3(wg_threads(TPR)), 0, stream, a);
}

template <typename T, bool WHOLE>
static void launch_block_norm(const NormArgs &a, hipStream_t stream) {
  constexpr int VEC = Vec16<T>::N;
  if (a.d <= 8 * VEC * 2) return launch<T, WHOLE, 2, 8>(a, stream);
  if (a.d <= 32 * VEC * 2) return launch<T, WHOLE, 2, 32>(a, stream);
  if (a.d <= 64 * VEC * 2) return launch<T, WHOLE, 2, 64>(a, stream);
  if (a.d <= 128 * VEC * 2) return launch<T, WHOLE, 2, 128>(a, stream);
  if (a.d <= 256 * VEC * 2) return launch<T, WHOLE, 2, 256>(a, stream);
  if (a.d <= 512 * VEC * 2) return launch<T, WHOLE, 2, 512>(a, stream);
  launch<T, WHOLE, 16 / VEC, 1024>(a, stream);  // d <= 16384: 2 (bf16) or 4 chunks
}

// Rows of a launch: its threads are counted in 32 bits, 1024 a row at most.
constexpr int64_t kLaunchRows = 1 << 21;

static bool norm_ok(const sm_norm *n) {
  return !n || ((n->kind == SM_NORM_RMS || n->kind == SM_NORM_LAYER) && n->eps >= 0.f && std::isfinite(n->eps));
}

}  // namespace sm

using namespace sm;

SM_API sm_status sm_block_norm(const void *h, int64_t h_stride, const void *y, int64_t y_stride, int rows, int d,
                               const sm_norm *post, const void *gate, int64_t gate_stride, float scale,
                               const sm_norm *pre, sm_dtype dt, void *h_out, int64_t h_out_stride, void *n_out,
                               int64_t n_out_stride, hipStream_t stream) {
  if ((dt != SM_F32 && dt != SM_BF16) || rows < 0 || d < 1 || d > 16384) return SM_EINVAL;
  if (!norm_ok(post) || !norm_ok(pre) || !std::isfinite(scale)) return SM_EINVAL;
  if (rows == 0) return SM_OK;
  if (!h || (!h_out && !n_out) || (n_out && !pre)) return SM_EINVAL;
  if (h_stride < d || (y && y_stride < d) || (gate && gate_stride != 0 && gate_stride < d)) return SM_EINVAL;
  if ((h_out && h_out_stride < d) || (n_out && n_out_stride < d) || (h_out && h_out == n_out)) return SM_EINVAL;
  // an output in an input's place lies where that is read
  const auto placed = [&](const void *out, int64_t out_stride) {
    return rows == 1 || !out || ((out != h || out_stride == h_stride) && (out != y || out_stride == y_stride) &&
                                 (out != gate || out_stride == gate_stride));
  };
  if (!placed(h_out, h_out_stride) || !placed(n_out, n_out_stride)) return SM_EINVAL;
  const int es = dt == SM_BF16 ? 2 : 4;
  const auto aligned = [&](const void *p, int64_t stride) { return (uintptr_t)p % 16 == 0 && stride * es % 16 == 0; };
  const bool wide = d * es % 16 == 0 && aligned(h, h_stride) && (!y || aligned(y, y_stride)) &&
                    (!gate || aligned(gate, gate_stride)) && (!h_out || aligned(h_out, h_out_stride)) &&
                    (!n_out || aligned(n_out, n_out_stride)) &&
                    (!post || (aligned(post->gain, 0) && aligned(post->bias, 0))) &&
                    (!pre || (aligned(pre->gain, 0) && aligned(pre->bias, 0)));
  NormArgs a{h, y, gate, post ? post->gain : nullptr, post ? post->bias : nullptr, pre ? pre->gain : nullptr,
             pre ? pre->bias : nullptr, h_out, n_out, h_stride, y_stride, gate_stride, h_out_stride, n_out_stride,
             rows, d, post ? post->kind : kNone, pre ? pre->kind : kNone, scale, post ? post->eps : 0.f,
             pre ? pre->eps : 0.f, (float)(1.0 / d)};
  for (int64_t r = 0; r < rows; r += kLaunchRows) {
    a.h = row_at(h, r, h_stride, es);
    a.y = row_at(y, r, y_stride, es);
    a.gate = row_at(gate, r, gate_stride, es);
    a.h_out = row_at(h_out, r, h_out_stride, es);
    a.n_out = row_at(n_out, r, n_out_stride, es);
    a.rows = (int)std::min(rows - r, kLaunchRows);
    if (dt == SM_BF16) wide ? launch_block_norm<uint16_t, true>(a, stream) : launch_block_norm<uint16_t, false>(a, stream);
    else wide ? launch_block_norm<float, true>(a, stream) : launch_block_norm<float, false>(a, stream);
    if (hipGetLastError() != hipSuccess) return SM_EHIP;
  }
  return SM_OK;
}
