// The residual stream past one block with the norms around it (gfx950):
//   h_out = h + scale gate norm_post(y),  n_out = norm_pre(h_out).
//
// Each row is read and written once: the row's features stay in registers
// (fp32) between the norms, so both norms, the gate and the sum cost no
// traffic beyond h, y, h_out and n_out, which bound the call.  LayerNorm
// takes its mean first and sums squares of the differences from registers.
#include <cmath>

#include "common.hpp"

namespace sm {

// A norm's kind: kNone leaves the row as it is.
enum { kNone = -1 };

struct NormArgs {
  const void *h, *y, *gate;
  const void *g_post, *b_post, *g_pre, *b_pre;
  void *h_out, *n_out;
  int64_t sh, sy, sg, sho, sno;
  int rows, d, post, pre;
  float scale, eps_post, eps_pre;
};

// Sum over the WPR waves that hold a row; `red`: WPR floats of the row's own.
template <int WPR>
__device__ __forceinline__ float row_sum(float v, float *red) {
  v = wave_sum(v);
  if constexpr (WPR > 1) {
    const int w = (threadIdx.x >> 6) % WPR;
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[w] = v;
    __syncthreads();
    v = 0.f;
#pragma unroll
    for (int i = 0; i < WPR; ++i) v += red[i];
  }
  return v;
}

template <typename T, int VEC>
struct Chunk {  // VEC features at once
  float f[VEC];
  __device__ __forceinline__ void load(const void *p, int64_t at) {
    if constexpr (VEC == 1) {
      f[0] = Elem<T>::load((const T *)p + at);
    } else if constexpr (sizeof(T) == 4) {
      const u32x4_t v = *(const u32x4_t *)((const T *)p + at);
#pragma unroll
      for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(v[i]);
    } else {
      const u32x4_t v = *(const u32x4_t *)((const T *)p + at);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        f[2 * i] = __uint_as_float(v[i] << 16);
        f[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u);
      }
    }
  }
  __device__ __forceinline__ void store(void *p, int64_t at) const {
    if constexpr (VEC == 1) {
      ((T *)p)[at] = Elem<T>::to_store(f[0]);
    } else if constexpr (sizeof(T) == 4) {
      *(u32x4_t *)((T *)p + at) = u32x4_t{__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]),
                                          __float_as_uint(f[3])};
    } else {
      *(u32x4_t *)((T *)p + at) = u32x4_t{pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]),
                                          pack_bf16x2(f[6], f[7])};
    }
  }
};

// x <- norm(x), the row spread over WPR waves, NV chunks a thread.
template <typename T, int VEC, int NV, int WPR>
__device__ __forceinline__ void norm_row(Chunk<T, VEC> (&x)[NV], int kind, float eps, const void *gain, const void *bias,
                                         int d, int lane0, float *red) {
  constexpr int STEP = 64 * WPR * VEC;
  float mean = 0.f;
  if (kind == SM_NORM_LAYER) {
    float s = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int e = 0; e < VEC; ++e) s += x[v].f[e];  // (chunks past d hold zeros)
    mean = row_sum<WPR>(s, red) / d;
  }
  float q = 0.f;
#pragma unroll
  for (int v = 0; v < NV; ++v)
    if (lane0 + v * STEP < d)
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        x[v].f[e] -= mean;
        q += x[v].f[e] * x[v].f[e];
      }
  const float inv = 1.f / sqrtf(row_sum<WPR>(q, red) / d + eps);
#pragma unroll
  for (int v = 0; v < NV; ++v)
    if (lane0 + v * STEP < d) {
      Chunk<T, VEC> g, b;
      if (gain) g.load(gain, lane0 + v * STEP);
      if (bias) b.load(bias, lane0 + v * STEP);
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        float n = x[v].f[e] * inv;
        if (gain) n *= g.f[e];
        if (bias) n += b.f[e];
        x[v].f[e] = n;
      }
    }
}

constexpr int wg_threads(int wpr) { return wpr < 4 ? 256 : 64 * wpr; }

// WPR waves hold a row, NV chunks of VEC features a thread.
template <typename T, int VEC, int NV, int WPR>
__global__ __launch_bounds__(wg_threads(WPR)) void block_norm_kernel(NormArgs a) {
  constexpr int RPW = wg_threads(WPR) / (64 * WPR);  // rows per workgroup
  constexpr int STEP = 64 * WPR * VEC;
  __shared__ float red[WPR];  // (several waves to a row: one row per workgroup)
  const int64_t r = (int64_t)blockIdx.x * RPW + threadIdx.x / (64 * WPR);
  if (r >= a.rows) return;  // (whole waves, and never a part of a row)
  const int lane0 = threadIdx.x % (64 * WPR) * VEC;
  Chunk<T, VEC> h[NV], y[NV];
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int at = lane0 + v * STEP;
#pragma unroll
    for (int e = 0; e < VEC; ++e) h[v].f[e] = y[v].f[e] = 0.f;
    if (at < a.d) {
      h[v].load(a.h, r * a.sh + at);
      if (a.y) y[v].load(a.y, r * a.sy + at);
    }
  }
  if (a.y) {
    if (a.post != kNone) norm_row<T, VEC, NV, WPR>(y, a.post, a.eps_post, a.g_post, a.b_post, a.d, lane0, red);
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int at = lane0 + v * STEP;
      if (at >= a.d) continue;
      Chunk<T, VEC> g;
      if (a.gate) g.load(a.gate, r * a.sg + at);
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const float t = a.gate ? y[v].f[e] * g.f[e] : y[v].f[e];
        h[v].f[e] += a.scale * t;
      }
    }
  }
  if (a.h_out)
#pragma unroll
    for (int v = 0; v < NV; ++v)
      if (lane0 + v * STEP < a.d) h[v].store(a.h_out, r * a.sho + lane0 + v * STEP);
  if (!a.n_out) return;
  norm_row<T, VEC, NV, WPR>(h, a.pre, a.eps_pre, a.g_pre, a.b_pre, a.d, lane0, red);
#pragma unroll
  for (int v = 0; v < NV; ++v)
    if (lane0 + v * STEP < a.d) h[v].store(a.n_out, r * a.sno + lane0 + v * STEP);
}

template <typename T, int VEC, int NV, int WPR>
static void launch(const NormArgs &a, hipStream_t stream) {
  constexpr int RPW = wg_threads(WPR) / (64 * WPR);
  hipLaunchKernelGGL((block_norm_kernel<T, VEC, NV, WPR>), dim3((unsigned)(((int64_t)a.rows + RPW - 1) / RPW)),
                     dim3(wg_threads(WPR)), 0, stream, a);
}

template <typename T>
static void launch_block_norm(const NormArgs &a, bool wide, hipStream_t stream) {
  constexpr int VEC = 16 / sizeof(T);
  if (wide) {
    if (a.d <= 64 * VEC * 2) return launch<T, VEC, 2, 1>(a, stream);
    if (a.d <= 256 * VEC * 2) return launch<T, VEC, 2, 4>(a, stream);
    if (a.d <= 512 * VEC * 2) return launch<T, VEC, 2, 8>(a, stream);
    return launch<T, VEC, 16 / VEC, 16>(a, stream);  // 1024 threads: 2 (bf16) or 4 chunks each
  }
  if (a.d <= 64 * 16) return launch<T, 1, 16, 1>(a, stream);
  if (a.d <= 256 * 16) return launch<T, 1, 16, 4>(a, stream);
  launch<T, 1, 16, 16>(a, stream);
}

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
  if ((h_out && h_out_stride < d) || (n_out && n_out_stride < d)) return SM_EINVAL;
  const int64_t es = dt == SM_BF16 ? 2 : 4;
  const auto aligned = [&](const void *p, int64_t stride) { return (uintptr_t)p % 16 == 0 && stride * es % 16 == 0; };
  const bool wide = d * es % 16 == 0 && aligned(h, h_stride) && (!y || aligned(y, y_stride)) &&
                    (!gate || aligned(gate, gate_stride)) && (!h_out || aligned(h_out, h_out_stride)) &&
                    (!n_out || aligned(n_out, n_out_stride)) &&
                    (!post || (aligned(post->gain, 0) && aligned(post->bias, 0))) &&
                    (!pre || (aligned(pre->gain, 0) && aligned(pre->bias, 0)));
  NormArgs a{h, y, gate, post ? post->gain : nullptr, post ? post->bias : nullptr, pre ? pre->gain : nullptr,
             pre ? pre->bias : nullptr, h_out, n_out, h_stride, y_stride, gate_stride, h_out_stride, n_out_stride,
             rows, d, post ? post->kind : kNone, pre ? pre->kind : kNone, scale, post ? post->eps : 0.f,
             pre ? pre->eps : 0.f};
  if (dt == SM_BF16) launch_block_norm<uint16_t>(a, wide, stream);
  else launch_block_norm<float>(a, wide, stream);
  return hipGetLastError() == hipSuccess ? SM_OK : SM_EHIP;
}
