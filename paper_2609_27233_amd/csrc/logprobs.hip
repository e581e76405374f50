// Log probabilities of given tokens, entropy and top alternatives of rows of
// logits (gfx950).
//
// With z = scale x, m = max z and S = sum exp(z - m):
//   log p_v = z_v - m - log S,   entropy = log S - sum (z - m) exp(z - m) / S.
// Alternatives are ordered by one 64-bit key per logit: the value's bits made
// to ascend with it, then the index counted down, so that no two are equal.
#include <cmath>

#include "common.hpp"

namespace sm {

constexpr int kLpThreads = 256;
constexpr float kLn2 = 0.69314718055994531f;

struct LogprobArgs {
  const void *logits;
  int64_t stride;
  int rows, vocab, k;
  float scale, c;  // c: scale x log2 e
  const int32_t *tokens;
  float *logprob, *entropy;
  int32_t *top_ids;
  float *top_logprobs;
  int32_t *err;
};

// Ascends with x; -0 counts as 0, NaN is below everything.
__device__ __forceinline__ uint32_t order_of(float x) {
  if (x != x) return 0;
  const uint32_t b = __float_as_uint(x + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}

__device__ __forceinline__ uint64_t wave_max64(uint64_t v) {
#pragma unroll
  for (int off = 32; off; off >>= 1) {
    const uint64_t u = __shfl_xor(v, off, kWave);
    v = u > v ? u : v;
  }
  return v;
}

template <typename T>
__global__ __launch_bounds__(kLpThreads) void logprobs_kernel(LogprobArgs a) {
  __shared__ float red[kLpThreads / 64];
  __shared__ uint64_t best[kLpThreads / 64];
  const int t = threadIdx.x;
  const int64_t r = blockIdx.x;
  const T *x = (const T *)a.logits + r * a.stride;
  float m = -INFINITY, odd = 0.f;
  for (int v = t; v < a.vocab; v += kLpThreads) {
    const float f = Elem<T>::load(x + v);
    m = fmaxf(m, f);
    if (!(f < INFINITY)) odd = 1.f;  // NaN or +infinity
  }
  m = block_max(m, red);
  odd = block_max(odd, red);
  float S = 0.f, E = 0.f;
  if (m > -INFINITY)
    for (int v = t; v < a.vocab; v += kLpThreads) {
      const float d = (Elem<T>::load(x + v) - m) * a.c, e = __builtin_amdgcn_exp2f(d);
      S += e;
      if (e > 0.f) E += e * d;
    }
  S = block_sum(S, red);
  E = block_sum(E, red);
  const float log_s = __builtin_amdgcn_logf(S);  // base 2
  const float nan = __uint_as_float(0x7fc00000u);
  auto logprob = [&](float f) {
    return odd != 0.f ? nan : f == -INFINITY ? -INFINITY : fmaf(f - m, a.scale, -log_s * kLn2);
  };
  if (t == 0) {
    if (a.entropy) a.entropy[r] = odd != 0.f ? nan : S > 0.f ? (log_s - E / S) * kLn2 : 0.f;
    if (a.logprob) {
      const int tok = a.tokens[r];
      float lp = 0.f;
      if (tok >= 0 && tok < a.vocab) lp = logprob(Elem<T>::load(x + tok));
      else if (tok != -1 && a.err) set_err(a.err, SM_ERR_EINVAL);
      a.logprob[r] = lp;
    }
  }
  uint64_t below = ~0ull;
  for (int i = 0; i < a.k; ++i) {
    uint64_t top = 0;
    for (int v = t; v < a.vocab; v += kLpThreads) {
      const uint64_t key = (uint64_t)order_of(Elem<T>::load(x + v)) << 32 | (uint32_t)~v;
      if (key < below && key > top) top = key;
    }
    top = wave_max64(top);
    __syncthreads();
    if ((t & 63) == 0) best[t >> 6] = top;
    __syncthreads();
    for (int w = 0; w < kLpThreads / 64; ++w) top = best[w] > top ? best[w] : top;
    below = top;
    if (t == 0) {
      const int v = (int)~(uint32_t)top;
      a.top_ids[r * a.k + i] = v;
      if (a.top_logprobs) a.top_logprobs[r * a.k + i] = logprob(Elem<T>::load(x + v));
    }
  }
}

}  // namespace sm

using namespace sm;

SM_API size_t sm_token_logprobs_workspace_bytes(int rows, int vocab, int k) {
  if (rows < 0 || vocab < 1 || k < 0 || k > SM_MAX_TOP || k > vocab) return 0;
  return 65536;
}

SM_API sm_status sm_token_logprobs(const void *logits, int64_t stride, int rows, int vocab, sm_dtype dt, float scale,
                                   const int32_t *tokens, float *logprob, float *entropy, int k, int32_t *top_ids,
                                   float *top_logprobs, void *ws, size_t ws_bytes, int32_t *err, hipStream_t stream) {
  if ((dt != SM_F32 && dt != SM_BF16) || rows < 0 || vocab < 1 || k < 0 || k > SM_MAX_TOP || k > vocab) return SM_EINVAL;
  const float c = (float)(scale * 1.4426950408889634);
  if (!(scale > 0.f) || !std::isfinite(c) || stride < vocab) return SM_EINVAL;
  if (rows == 0) return SM_OK;
  if (!logits || (logprob && !tokens) || (k > 0 && !top_ids) || (uintptr_t)ws % 16 != 0) return SM_EINVAL;
  if (!ws || ws_bytes < sm_token_logprobs_workspace_bytes(rows, vocab, k)) return SM_EINVAL;
  const LogprobArgs a{logits, stride, rows, vocab, k, scale, c, tokens, logprob, entropy, top_ids,
                      top_logprobs, err};
  if (dt == SM_BF16)
    hipLaunchKernelGGL(logprobs_kernel<uint16_t>, dim3(rows), dim3(kLpThreads), 0, stream, a);
  else
    hipLaunchKernelGGL(logprobs_kernel<float>, dim3(rows), dim3(kLpThreads), 0, stream, a);
  return hipGetLastError() == hipSuccess ? SM_OK : SM_EHIP;
}
