// A token from each row of logits, under temperature, top-k, min-p and top-p,
// by one given random number a row (gfx950).
//
// With the largest logit M, a token weighs w = exp((x - M) / T).  Each filter
// keeps a start of the tokens in descending order (the lower index first among
// equal logits): the first k; of those the ones with w >= min_p; of those the
// ones with less than top_p of the mass before them.  So what is kept is
// "every logit above a value, and the first few of those equal to it", and the
// token is the first, in the order of the vocabulary, at which the cumulative
// kept mass passes u times the whole of it.
//
// A token is a whole number: masses have to be right to far less than a
// token's share.  A weight is formed in double precision (a table of 64 and a
// polynomial, off by 2^-50) and rounded to a multiple of 2^-44; masses are
// 64-bit integers.  Their sums are exact and the same in any order, so that
// workgroups, waves and atomics may add them as they come.  Over 128,256
// tokens the roundings come to about 2^-37 of the largest weight.
//
// One workgroup takes a row.  It finds M; a histogram over (M - x), 2048 bins,
// of counts (top-k) or masses (top-p) names the bin in which the last kept
// token lies, and the bin's values are cut in turn until one value is left;
// the kept mass of each piece of 512 tokens is scanned, and the piece that the
// random number falls into is looked at token by token.
#include <algorithm>
#include <cmath>

#include "common.hpp"

namespace sm {

constexpr int kSampThreads = 1024, kSampWaves = kSampThreads / 64;
constexpr int kPiece = 512;                    // tokens of a piece: 8 a lane
constexpr int kMostVocab = 1 << 19;            // a mass of 2^44 times this many fits 63 bits
constexpr int kMostPieces = kMostVocab / kPiece;
constexpr int kBins = 2048;
constexpr int kUnit = 44;                      // a weight of 1 is 2^44
constexpr double kLog2eD = 1.4426950408889634073599246810019;

struct SampleArgs {
  const void *logits;
  int64_t stride;
  int rows, vocab;
  const float *u, *temperature, *top_p, *min_p;
  const int32_t *top_k;
  int32_t *tokens;
  float *logprob;
  int32_t *err;
  int64_t first;  // row of the launch's first workgroup
};

// Ascends with x; -0 counts as 0.
__device__ __forceinline__ uint32_t order_key(float x) {
  const uint32_t b = __float_as_uint(x + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of_key(uint32_t o) { return __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o); }

// 2^t for t <= 0 in multiples of 2^-44; 0 from 2^-46 on.  table: 2^(j / 64).
__device__ __forceinline__ uint64_t unit_weight(double t, const double *table) {
  if (t < -46.0) return 0;
  const double k = rint(t * 64.0);
  const double r = (t - k * 0.015625) * 0.69314718055994530941723212145818;  // |r| <= 0.0055
  const int i = (int)k;
  // e^r to 2^-53: the next term, r^6 / 720, is below 4e-17
  double p = fma(r, 1.0 / 120, 1.0 / 24);
  p = fma(r, p, 1.0 / 6);
  p = fma(r, p, 0.5);
  p = fma(r, p, 1.0);
  p = fma(r, p, 1.0);
  const double w = ldexp(table[i & 63] * p, (i >> 6) + kUnit);
  return __double_as_longlong(w + 4503599627370496.0) & 0xfffffffffffffll;  // to nearest
}

__device__ __forceinline__ uint64_t shfl_xor64(uint64_t v, int m) {
  const uint32_t lo = __shfl_xor((uint32_t)v, m, kWave), hi = __shfl_xor((uint32_t)(v >> 32), m, kWave);
  return (uint64_t)hi << 32 | lo;
}
__device__ __forceinline__ uint64_t wave_sum64(uint64_t v) {
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) v += shfl_xor64(v, m);
  return v;
}
__device__ __forceinline__ uint64_t wave_scan64(uint64_t v) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t lo = __shfl_up((uint32_t)v, d, kWave), hi = __shfl_up((uint32_t)(v >> 32), d, kWave);
    if (lane >= d) v += (uint64_t)hi << 32 | lo;
  }
  return v;
}
// Inclusive over the workgroup; red: one value a wave.  The last barrier lets red be used again.
__device__ __forceinline__ uint64_t block_scan64(uint64_t v, uint64_t *red, uint64_t *total) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  v = wave_scan64(v);
  if (lane == 63) red[w] = v;
  __syncthreads();
  uint64_t before = 0, all = 0;
  for (int i = 0; i < kSampWaves; ++i) {
    if (i < w) before += red[i];
    all += red[i];
  }
  __syncthreads();
  *total = all;
  return v + before;
}

struct SampleShared {
  uint64_t mass[kBins];          // then the pieces' masses
  uint32_t count[kBins];         // then the pieces' ties
  double table[64];
  uint64_t red[kSampWaves];
  float fred[kSampWaves];
  uint64_t before;               // mass (or count) above the bin
  int bin, bad;
  uint32_t klo, khi;
};
static_assert(kMostPieces <= kSampThreads && kMostPieces <= kBins, "a piece a thread");

// A row, or what is left of it: tokens with keys above `tie`, and `ties` of those equal to it.
struct Kept {
  uint32_t tie;
  uint64_t ties;
};

template <typename T>
struct Row {
  const T *x;
  int vocab;
  float M;
  double c;    // log2 e / temperature
  double lm;   // log2 min_p (least exponent that is kept)

  // The eight logits of this lane in piece p, -infinity behind the last.
  __device__ __forceinline__ void load(int p, float (&f)[8]) const {
    const int at = p * kPiece + 8 * (threadIdx.x & 63);
    if (at + 8 <= vocab) {
      T t[8];
      __builtin_memcpy(t, x + at, sizeof t);  // (any element-aligned address)
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = Elem<T>::load(t + e);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = at + e < vocab ? Elem<T>::load(x + at + e) : -INFINITY;
    }
  }
  __device__ __forceinline__ double exponent(float v) const { return ((double)v - (double)M) * c; }
  __device__ __forceinline__ int pieces() const { return (vocab + kPiece - 1) / kPiece; }
  __device__ __forceinline__ int bin(float v) const {  // descends as v ascends
    const float d = (M - v) * 16.f * 1.44269504f;
    return d < (float)(kBins - 1) ? (int)d : kBins - 1;
  }
};

// The smallest start of the kept tokens in descending order whose amount
// (MASS: of their masses; else their number) reaches `part` of all of it (MASS) or
// `part` itself.  All threads; returns the same in each.
template <bool MASS, typename T>
__device__ Kept cut(const Row<T> &row, Kept kept, double part, SampleShared &sh) {
  const int t = threadIdx.x, w = t >> 6;
  // what a token adds, for keys above the tie and exponents that min_p keeps
  const auto amount = [&](float v, double e) { return MASS ? unit_weight(e, sh.table) : (uint64_t)1; };
  const float tie_value = value_of_key(kept.tie);
  const bool tie_in = kept.ties > 0 && row.exponent(tie_value) >= row.lm;
  const uint64_t tie_amount = tie_in ? kept.ties * amount(tie_value, row.exponent(tie_value)) : 0;
  double target = part;
  uint32_t klo = 0, khi = 0;
  uint64_t before = 0;
  int shift = -1, bin = 0;  // round 0 goes by bins of M - x, the others by keys from klo on
  for (;;) {
    for (int i = t; i < kBins; i += kSampThreads) sh.mass[i] = sh.count[i] = 0;
    __syncthreads();
    const auto place = [&](float v, uint32_t key) {
      return shift < 0 ? row.bin(v) : (int)((khi - key) >> shift);
    };
    const auto inside = [&](float v, uint32_t key) { return shift < 0 || (row.bin(v) == bin && key >= klo && key <= khi); };
    for (int p = w; p < row.pieces(); p += kSampWaves) {
      float f[8];
      row.load(p, f);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t key = order_key(f[e]);
        if (!(f[e] > -INFINITY) || key <= kept.tie || !inside(f[e], key)) continue;
        const double ex = row.exponent(f[e]);
        if (ex < row.lm) continue;
        const int b = place(f[e], key);
        atomicAdd(&sh.count[b], 1u);
        if constexpr (MASS) atomicAdd((unsigned long long *)&sh.mass[b], amount(f[e], ex));
      }
    }
    if (t == 0 && tie_in && inside(tie_value, kept.tie)) {
      const int b = place(tie_value, kept.tie);
      atomicAdd(&sh.count[b], (uint32_t)kept.ties);
      if constexpr (MASS) atomicAdd((unsigned long long *)&sh.mass[b], tie_amount);
    }
    if (t == 0) sh.bin = kBins;
    __syncthreads();
    uint64_t mine[2], total;
#pragma unroll
    for (int i = 0; i < 2; ++i) mine[i] = MASS ? sh.mass[2 * t + i] : sh.count[2 * t + i];
    const uint64_t end = block_scan64(mine[0] + mine[1], sh.red, &total) + before;
    total += before;
    if (shift < 0 && MASS) target = part * (double)total;
    // the first bin with a token at which the target is reached, or the last with one
    const uint64_t ends[2] = {end - mine[1], end};
#pragma unroll
    for (int i = 1; i >= 0; --i)
      if (sh.count[2 * t + i] && ((double)ends[i] >= target || ends[i] == total)) atomicMin(&sh.bin, 2 * t + i);
    if (t == 0) {
      sh.klo = 0xffffffffu;
      sh.khi = 0;
    }
    __syncthreads();
    const int b = sh.bin;
    if (b >= kBins) return kept;  // nothing is kept at all
    if (b >> 1 == t) sh.before = ends[b & 1] - mine[b & 1];
    const uint32_t n = sh.count[b];
    const uint64_t sum = MASS ? sh.mass[b] : n;
    // its least and largest key
    uint32_t lo = 0xffffffffu, hi = 0;
    const auto see = [&](float v, uint32_t key) {
      if (!inside(v, key) || place(v, key) != b) return;
      lo = min(lo, key);
      hi = max(hi, key);
    };
    for (int p = w; p < row.pieces(); p += kSampWaves) {
      float f[8];
      row.load(p, f);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t key = order_key(f[e]);
        if (f[e] > -INFINITY && key > kept.tie && row.exponent(f[e]) >= row.lm) see(f[e], key);
      }
    }
    if (t == 0 && tie_in) see(tie_value, kept.tie);
    if (hi) {
      atomicMin(&sh.klo, lo);
      atomicMax(&sh.khi, hi);
    }
    __syncthreads();
    klo = sh.klo;
    khi = sh.khi;
    before = sh.before;
    if (klo == khi) {  // one value: its first few
      const double each = (double)(sum / n), need = (target - (double)before) / each;
      const uint64_t few = each > 0 && need < (double)n ? (need > 1.0 ? (uint64_t)ceil(need) : 1) : n;
      return Kept{klo, few};
    }
    if (shift < 0) bin = b;
    shift = 0;
    while ((khi - klo) >> shift >= (uint32_t)kBins) ++shift;
    __syncthreads();
  }
}

template <typename T>
__global__ __launch_bounds__(kSampThreads) void sample_kernel(SampleArgs a) {
  __shared__ SampleShared sh;
  const int t = threadIdx.x, lane = t & 63, w = t >> 6;
  const int64_t r = a.first + blockIdx.x;
  Row<T> row;
  row.x = (const T *)a.logits + r * a.stride;
  row.vocab = a.vocab;
  if (t < 64) sh.table[t] = exp2(t / 64.0);
  if (t == 0) sh.bad = 0;
  // ---- the largest logit ----
  float M = -INFINITY;
  bool nan = false;
  for (int p = w; p < row.pieces(); p += kSampWaves) {
    float f[8];
    row.load(p, f);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      nan |= f[e] != f[e];
      M = fmaxf(M, f[e]);
    }
  }
  M = wave_max(M);
  if (lane == 0) sh.fred[w] = M;
  __syncthreads();
  for (int i = 0; i < kSampWaves; ++i) M = fmaxf(M, sh.fred[i]);
  if (__ballot(nan) != 0 && lane == 0) sh.bad = 1;
  __syncthreads();
  const float temp = a.temperature ? a.temperature[r] : 1.f, top_p = a.top_p ? a.top_p[r] : 1.f;
  const float min_p = a.min_p ? a.min_p[r] : 0.f, u = a.u[r];
  const int top_k = a.top_k ? a.top_k[r] : 0;
  const bool fine = temp >= 0.f && temp < INFINITY && top_p >= 0.f && min_p >= 0.f && min_p <= 1.f && u >= 0.f && u < 1.f &&
                    top_k >= 0 && !sh.bad && M < INFINITY && M > -INFINITY;
  if (!fine) {
    if (t == 0) {
      a.tokens[r] = -1;
      if (a.logprob) a.logprob[r] = NAN;
      if (a.err) set_err(a.err, SM_ERR_EINVAL);
    }
    return;
  }
  row.M = M;
  row.c = temp > 0.f ? kLog2eD / (double)temp : kLog2eD;
  row.lm = min_p > 0.f ? log2((double)min_p) : -INFINITY;
  // ---- the filters ----
  Kept kept{0, 0};  // (no finite logit has key 0)
  if (temp == 0.f || top_k == 1) kept = Kept{order_key(M), 1};
  else {
    if (top_k > 0 && top_k < a.vocab) {
      const double lm = row.lm;
      row.lm = -INFINITY;  // (the first k whatever they weigh)
      kept = cut<false>(row, kept, (double)top_k, sh);
      row.lm = lm;
    }
    if (top_p < 1.f) kept = cut<true>(row, kept, (double)top_p, sh);
  }
  // ---- kept masses of the pieces ----
  const float tie_value = value_of_key(kept.tie);
  if (kept.ties > 0 && row.exponent(tie_value) < row.lm) kept.ties = 0;
  const uint64_t each = kept.ties > 0 ? unit_weight(row.exponent(tie_value), sh.table) : 0;
  const int pieces = row.pieces();
  __syncthreads();
  const auto weights = [&](int p, uint64_t (&m)[8], uint32_t &tied) {
    float f[8];
    row.load(p, f);
    tied = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t key = order_key(f[e]);
      m[e] = 0;
      if (f[e] > -INFINITY && key > kept.tie) {
        const double ex = row.exponent(f[e]);
        if (ex >= row.lm) m[e] = unit_weight(ex, sh.table);
      }
      tied |= (uint32_t)(kept.ties > 0 && key == kept.tie && f[e] > -INFINITY) << e;
    }
  };
  for (int p = w; p < pieces; p += kSampWaves) {
    uint64_t m[8], sum = 0;
    uint32_t tied;
    weights(p, m, tied);
#pragma unroll
    for (int e = 0; e < 8; ++e) sum += m[e];
    // the number of tied tokens rides above the mass: 2^9 tokens of at most 2^44 each
    sum = wave_sum64(sum + ((uint64_t)__popc(tied) << 54));
    if (lane == 0) {
      sh.mass[p] = sum & ((1ull << 54) - 1);
      sh.count[p] = (uint32_t)(sum >> 54);
    }
  }
  __syncthreads();
  uint64_t all_ties, S;
  const uint64_t tied = t < pieces ? sh.count[t] : 0;
  const uint64_t tied_before = block_scan64(tied, sh.red, &all_ties) - tied;
  const uint64_t mine_ties = tied_before >= kept.ties ? 0 : min(tied, kept.ties - tied_before);
  const uint64_t mine = t < pieces ? sh.mass[t] + mine_ties * each : 0;
  const uint64_t end = block_scan64(mine, sh.red, &S);
  const uint64_t target = (uint64_t)((double)u * (double)S);  // passed by the first cumulative mass above it
  // ---- the piece, then its token ----
  if (end > target && end - mine <= target) {
    sh.bin = t;
    sh.before = end - mine;
    sh.count[0] = (uint32_t)(kept.ties - min(kept.ties, tied_before));  // ties that are left for it
  }
  __syncthreads();
  if (w != 0) return;
  uint64_t m[8], sum = 0;
  uint32_t ties;
  weights(sh.bin, m, ties);
  int ties_before = (int)(wave_scan64(__popc(ties)) - __popc(ties));
  const int left = (int)min(sh.count[0], (uint32_t)kPiece);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    if (ties >> e & 1) {
      if (ties_before < left) m[e] = each;
      ++ties_before;
    }
    sum += m[e];
  }
  uint64_t cum = sh.before + wave_scan64(sum) - sum;
  if (!(cum <= target && target < cum + sum)) return;
  int at = 7;  // (the last one with a mass, at the latest)
#pragma unroll
  for (int e = 7; e >= 0; --e)
    if (cum + sum > target) {  // sum: the masses up to e
      at = e;
      sum -= m[e];
    }
  const int token = sh.bin * kPiece + 8 * lane + at;
  a.tokens[r] = token;
  if (a.logprob) {
    const double ex = row.exponent(Elem<T>::load(row.x + token));
    a.logprob[r] = (float)((ex - (log2((double)S) - kUnit)) / kLog2eD);
  }
}

}  // namespace sm

using namespace sm;

SM_API size_t sm_sample_workspace_bytes(int rows, int vocab) {
  return rows > 0 && vocab > 0 ? 256 : 0;
}

SM_API sm_status sm_sample_tokens(const void *logits, int64_t stride, int rows, int vocab, sm_dtype dt, const float *u,
                                  const float *temperature, const int32_t *top_k, const float *top_p, const float *min_p,
                                  int32_t *tokens, float *logprob, void *ws, size_t ws_bytes, int32_t *err, hipStream_t stream) {
  if ((dt != SM_F32 && dt != SM_BF16) || rows < 0 || vocab < 1 || vocab > kMostVocab || stride < vocab) return SM_EINVAL;
  if (rows == 0) return SM_OK;
  if (!logits || !u || !tokens || !ws || (uintptr_t)ws % 16 || ws_bytes < sm_sample_workspace_bytes(rows, vocab)) return SM_EINVAL;
  SampleArgs a{logits, stride, rows, vocab, u, temperature, top_p, min_p, top_k, tokens, logprob, err, 0};
  constexpr int kLaunchRows = 1 << 20;  // a launch's threads are counted in 32 bits
  for (; a.first < rows; a.first += kLaunchRows) {
    const dim3 grid(std::min<int64_t>(rows - a.first, kLaunchRows));
    if (dt == SM_BF16) hipLaunchKernelGGL(sample_kernel<uint16_t>, grid, dim3(kSampThreads), 0, stream, a);
    else hipLaunchKernelGGL(sample_kernel<float>, grid, dim3(kSampThreads), 0, stream, a);
    if (hipGetLastError() != hipSuccess) return SM_EHIP;
  }
  return SM_OK;
}
