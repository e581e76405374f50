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
// One workgroup takes a row.  It finds M.  A filter looks for the value at
// which its start of the tokens ends: a histogram over M - x in 32-bit
// integers, of counts (top-k, exact) or of masses to 2^-14 of themselves
// (top-p), names a bin or two; one pass in full precision takes the mass above
// them, and their tokens into a list, which is cut by its values until one is
// left.  The kept masses of the pieces of 512 tokens are scanned, and the piece
// that the random number falls into is looked at token by token.
#include <algorithm>
#include <cmath>

#include "common.hpp"

namespace sm {

constexpr int kSampThreads = 1024, kSampWaves = kSampThreads / 64;
constexpr int kPiece = 512;                    // tokens of a piece: 8 a lane
constexpr int kMostVocab = 1 << 19;            // a mass of 2^44 times this many fits 63 bits
constexpr int kMostPieces = kMostVocab / kPiece;
constexpr int kBins = 2048;
constexpr float kBinsPerLog2 = 16.f;           // bins of a factor of 2
constexpr int kList = 4096;                    // tokens that are cut in LDS
constexpr int kUnit = 44;                      // a weight of 1 is 2^44
constexpr double kLeast = -46.0;               // exponents from here down weigh nothing
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

// 2^t for t <= 0 in multiples of 2^-44; 0 from 2^-46 on.  table: 2^(j / 128).
// t = k / 128 + r, |r| <= 2^-8, 2^r = e^(r ln 2) to its fourth power: the next
// term is below 2^-49.
__device__ __forceinline__ uint64_t unit_weight(double t, const double *table) {
  constexpr double ln2 = 0.69314718055994530941723212145818;
  constexpr double c1 = ln2, c2 = c1 * ln2 / 2, c3 = c2 * ln2 / 3, c4 = c3 * ln2 / 4;
  constexpr double magic = 6755399441055744.0;  // 1.5 x 2^52: a sum with it is a whole number in its low bits
  const double sum = fma(t, 128.0, magic);
  const int k = (int)__double_as_longlong(sum);
  const double r = fma(sum - magic, -0.0078125, t);
  double p = fma(r, c4, c3);
  p = fma(r, p, c2);
  p = fma(r, p, c1);
  p = fma(r, p, 1.0);
  const double w = ldexp(table[k & 127] * p, (k >> 7) + kUnit) + 4503599627370496.0;  // to nearest
  return t < kLeast ? 0 : __double_as_longlong(w) & 0xfffffffffffffll;
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

__device__ __forceinline__ double block_scan_f64(double v, double *red) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const double u = __shfl_up(v, d, kWave);
    if (lane >= d) v += u;
  }
  if (lane == 63) red[w] = v;
  __syncthreads();
  double before = 0;
  for (int i = 0; i < w; ++i) before += red[i];
  __syncthreads();
  return v + before;
}

struct SampleShared {
  uint64_t mass[kBins];          // of a cut's bins, or of the pieces
  uint32_t count[kBins];         // of a cut's bins, or of the pieces' ties
  uint64_t list[kList];          // key << 32 | token
  double table[128];
  uint64_t red[kSampWaves];
  float fred[kSampWaves];
  uint64_t before;               // mass (or count) above the bin
  int bin, last, bad, listed;
  uint32_t klo, khi;
  uint64_t above;
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
  float bin_scale;

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
  // How far below M, in bins; descends as v ascends.
  __device__ __forceinline__ float depth(float v) const { return (M - v) * bin_scale; }
  __device__ __forceinline__ int bin(float v) const {
    const float d = depth(v);
    return d < (float)(kBins - 1) ? (int)d : kBins - 1;
  }
  // The masses of this lane's tokens in piece p above the tie, and which are equal to it.
  __device__ __forceinline__ void weights(int p, const Kept &kept, const double *table, uint64_t (&m)[8], uint32_t &tied) const {
    float f[8];
    load(p, f);
    tied = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t key = order_key(f[e]);
      m[e] = 0;
      if (f[e] > -INFINITY && key > kept.tie) {
        const double ex = exponent(f[e]);
        if (ex >= lm) m[e] = unit_weight(ex, table);
      }
      tied |= (uint32_t)(kept.ties > 0 && key == kept.tie && f[e] > -INFINITY) << e;
    }
  }
  // f(value, token) of the tokens of this wave's pieces
  template <class F>
  __device__ __forceinline__ void each(F f) const {
    for (int p = threadIdx.x >> 6; p < pieces(); p += kSampWaves) {
      float v[8];
      load(p, v);
#pragma unroll
      for (int e = 0; e < 8; ++e) f(v[e], p * kPiece + 8 * (int)(threadIdx.x & 63) + e);
    }
  }
};

// What a cut looks at: the tokens of a row with keys above the tie, or those of
// them that are listed (a range of bins, complete).
template <typename T>
struct Tokens {
  const Row<T> &row;
  const SampleShared &sh;
  Kept kept;
  bool listed;
  template <class F>
  __device__ __forceinline__ void each(F f) const {  // f(value, key)
    if (listed) {
      for (int i = threadIdx.x; i < sh.listed; i += kSampThreads) {
        const uint32_t key = (uint32_t)(sh.list[i] >> 32);
        f(value_of_key(key), key);
      }
    } else {
      row.each([&](float v, int) {
        const uint32_t key = order_key(v);
        if (v > -INFINITY && key > kept.tie && row.exponent(v) >= row.lm) f(v, key);
      });
    }
  }
};

// The smallest start of these tokens in descending order at which `before`
// plus their amount (MASS: of their masses; else their number) reaches the
// target; ties: how many more of the tie's value there are (the last of all).
// All threads; returns the same in each.  Rounds of 2048 bins, the first by
// M - x, the others by keys, until a single value is left.
template <bool MASS, typename T>
__device__ Kept cut(const Row<T> &row, const Tokens<T> &tokens, uint64_t before, double target, bool tie_in, SampleShared &sh) {
  const int t = threadIdx.x;
  const Kept kept = tokens.kept;
  const auto amount = [&](float v) { return MASS ? unit_weight(row.exponent(v), sh.table) : (uint64_t)1; };
  const float tie_value = value_of_key(kept.tie);
  uint32_t klo = 0, khi = 0;
  int shift = -1, bin = 0;
  for (;;) {
    for (int i = t; i < kBins; i += kSampThreads) sh.mass[i] = sh.count[i] = 0;
    if (t == 0) sh.bin = kBins;
    __syncthreads();
    const auto place = [&](float v, uint32_t key) { return shift < 0 ? row.bin(v) : (int)((khi - key) >> shift); };
    const auto inside = [&](float v, uint32_t key) { return shift < 0 || (key >= klo && key <= khi && row.bin(v) == bin); };
    tokens.each([&](float v, uint32_t key) {
      if (!inside(v, key)) return;
      const int b = place(v, key);
      atomicAdd(&sh.count[b], 1u);
      if constexpr (MASS) atomicAdd((unsigned long long *)&sh.mass[b], amount(v));
    });
    if (t == 0 && tie_in && inside(tie_value, kept.tie)) {
      const int b = place(tie_value, kept.tie);
      atomicAdd(&sh.count[b], (uint32_t)kept.ties);
      if constexpr (MASS) atomicAdd((unsigned long long *)&sh.mass[b], kept.ties * amount(tie_value));
    }
    __syncthreads();
    uint64_t mine[2], total;
#pragma unroll
    for (int i = 0; i < 2; ++i) mine[i] = MASS ? sh.mass[2 * t + i] : sh.count[2 * t + i];
    const uint64_t end = block_scan64(mine[0] + mine[1], sh.red, &total) + before;
    total += before;
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
    if (b >= kBins) return kept;  // no tokens
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
    tokens.each(see);
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

// Adds token (key, index) to the list; past its end only the count goes on.
__device__ __forceinline__ void list_token(SampleShared &sh, uint32_t key, int token) {
  const int at = atomicAdd(&sh.listed, 1);
  if (at < kList) sh.list[at] = (uint64_t)key << 32 | (uint32_t)token;
}

// The first k tokens (lower index first among equal ones).
template <typename T>
__device__ Kept first_k(const Row<T> &row, int k, SampleShared &sh) {
  const int t = threadIdx.x;
  const Kept all{0, 0};
  for (int i = t; i < kBins; i += kSampThreads) sh.count[i] = 0;
  if (t == 0) {
    sh.bin = kBins;
    sh.listed = 0;
  }
  __syncthreads();
  row.each([&](float v, int) {
    if (v > -INFINITY) atomicAdd(&sh.count[row.bin(v)], 1u);
  });
  __syncthreads();
  const uint32_t c0 = sh.count[2 * t], c1 = sh.count[2 * t + 1];
  uint64_t total;
  const uint64_t end = block_scan64(c0 + c1, sh.red, &total);
  if (total <= (uint64_t)k) return all;  // (-infinity has no place)
  if (end >= (uint64_t)k && end - c0 - c1 < (uint64_t)k) {
    const bool second = end - c1 < (uint64_t)k;
    sh.bin = 2 * t + second;
    sh.before = end - c1 - (second ? 0 : c0);
  }
  __syncthreads();
  const int b = sh.bin;
  const uint64_t before = sh.before;
  row.each([&](float v, int token) {
    if (v > -INFINITY && row.bin(v) == b) list_token(sh, order_key(v), token);
  });
  __syncthreads();
  const bool listed = sh.listed <= kList;
  return cut<false>(row, Tokens<T>{row, sh, all, listed}, listed ? before : 0, (double)k, false, sh);
}

// The start of the kept tokens before whose last lies less than `part` of their
// mass.  True: the pieces' kept masses and ties are in sh.mass and sh.count.
template <typename T>
__device__ bool first_mass(const Row<T> &row, Kept &kept, double part, SampleShared &sh) {
  const int t = threadIdx.x, w = t >> 6, lane = t & 63, pieces = row.pieces();
  const float tie_value = value_of_key(kept.tie);
  const uint64_t tie_each = kept.ties > 0 ? unit_weight(row.exponent(tie_value), sh.table) : 0;
  // a bin's masses as parts of its largest, in whole numbers of `bits` bits: no sum of them passes 32
  int bits = 31;
  while (bits > 0 && (row.vocab - 1) >> (31 - bits)) --bits;
  const float one = (float)(1 << bits), least = -(float)kLeast * kBinsPerLog2;
  for (int i = t; i < kBins; i += kSampThreads) sh.count[i] = 0;
  if (t == 0) {
    sh.bin = sh.last = kBins;
    sh.listed = 0;
    sh.above = 0;
  }
  __syncthreads();
  const float floor_depth = row.lm > -INFINITY ? (float)-row.lm * kBinsPerLog2 : INFINITY;
  const auto approximate = [&](float v) {
    const float d = row.depth(v), b = floorf(d);
    if (d < least && d <= floor_depth)
      atomicAdd(&sh.count[(int)b], (uint32_t)(__builtin_amdgcn_exp2f((b - d) * (1.f / kBinsPerLog2)) * one + 0.5f));
  };
  row.each([&](float v, int) {
    if (order_key(v) > kept.tie) approximate(v);  // (-infinity is too deep)
  });
  __syncthreads();
  // Bin b's largest weight is 2^(-b / 16).  The slack is what the roundings come
  // to as a rule; where they come to more, the masses below tell.
  double mine[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) mine[i] = (double)sh.count[2 * t + i] * exp2((double)-(2 * t + i) / kBinsPerLog2) / one;
  if (kept.ties > 0) {
    const float d = row.depth(tie_value);
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (d < least && (int)d == 2 * t + i) mine[i] += (double)(kept.ties * tie_each) * 0x1p-44;
  }
  const double end = block_scan_f64(mine[0] + mine[1], (double *)sh.red);
  if (t == kSampThreads - 1) *(double *)&sh.before = end;
  __syncthreads();
  const double all = *(double *)&sh.before, slack = 0.5 / one + 1e-6, target_a = part * all;
  const double ends[2] = {end - mine[1], end};
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    if (ends[i] >= target_a - slack * all) atomicMin(&sh.bin, 2 * t + i);
    if (ends[i] >= target_a + slack * all) atomicMin(&sh.last, 2 * t + i);
  }
  __syncthreads();
  // ---- the masses above the bins in which the end lies, and their tokens ----
  const int b1 = sh.bin, b2 = sh.last;
  uint64_t S = 0;
  for (int p = w; p < pieces; p += kSampWaves) {
    uint64_t m[8], above = 0;
    float f[8];
    row.load(p, f);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t key = order_key(f[e]);
      m[e] = 0;
      if (f[e] > -INFINITY && key > kept.tie) {
        const double ex = row.exponent(f[e]);
        if (ex >= row.lm) {
          m[e] = unit_weight(ex, sh.table);
          const int b = row.bin(f[e]);
          if (b < b1) above += m[e];
          else if (b <= b2) list_token(sh, key, p * kPiece + 8 * lane + e);
        }
      }
      S += m[e];
    }
    above = wave_sum64(above);
    if (lane == 0) sh.mass[p] = above;
  }
  S = wave_sum64(S);
  if (lane == 0) atomicAdd((unsigned long long *)&sh.above, S);
  __syncthreads();
  S = sh.above + kept.ties * tie_each;
  uint64_t above;
  {
    const uint64_t a = t < pieces ? sh.mass[t] : 0;
    block_scan64(a, sh.red, &above);
    __syncthreads();
    // (the cut's bins take the place of the pieces)
    const double target = part * (double)S;
    const int tie_bin = kept.ties > 0 ? row.bin(tie_value) : kBins;
    const bool tie_above = tie_bin < b1, tie_in = tie_bin >= b1 && tie_bin <= b2;
    if (tie_above) above += kept.ties * tie_each;
    uint64_t inside = 0, rest;
    const bool whole = sh.listed <= kList;
    if (whole)
      for (int i = t; i < sh.listed; i += kSampThreads)
        inside += unit_weight(row.exponent(value_of_key((uint32_t)(sh.list[i] >> 32))), sh.table);
    if (t == 0 && tie_in) inside += kept.ties * tie_each;
    block_scan64(inside, sh.red, &rest);
    if (!whole || (double)above >= target || (double)(above + rest) < target) {
      kept = cut<true>(row, Tokens<T>{row, sh, kept, false}, 0, target, kept.ties > 0, sh);
      return false;
    }
    const Kept was = kept;
    kept = cut<true>(row, Tokens<T>{row, sh, was, true}, above, target, tie_in, sh);
    __syncthreads();
    for (int i = t; i < kBins; i += kSampThreads) sh.count[i] = 0;
    sh.mass[t] = a;
    __syncthreads();
    for (int i = t; i < sh.listed; i += kSampThreads) {
      const uint32_t key = (uint32_t)(sh.list[i] >> 32), token = (uint32_t)sh.list[i];
      if (key > kept.tie)
        atomicAdd((unsigned long long *)&sh.mass[token / kPiece], unit_weight(row.exponent(value_of_key(key)), sh.table));
      else if (key == kept.tie) atomicAdd(&sh.count[token / kPiece], 1u);
    }
    __syncthreads();
    return kept.tie != was.tie;  // (the tokens of the tie itself are not listed)
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
  if (t < 128) sh.table[t] = exp2(t / 128.0);
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
  row.bin_scale = kBinsPerLog2 * (float)row.c;
  // ---- the filters ----
  Kept kept{0, 0};  // (no finite logit has key 0)
  const double lm = min_p > 0.f ? log2((double)min_p) : -INFINITY;
  row.lm = -INFINITY;  // (the first k whatever they weigh)
  if (temp == 0.f || top_k == 1) kept = Kept{order_key(M), 1};
  else if (top_k > 0 && top_k < a.vocab) kept = first_k(row, top_k, sh);
  row.lm = lm;
  if (kept.ties > 0 && row.exponent(value_of_key(kept.tie)) < row.lm) kept.ties = 0;
  bool have_pieces = false;
  if (top_p < 1.f && temp > 0.f && top_k != 1) have_pieces = first_mass(row, kept, (double)top_p, sh);
  // ---- kept masses of the pieces ----
  const float tie_value = value_of_key(kept.tie);
  const uint64_t each = kept.ties > 0 ? unit_weight(row.exponent(tie_value), sh.table) : 0;
  const int pieces = row.pieces();
  __syncthreads();
  if (!have_pieces) {
    for (int p = w; p < pieces; p += kSampWaves) {
      uint64_t m[8], sum = 0;
      uint32_t tied;
      row.weights(p, kept, sh.table, m, tied);
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
  }
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
  row.weights(sh.bin, kept, sh.table, m, ties);
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
