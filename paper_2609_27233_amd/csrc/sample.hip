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
// token's share.  A weight is formed in double precision (a table of 128 and a
// polynomial, off by 2^-49) and rounded to a multiple of 2^-44; masses are
// 64-bit integers.  Their sums are exact and the same in any order, so that
// workgroups, waves and atomics may add them as they come.  Over 128,256
// tokens the roundings come to about 2^-37 of the largest weight.
//
// Three launches, none of which waits inside:
//   scan    M, and a histogram over the logits (2048 bins of 1/23): counts for
//           top-k; for top-p masses in 32-bit integers, right to 2^-14 or so
//   weigh   the histogram names the bin or two in which the filter's last token
//           lies; their tokens are listed, and what is above is weighed in full
//           precision, by pieces of 512 tokens
//   choose  a workgroup a row: the list is cut by its values until one is left,
//           the pieces' masses are scanned, and the piece that the random
//           number falls into is looked at token by token
// A row is read twice, in slices dealt over the device, four 16-byte loads a
// lane in flight.  A row whose list does not suffice (thousands of equal logits
// where the filter ends, a k of thousands, logits hundreds apart) is cut by
// passes over the whole row, in `choose`, to the same result.
#include <algorithm>
#include <cmath>

#include "common.hpp"

namespace sm {

constexpr int kSampThreads = 256, kSampWaves = kSampThreads / 64;
constexpr int kPiece = 512;                    // tokens of a piece: 8 a lane
constexpr int kMostVocab = 1 << 19;            // a mass of 2^44 times this many fits 63 bits
constexpr int kMostPieces = kMostVocab / kPiece;
constexpr int kInFlight = 4;                   // pieces that a wave loads at a time
constexpr int kUnit = 44;                      // a weight of 1 is 2^44
constexpr double kLeast = -46.0;               // exponents from here down weigh nothing
constexpr double kLog2eD = 1.4426950408889634073599246810019;

// The histogram: bins of 1/23 in the logits, the first 512 above the largest
// of the row's first piece.
constexpr int kBins = 2048, kBinsAbove = 512;
constexpr float kBinsPerUnit = 16.f * 1.44269504f;
constexpr float kSharpest = 0.25f;             // temperatures below go by a list of all that weighs anything
constexpr int kList = 4096;                    // tokens that are cut in LDS
constexpr int kCutBins = 1024;

// What a row has in the workspace.  The first part is zero between calls.
struct RowState {
  uint32_t top;       // key of M
  uint32_t bad;       // a NaN
  uint32_t listed;    // tokens listed; more than kList: not all of them
  uint32_t unused;
  uint64_t mass;      // of all tokens (MASS)
  uint32_t bins[kBins];
  // not cleared
  uint64_t pieces[kMostPieces];  // ties << 54 | mass
  uint64_t list[kList];          // key << 32 | token
};
constexpr int kRowsAtATime = 1024;  // rows that the workspace holds

struct SampleArgs {
  const void *logits;
  int64_t stride;
  int rows, vocab;
  const float *u, *temperature, *top_p, *min_p;
  const int32_t *top_k;
  int32_t *tokens;
  float *logprob;
  int32_t *err;
  RowState *state;
  int slices, per_slice;  // per_slice: pieces
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
__device__ __forceinline__ void fill_table(double *table) {
  if (threadIdx.x < 128) table[threadIdx.x] = exp2(threadIdx.x / 128.0);
}

// ---- sums ------------------------------------------------------------------
__device__ __forceinline__ uint64_t wave_sum64(uint64_t v) {
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) {
    const uint32_t lo = __shfl_xor((uint32_t)v, m, kWave), hi = __shfl_xor((uint32_t)(v >> 32), m, kWave);
    v += (uint64_t)hi << 32 | lo;
  }
  return v;
}
__device__ __forceinline__ uint64_t wave_scan(uint64_t v) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t lo = __shfl_up((uint32_t)v, d, kWave), hi = __shfl_up((uint32_t)(v >> 32), d, kWave);
    if (lane >= d) v += (uint64_t)hi << 32 | lo;
  }
  return v;
}
__device__ __forceinline__ float wave_scan(float v) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const float u = __shfl_up(v, d, kWave);
    if (lane >= d) v += u;
  }
  return v;
}
// Inclusive over the workgroup; red: one value a wave.  The last barrier lets red be used again.
template <typename V>
__device__ __forceinline__ V block_scan(V v, V *red, V *total) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  v = wave_scan(v);
  if (lane == 63) red[w] = v;
  __syncthreads();
  V before = 0, all = 0;
  for (int i = 0; i < kSampWaves; ++i) {
    if (i < w) before += red[i];
    all += red[i];
  }
  __syncthreads();
  *total = all;
  return v + before;
}

// (An atomic minimum of every lane's own value at one place would be taken lane
// by lane: 64 rounds.  These leave one a wave.)
__device__ __forceinline__ uint32_t wave_min_u32(uint32_t v) {
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) v = min(v, (uint32_t)__shfl_xor((int)v, m, kWave));
  return v;
}
// The least value over the workgroup of the threads that have one, kNone of
// none; values ascend with the thread.  red: one value a wave.
constexpr int kNone = 0x7fffffff;
__device__ __forceinline__ int block_first(bool has, int value, int *red) {
  const int w = threadIdx.x >> 6;
  const uint64_t who = __ballot(has);
  const int first = __shfl(value, who ? __builtin_ctzll(who) : 0, kWave);
  if ((threadIdx.x & 63) == 0) red[w] = who ? first : kNone;
  __syncthreads();
  int least = kNone;
  for (int i = kSampWaves - 1; i >= 0; --i)
    if (red[i] != kNone) least = red[i];
  __syncthreads();
  return least;
}

// ---- a row -----------------------------------------------------------------

// Tokens with keys above `tie`, and `ties` of those equal to it.
struct Kept {
  uint32_t tie;
  uint32_t ties;
};

enum Mode {
  kPlain,  // the pieces' masses, of the tokens that min_p keeps (greedy: of the largest alone)
  kListK,  // list the bins that hold the first k
  kListM,  // list the tokens that min_p keeps, or that weigh anything
  kMass,   // top-p over everything: list the bins in which it ends, weigh what is above
};

struct Settings {
  bool fine;
  Mode mode;
  int k;        // 0: all
  float p, u;
  double c;     // log2 e / temperature
  double lm;    // least exponent that min_p keeps
  bool greedy;
};

__device__ __forceinline__ Settings settings_of(const SampleArgs &a, int64_t r) {
  const float t = a.temperature ? a.temperature[r] : 1.f, p = a.top_p ? a.top_p[r] : 1.f, m = a.min_p ? a.min_p[r] : 0.f;
  const int k = a.top_k ? a.top_k[r] : 0;
  Settings s;
  s.u = a.u[r];
  s.fine = t >= 0.f && t < INFINITY && p >= 0.f && m >= 0.f && m <= 1.f && s.u >= 0.f && s.u < 1.f && k >= 0;
  s.greedy = t == 0.f || k == 1;
  s.k = k < a.vocab ? k : 0;
  s.p = p;
  s.c = t > 0.f ? kLog2eD / (double)t : kLog2eD;
  s.lm = m > 0.f ? log2((double)m) : -INFINITY;
  s.mode = s.greedy ? kPlain : s.k > 0 ? kListK : p >= 1.f ? kPlain : m > 0.f || t < kSharpest ? kListM : kMass;
  return s;
}

// A row's logits.
template <typename T>
struct Row {
  const T *x;
  int vocab;
  float M;
  double c;
  float origin;  // of the bins

  __device__ __forceinline__ Row(const SampleArgs &a, int64_t r) : x((const T *)a.logits + r * a.stride), vocab(a.vocab) {}

  // The eight logits of this lane in piece p, -infinity behind the last, as they
  // lie in memory, and as floats.
  struct Eight {
    T t[8];
    __device__ __forceinline__ float operator[](int e) const { return Elem<T>::load(t + e); }
  };
  __device__ __forceinline__ Eight raw(int p) const {
    const int at = p * kPiece + 8 * (threadIdx.x & 63);
    Eight f;
    if (at + 8 <= vocab) {
      __builtin_memcpy(f.t, x + at, sizeof f.t);  // (any element-aligned address)
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) f.t[e] = at + e < vocab ? x[at + e] : Elem<T>::to_store(-INFINITY);
    }
    return f;
  }
  __device__ __forceinline__ int pieces() const { return (vocab + kPiece - 1) / kPiece; }
  // g(eight logits, piece) of this wave's pieces among [p0, p1).
  template <class G>
  __device__ __forceinline__ void each_piece(int p0, int p1, G g) const {
    for (int p = p0 + (threadIdx.x >> 6); p < p1; p += kInFlight * kSampWaves) {
      Eight f[kInFlight];
#pragma unroll
      for (int i = 0; i < kInFlight; ++i) f[i] = raw(min(p + i * kSampWaves, p1 - 1));
#pragma unroll 1
      for (int i = 0; i < kInFlight; ++i) {
        if (p + i * kSampWaves < p1) g(f[0], p + i * kSampWaves);
#pragma unroll
        for (int j = 1; j < kInFlight; ++j) f[j - 1] = f[j];
      }
    }
  }
  __device__ __forceinline__ double exponent(float v) const { return ((double)v - (double)M) * c; }

  // The bins descend as the logits ascend.
  __device__ __forceinline__ void set_origin() {
    float top = -INFINITY;
    const Eight f = raw(0);
#pragma unroll
    for (int e = 0; e < 8; ++e) top = fmaxf(top, f[e]);
    top = wave_max(top);
    origin = fabsf(top) < INFINITY ? top : 0.f;
  }
  __device__ __forceinline__ float depth(float v) const {
    return fmaxf((origin - v) * kBinsPerUnit + (float)kBinsAbove, 0.f);
  }
  __device__ __forceinline__ int bin(float v) const { return (int)fminf(depth(v), (float)(kBins - 1)); }
};

// ---- scan ------------------------------------------------------------------

// A bin's masses are parts of its largest, 2^(-its depth's exponent), in whole
// numbers of which all the tokens together stay below 2^32.
__device__ __forceinline__ float mass_one(int vocab) { return (float)(1 << (31 - (32 - __clz((vocab - 1) | 1)))); }
__device__ __forceinline__ float log2_per_bin(const Settings &s) { return (float)(s.c * (1.0 / (16.0 * kLog2eD))); }

template <typename T>
__global__ __launch_bounds__(kSampThreads) void sample_scan_kernel(SampleArgs a) {
  __shared__ uint32_t bins[kBins];
  const int t = threadIdx.x, lane = t & 63;
  const int64_t r = blockIdx.x / a.slices;
  const int p0 = (int)(blockIdx.x % a.slices) * a.per_slice;
  Row<T> row(a, r);
  const int p1 = min(p0 + a.per_slice, row.pieces());
  RowState &st = a.state[r];
  const Settings s = settings_of(a, r);
  if (!s.fine) return;
  const bool counts = s.mode == kListK, masses = s.mode == kMass;
  float M = -INFINITY;
  bool nan = false;
  if (counts || masses) {
    for (int i = t; i < kBins; i += kSampThreads) bins[i] = 0;
    row.set_origin();
    const float one = mass_one(a.vocab), slope = log2_per_bin(s);
    __syncthreads();
    row.each_piece(p0, p1, [&](const typename Row<T>::Eight &f, int) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float v = f[e];
        nan |= v != v;
        M = fmaxf(M, v);
        const float d = row.depth(v), b = floorf(fminf(d, (float)(kBins - 1)));
        const uint32_t part = masses ? (uint32_t)fmaf(__builtin_amdgcn_exp2f((b - d) * slope), one, 0.5f) : 1u;
        if (v > -INFINITY) atomicAdd(&bins[(int)b], part);
      }
    });
    __syncthreads();
    for (int i = t; i < kBins; i += kSampThreads)
      if (bins[i]) atomicAdd(&st.bins[i], bins[i]);
  } else {
    row.each_piece(p0, p1, [&](const typename Row<T>::Eight &f, int) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        nan |= f[e] != f[e];
        M = fmaxf(M, f[e]);
      }
    });
  }
  M = wave_max(M);
  const bool any = __ballot(nan) != 0;
  if (lane == 0) {
    if (M > -INFINITY) atomicMax(&st.top, order_key(M));
    if (any) atomicOr(&st.bad, 1u);
  }
}

// ---- weigh -----------------------------------------------------------------

// A range of bins: [first, last] are listed, what is above counts as it is.
struct Range {
  int first, last;
};

// The bins in which the first k tokens, or the masses' first part p, end (all,
// if there are no more than k; none: masses that came to nothing).  All threads.
__device__ __forceinline__ Range end_bins(const RowState &st, const Settings &s, float top_depth, int vocab, uint64_t *red) {
  constexpr int N = kBins / kSampThreads;
  const int t = threadIdx.x;
  u32x4_t raw[N / 4];
#pragma unroll
  for (int i = 0; i < N / 4; ++i) raw[i] = *(const u32x4_t *)(st.bins + N * t + 4 * i);
  if (s.mode == kListK) {
    uint64_t n = 0, total;
#pragma unroll
    for (int i = 0; i < N; ++i) n += raw[i / 4][i % 4];
    uint64_t at = block_scan(n, red, &total) - n;
    const bool here = at < (uint64_t)s.k && at + n >= (uint64_t)s.k;
    int b = 0;
#pragma unroll
    for (int i = N - 1; i >= 0; --i) {  // the first bin at which k are reached
      if (at + n >= (uint64_t)s.k) b = i;
      n -= raw[i / 4][i % 4];
    }
    const int last = block_first(here, N * t + b, (int *)red);
    return Range{0, min(last, kBins - 1)};
  }
  // masses relative to the bin of M, in fp32: the slack takes the roundings of
  // these sums and, as a rule, those of the histogram; where they come to more,
  // the masses of full precision tell
  const float one = mass_one(vocab), per_bin = log2_per_bin(s), from = floorf(fminf(top_depth, (float)(kBins - 1)));
  float m[N], sum = 0.f, total;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const uint32_t n = raw[i / 4][i % 4];  // (none above M's bin)
    m[i] = n ? (float)n * (1.f / one) * __builtin_amdgcn_exp2f((from - (float)(N * t + i)) * per_bin) : 0.f;
    sum += m[i];
  }
  float at = block_scan(sum, (float *)red, &total);
  const float slack = (0.5f / one + 2e-6f) * total, lo = s.p * total - slack, hi = s.p * total + slack;
  int b1 = kNone, b2 = kNone;
#pragma unroll
  for (int i = N - 1; i >= 0; --i) {
    if (at >= lo) b1 = N * t + i;
    if (at >= hi) b2 = N * t + i;
    at -= m[i];
  }
  b1 = block_first(b1 != kNone, b1, (int *)red);
  b2 = block_first(b2 != kNone, b2, (int *)red);
  return Range{b1, min(b2, kBins - 1)};
}

// tokens that a workgroup of `weigh` gathers before it takes their places in the row's list
constexpr int kSliceList = 1024;

template <typename T>
__global__ __launch_bounds__(kSampThreads) void sample_weigh_kernel(SampleArgs a) {
  __shared__ double table[128];
  __shared__ uint64_t list[kSliceList], red[kSampWaves];
  __shared__ int listed, place;
  const int t = threadIdx.x, lane = t & 63;
  const int64_t r = blockIdx.x / a.slices;
  const int p0 = (int)(blockIdx.x % a.slices) * a.per_slice;
  Row<T> row(a, r);
  const int p1 = min(p0 + a.per_slice, row.pieces());
  RowState &st = a.state[r];
  const Settings s = settings_of(a, r);
  const uint32_t top = st.top;
  row.M = value_of_key(top);
  if (!s.fine || st.bad || top == 0 || !(row.M < INFINITY)) return;
  row.c = s.c;
  fill_table(table);
  if (t == 0) listed = 0;
  Range range{0, -1};
  if (s.mode == kListK || s.mode == kMass) {
    row.set_origin();
    range = end_bins(st, s, row.depth(row.M), a.vocab, red);
    if (range.first == kNone) {  // (masses that came to nothing)
      if (t == 0 && p0 == 0) atomicAdd(&st.listed, kList + 1);
      return;
    }
  }
  __syncthreads();
  const auto add = [&](float v, int token) {
    const int at = atomicAdd(&listed, 1);
    if (at < kSliceList) list[at] = (uint64_t)order_key(v) << 32 | (uint32_t)token;
  };
  const double lm = s.mode == kListM ? fmax(s.lm, kLeast) : s.lm;
  if (s.mode == kListK) {
    row.each_piece(p0, p1, [&](const typename Row<T>::Eight &f, int p) {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (f[e] > -INFINITY && row.bin(f[e]) <= range.last) add(f[e], p * kPiece + 8 * lane + e);
    });
  } else if (s.mode == kListM) {
    row.each_piece(p0, p1, [&](const typename Row<T>::Eight &f, int p) {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (f[e] > -INFINITY && row.exponent(f[e]) >= lm) add(f[e], p * kPiece + 8 * lane + e);
    });
  } else if (s.mode == kMass) {
    uint64_t S = 0;
    row.each_piece(p0, p1, [&](const typename Row<T>::Eight &f, int p) {
      uint64_t above = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint64_t m = f[e] > -INFINITY ? unit_weight(row.exponent(f[e]), table) : 0;
        const int b = row.bin(f[e]);
        S += m;
        above += b < range.first ? m : 0;
        if (b >= range.first && b <= range.last && f[e] > -INFINITY) add(f[e], p * kPiece + 8 * lane + e);
      }
      above = wave_sum64(above);
      if (lane == 0) st.pieces[p] = above;
    });
    S = wave_sum64(S);
    if (lane == 0) atomicAdd((unsigned long long *)&st.mass, S);
  } else if (s.greedy) {
    row.each_piece(p0, p1, [&](const typename Row<T>::Eight &f, int p) {
      int n = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) n += __popcll(__ballot(order_key(f[e]) == top));
      if (lane == 0) st.pieces[p] = (uint64_t)n << 54;
    });
  } else {
    row.each_piece(p0, p1, [&](const typename Row<T>::Eight &f, int p) {
      uint64_t sum = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const double ex = row.exponent(f[e]);
        if (f[e] > -INFINITY && ex >= lm) sum += unit_weight(ex, table);
      }
      sum = wave_sum64(sum);
      if (lane == 0) st.pieces[p] = sum;
    });
  }
  if (s.mode == kPlain) return;
  __syncthreads();
  if (t == 0) place = (int)atomicAdd(&st.listed, listed <= kSliceList ? (uint32_t)listed : kList + 1u);
  __syncthreads();
  const int at = place;
  for (int i = t; i < min(listed, kSliceList) && at + i < kList; i += kSampThreads) st.list[at + i] = list[i];
}

// ---- choose ----------------------------------------------------------------

struct ChooseShared {
  uint64_t mass[kCutBins];       // of a cut's bins, or of the pieces
  uint32_t count[kCutBins];      // of a cut's bins, or of the pieces' ties
  uint64_t list[kList];
  double table[128];
  uint64_t red[kSampWaves];
  uint64_t before;               // mass (or count) above the bin
  int bin, left;
  uint32_t klo, khi;
};
static_assert(kMostPieces <= kCutBins, "the pieces in the bins' place");
constexpr int kPer = kCutBins / kSampThreads;  // bins, or pieces, of a thread

// f(value, key, token) of the row's list, as it is in LDS, or of all its
// tokens above -infinity.
template <typename T>
struct Tokens {
  const Row<T> &row;
  const ChooseShared &sh;
  int listed;  // below 0: the whole row
  template <class F>
  __device__ __forceinline__ void each(F f) const {
    if (listed >= 0) {
      for (int i = threadIdx.x; i < listed; i += kSampThreads) {
        const uint32_t key = (uint32_t)(sh.list[i] >> 32);
        f(value_of_key(key), key, (int)(uint32_t)sh.list[i]);
      }
    } else {
      for (int p = threadIdx.x >> 6; p < row.pieces(); p += kSampWaves) {
        const typename Row<T>::Eight v = row.raw(p);
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (v[e] > -INFINITY) f(v[e], order_key(v[e]), p * kPiece + 8 * (int)(threadIdx.x & 63) + e);
      }
    }
  }
};

// The smallest start of the kept ones of these tokens, in descending order, at
// which `before` plus their amount (MASS: of their masses; else their number)
// reaches the target.  All threads; returns the same in each.  Rounds of 1024
// bins over keys from the largest down, until a single value is left.
template <bool MASS, typename T>
__device__ __noinline__ Kept cut(const Row<T> &row, const Tokens<T> &tokens, Kept kept, double lm, uint64_t before, double target,
                                 ChooseShared &sh) {
  const int t = threadIdx.x;
  const auto amount = [&](float v) { return MASS ? unit_weight(row.exponent(v), sh.table) : (uint64_t)1; };
  const float tie_value = value_of_key(kept.tie);
  const bool tie_in = kept.ties > 0 && row.exponent(tie_value) >= lm;
  uint32_t klo = 0, khi = 0xffffffffu;
  for (;;) {
    // ---- least and largest key ----
    if (t == 0) {
      sh.klo = 0xffffffffu;
      sh.khi = 0;
    }
    for (int i = t; i < kCutBins; i += kSampThreads) sh.mass[i] = sh.count[i] = 0;
    __syncthreads();
    uint32_t lo = 0xffffffffu, hi = 0;
    tokens.each([&](float v, uint32_t key, int) {
      if (key <= kept.tie || key < klo || key > khi || row.exponent(v) < lm) return;
      lo = min(lo, key);
      hi = max(hi, key);
    });
    if (t == 0 && tie_in && kept.tie >= klo && kept.tie <= khi) {
      lo = min(lo, kept.tie);
      hi = max(hi, kept.tie);
    }
    lo = wave_min_u32(lo);
    hi = ~wave_min_u32(~hi);
    if ((t & 63) == 0 && hi) {
      atomicMin(&sh.klo, lo);
      atomicMax(&sh.khi, hi);
    }
    __syncthreads();
    klo = sh.klo;
    khi = sh.khi;
    if (khi == 0) return kept;  // no tokens
    int shift = 0;
    while ((khi - klo) >> shift >= (uint32_t)kCutBins) ++shift;
    // ---- amounts by bins ----
    tokens.each([&](float v, uint32_t key, int) {
      if (key <= kept.tie || key < klo || key > khi || row.exponent(v) < lm) return;
      const int b = (khi - key) >> shift;
      atomicAdd(&sh.count[b], 1u);
      if constexpr (MASS) atomicAdd((unsigned long long *)&sh.mass[b], amount(v));
    });
    if (t == 0 && tie_in && kept.tie >= klo && kept.tie <= khi) {
      const int b = (khi - kept.tie) >> shift;
      atomicAdd(&sh.count[b], kept.ties);
      if constexpr (MASS) atomicAdd((unsigned long long *)&sh.mass[b], kept.ties * amount(tie_value));
    }
    __syncthreads();
    uint64_t mine[kPer], sum = 0, total;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      mine[i] = MASS ? sh.mass[kPer * t + i] : sh.count[kPer * t + i];
      sum += mine[i];
    }
    uint64_t at = block_scan(sum, sh.red, &total) + before - sum;
    total += before;
    // the first bin with a token at which the target is reached, or the last with one
    int mine_first = kNone;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      at += mine[i];
      if (mine_first == kNone && sh.count[kPer * t + i] && ((double)at >= target || at == total)) mine_first = kPer * t + i;
    }
    const int b = block_first(mine_first != kNone, mine_first, (int *)sh.red);
    if (b / kPer == t) {
      uint64_t end = at;
#pragma unroll
      for (int i = kPer - 1; i >= 0; --i)
        if (i >= b % kPer) end -= mine[i];
      sh.before = end;
    }
    __syncthreads();
    before = sh.before;
    const uint32_t n = sh.count[b];
    const uint64_t amounts = MASS ? sh.mass[b] : n;
    const uint32_t lower = khi - min(khi - klo, ((uint32_t)(b + 1) << shift) - 1), upper = khi - ((uint32_t)b << shift);
    if (lower == upper) {  // one value: its first few
      const double each = (double)(amounts / n), need = (target - (double)before) / each;
      const uint32_t few = each > 0 && need < (double)n ? (need > 1.0 ? (uint32_t)ceil(need) : 1u) : n;
      return Kept{lower, few};
    }
    klo = lower;
    khi = upper;
    __syncthreads();
  }
}

template <typename T>
__global__ __launch_bounds__(kSampThreads) void sample_choose_kernel(SampleArgs a) {
  __shared__ ChooseShared sh;
  const int t = threadIdx.x, lane = t & 63, w = t >> 6;
  const int64_t r = blockIdx.x;
  Row<T> row(a, r);
  RowState &st = a.state[r];
  Settings s = settings_of(a, r);
  const uint32_t top = st.top;
  const int listed = (int)min(st.listed, kList + 1u);
  const uint64_t mass = st.mass;
  row.M = value_of_key(top);
  row.c = s.c;
  const bool fine = s.fine && !st.bad && top != 0 && row.M < INFINITY;
  fill_table(sh.table);
  if (fine && listed <= kList)
    for (int i = t; i < listed; i += kSampThreads) sh.list[i] = st.list[i];
  const int pieces = row.pieces();
  uint64_t mine[kPer];  // the pieces of this thread: ties << 54 | mass
#pragma unroll
  for (int i = 0; i < kPer; ++i)
    mine[i] = fine && (s.mode == kPlain || s.mode == kMass) && kPer * t + i < pieces ? st.pieces[kPer * t + i] : 0;
  __syncthreads();
  // ---- the row's state is zero again ----
  if (t < 4) (&st.top)[t] = 0;
  if (t == 4) st.mass = 0;
  for (int i = t; i < kBins / 4; i += kSampThreads) *(u32x4_t *)(st.bins + 4 * i) = u32x4_t{0u, 0u, 0u, 0u};
  if (!fine) {
    if (t == 0) {
      a.tokens[r] = -1;
      if (a.logprob) a.logprob[r] = NAN;
      if (a.err) set_err(a.err, SM_ERR_EINVAL);
    }
    return;
  }
  // ---- the filters ----
  Kept kept{0, 0};  // (no finite logit has key 0)
  if (s.greedy) {
    kept = Kept{top, 1};
  } else if (s.mode != kPlain) {
    Tokens<T> tokens{row, sh, listed <= kList ? listed : -1};
    if (s.k > 0) kept = cut<false>(row, tokens, kept, -INFINITY, 0, (double)s.k, sh);
    if (kept.ties > 0 && row.exponent(value_of_key(kept.tie)) < s.lm) kept.ties = 0;
    if (s.p < 1.f) {
      uint64_t before = 0, all = 0;
      if (s.mode == kMass && tokens.listed >= 0) {
        uint64_t sum = 0, rest = 0;
#pragma unroll
        for (int i = 0; i < kPer; ++i) sum += mine[i];
        block_scan(sum, sh.red, &before);
        tokens.each([&](float v, uint32_t, int) { rest += unit_weight(row.exponent(v), sh.table); });
        block_scan(rest, sh.red, &rest);
        all = mass;
        const double target = (double)s.p * (double)all;
        if (((double)before >= target && before > 0) || (double)(before + rest) < target) tokens.listed = -1;  // it ends elsewhere
      }
      if (!(s.mode == kMass && tokens.listed >= 0)) {
        uint64_t sum = 0;
        before = 0;
        tokens.each([&](float v, uint32_t key, int) {
          if (key > kept.tie && row.exponent(v) >= s.lm) sum += unit_weight(row.exponent(v), sh.table);
        });
        if (t == 0 && kept.ties > 0) sum += kept.ties * unit_weight(row.exponent(value_of_key(kept.tie)), sh.table);
        block_scan(sum, sh.red, &all);
      }
      kept = cut<true>(row, tokens, kept, s.lm, before, (double)s.p * (double)all, sh);
    }
    // ---- the pieces' masses and ties, above the list and in it ----
    const bool add = s.mode == kMass && tokens.listed >= 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      sh.mass[kPer * t + i] = add ? mine[i] : 0;
      sh.count[kPer * t + i] = 0;
    }
    __syncthreads();
    tokens.each([&](float v, uint32_t key, int token) {
      const double ex = row.exponent(v);
      if (key > kept.tie && ex >= s.lm)
        atomicAdd((unsigned long long *)&sh.mass[token / kPiece], unit_weight(ex, sh.table));
      else if (key == kept.tie && kept.ties > 0) atomicAdd(&sh.count[token / kPiece], 1u);
    });
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kPer; ++i) mine[i] = sh.mass[kPer * t + i] | (uint64_t)sh.count[kPer * t + i] << 54;
  }
  // ---- the piece: the first at which the cumulative mass passes u times all of it ----
  const float tie_value = value_of_key(kept.tie);
  const uint64_t each = kept.ties > 0 ? unit_weight(row.exponent(tie_value), sh.table) : 0;
  uint64_t ties = 0, sum = 0, unused, S;
#pragma unroll
  for (int i = 0; i < kPer; ++i) ties += mine[i] >> 54;
  uint64_t ties_before = block_scan(ties, sh.red, &unused) - ties, first_ties = ties_before;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const uint64_t n = mine[i] >> 54;
    mine[i] &= (1ull << 54) - 1;
    mine[i] += (ties_before >= kept.ties ? 0 : min(n, kept.ties - ties_before)) * each;
    ties_before += n;
    sum += mine[i];
  }
  const uint64_t start = block_scan(sum, sh.red, &S) - sum;
  const uint64_t target = (uint64_t)((double)s.u * (double)S);
  if (start <= target && target < start + sum) {
    uint64_t at = start;
    bool found = false;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      if (!found && at + mine[i] > target) {
        found = true;
        sh.bin = kPer * t + i;
        sh.before = at;
      }
      at += mine[i];
    }
    // ties that are left for it: those of its thread's pieces before it are counted below
    sh.left = (int)min<uint64_t>(kept.ties, first_ties);
  }
  __syncthreads();
  if (w != 0) return;
  // ---- its token, by one wave ----
  const int piece = sh.bin;
  const typename Row<T>::Eight f = row.raw(piece);
  const uint64_t goal = target - sh.before;
  uint64_t m[8];
  uint32_t tied = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const uint32_t key = order_key(f[e]);
    const double ex = row.exponent(f[e]);
    m[e] = f[e] > -INFINITY && key > kept.tie && ex >= s.lm && !s.greedy ? unit_weight(ex, sh.table) : 0;
    tied |= (uint32_t)(kept.ties > 0 && key == kept.tie) << e;
  }
  // the ties of the pieces before this one: `left` up to the first piece of its thread, the others looked at again
  int seen = sh.left;
  if (kept.ties > 0)
    for (int q = piece / kPer * kPer; q < piece; ++q) {
      const typename Row<T>::Eight g = row.raw(q);
#pragma unroll
      for (int e = 0; e < 8; ++e) seen += __popcll(__ballot(order_key(g[e]) == kept.tie));
    }
  int rank = seen + (int)wave_scan((uint64_t)__popc(tied)) - __popc(tied);
  sum = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    if (tied >> e & 1) {
      if (rank < (int)kept.ties) m[e] = each;
      ++rank;
    }
    sum += m[e];
  }
  const uint64_t before = wave_scan(sum) - sum;
  if (!(before <= goal && goal < before + sum)) return;
  int at = 7;
#pragma unroll
  for (int e = 7; e >= 0; --e)
    if (before + sum > goal) {  // sum: the masses up to e
      at = e;
      sum -= m[e];
    }
  const int token = piece * kPiece + 8 * lane + at;
  a.tokens[r] = token;
  if (a.logprob) {
    const double ex = row.exponent(Elem<T>::load(row.x + token));
    a.logprob[r] = (float)((ex - (log2((double)S) - kUnit)) / kLog2eD);
  }
}

}  // namespace sm

using namespace sm;

SM_API size_t sm_sample_workspace_bytes(int rows, int vocab) {
  return rows > 0 && vocab > 0 ? sizeof(RowState) * std::min(rows, kRowsAtATime) : 0;
}

template <typename T>
static sm_status launch_sample(const SampleArgs &a, hipStream_t stream) {
  const dim3 grid((unsigned)(a.rows * a.slices)), threads(kSampThreads);
  hipLaunchKernelGGL(sample_scan_kernel<T>, grid, threads, 0, stream, a);
  hipLaunchKernelGGL(sample_weigh_kernel<T>, grid, threads, 0, stream, a);
  hipLaunchKernelGGL(sample_choose_kernel<T>, dim3(a.rows), threads, 0, stream, a);
  return hipGetLastError() == hipSuccess ? SM_OK : SM_EHIP;
}

SM_API sm_status sm_sample_tokens(const void *logits, int64_t stride, int rows, int vocab, sm_dtype dt, const float *u,
                                  const float *temperature, const int32_t *top_k, const float *top_p, const float *min_p,
                                  int32_t *tokens, float *logprob, void *ws, size_t ws_bytes, int32_t *err, hipStream_t stream) {
  if ((dt != SM_F32 && dt != SM_BF16) || rows < 0 || vocab < 1 || vocab > kMostVocab || stride < vocab) return SM_EINVAL;
  if (rows == 0) return SM_OK;
  if (!logits || !u || !tokens || !ws || (uintptr_t)ws % 16 || ws_bytes < sm_sample_workspace_bytes(rows, vocab)) return SM_EINVAL;
  const int pieces = (vocab + kPiece - 1) / kPiece, es = dt == SM_BF16 ? 2 : 4;
  // Slices of 16 pieces, all loaded at once, until there are plenty of
  // workgroups; then of 64.
  const int per = (int64_t)std::min(rows, kRowsAtATime) * ((pieces + 15) / 16) <= 4096 ? 16 : 64;
  for (int first = 0; first < rows; first += kRowsAtATime) {
    const SampleArgs a{(const char *)logits + first * stride * es, stride, std::min(rows - first, kRowsAtATime), vocab, u + first,
                       temperature ? temperature + first : nullptr, top_p ? top_p + first : nullptr,
                       min_p ? min_p + first : nullptr, top_k ? top_k + first : nullptr, tokens + first,
                       logprob ? logprob + first : nullptr, err, (RowState *)ws, (pieces + per - 1) / per, per};
    const sm_status st = dt == SM_BF16 ? launch_sample<uint16_t>(a, stream) : launch_sample<float>(a, stream);
    if (st != SM_OK) return st;
  }
  return SM_OK;
}
