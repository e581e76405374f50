// Log probabilities of given tokens, entropy and top alternatives of rows of
// logits (gfx950), in one pass over the logits.
//
// With a reference r and d = x - r:
//   S = sum exp(scale d), E = sum d exp(scale d),
//   log p_v = scale d_v - log S,   entropy = log S - scale E / S.
// r is the maximum of the workgroup's first chunk, and moves only when a later
// logit is 2^kLift times as probable, so that the loop rescales nothing: 5
// instructions and one exponential a logit.  A logit of -infinity would make
// E NaN (0 x infinity).  A chunk of either kind is added again, with r moved
// and d clamped.
//
// Alternatives are ordered by one 64-bit key per logit: the value's bits made
// to ascend with it, then the index counted down, so that no two are equal.
// Lanes' maxima give a bound below the k-th largest (a count over them, bit by
// bit), after the first chunk and whenever the chunks seen have doubled.  A
// wave notes the 16-byte vectors that reach the bound, in LDS, and looks at
// their logits 64 vectors at a time: keys above the bound go to LDS, where they
// are reduced to the k largest, with a bound of the wave's own, when there is
// no room.
//
// A row is one workgroup's (of one wave where it is short), or for few rows
// its slices are several ones', joined by the last to arrive at the row's
// counter.
//
// Many rows are bound by the read and, in bf16, by the vector instructions,
// which a compute unit issues all the time: 4096 rows of 128,256 bf16 logits
// (1.05 GB) take 167 us without alternatives, 6.3 TB/s, and 169 with one or with
// 20 (one call after another, as the clock falls, 177, 188 and 201); fp32 rows
// of the same size 169 us with 20.  Few rows are bound by latency: 16 rows 5.3 us
// without alternatives and 9.4 with 8 (bound, look, sort, then the same of the
// slices' keys), 300 rows 17.9 and 22.9 of the 11.4 that their read takes.
#include <algorithm>
#include <cmath>

#include "vec16.hpp"

namespace sm {

constexpr int kLpWaves = 4;                                   // waves of a workgroup, but for short rows
constexpr int kLpUnroll = 4;                                  // 16-byte vectors that a thread holds at a time
constexpr int kLpChunk = 64 * kLpWaves * kLpUnroll;           // vectors that they hold
constexpr int kKeep = 256;                                    // keys that a wave keeps: SM_MAX_TOP and one of each lane at least
constexpr int kNoted = 64 + 64 * kLpUnroll;                   // vectors that it has noted: a chunk's, and those before
constexpr int kMostSlices = 64;                               // (one wave reads their sums)
constexpr int kMostKeys = kLpWaves * kKeep;                   // of all slices of a row
constexpr int kCounterStep = 32;                              // counters stand 128 bytes apart
// Up to this many lanes' largest of a wave bound its first chunk, beyond it its
// vectors' largest: the lanes' few largest are in different vectors, but all of
// them are a weak bound.  64 rows of 2000 bf16 logits, us: 64 alternatives
// 12.5 by lanes and 8.4 by vectors, 20 alternatives 6.1 and 6.9.
constexpr int kLanesWanted = 32;
constexpr float kLn2 = 0.69314718055994531f;
constexpr float kLowest = -3.4028234663852886e38f;
constexpr float kLift = 4.f;

struct LogprobArgs {
  const void *logits;
  int64_t stride;
  int rows, vocab, k;
  float scale, c;  // c: scale x log2 e, in fp32: an exponent is off by a unit of itself, as its product with d is
  const int32_t *tokens;
  float *logprob, *entropy;
  int32_t *top_ids;
  float *top_logprobs;
  int32_t *err;
  int slices, per_slice;  // per_slice: vectors
  int *counters;
  float4 *part_sums;    // [row][slice] {r, S, E}
  uint64_t *part_keys;  // [row][slice][k], 0 behind the last
};

// Ascends with x; -0 counts as 0.  NaN has no place: one without the sign bit
// would come above +infinity, so none is asked for.
__device__ __forceinline__ uint32_t order_of(float x) {
  const uint32_t b = __float_as_uint(x + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t o) { return __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o); }
__device__ __forceinline__ uint64_t key_of(float x, int v) { return (uint64_t)order_of(x) << 32 | (uint32_t)~v; }

__device__ __forceinline__ int lanes_below(uint64_t mask) {
  return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
}

// Sums over logits relative to r.
struct Sums {
  float r, S, E;
};

// s relative to another reference
__device__ __forceinline__ void move_to(Sums &s, float r, float c) {
  const float d = s.r - r, f = __builtin_amdgcn_exp2f(d * c);
  s.E = f == 0.f ? 0.f : f * fmaf(s.S, d, s.E);
  s.S *= f;
  s.r = r;
}

// One wave's sums of its lanes'.
__device__ __forceinline__ Sums wave_sums(Sums s, float c) {
  move_to(s, wave_max(s.r), c);
  s.S = wave_sum(s.S);
  s.E = wave_sum(s.E);
  return s;
}

__device__ __forceinline__ void wave_order() {  // LDS accesses of the wave's lanes, in program order
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
}

// rank[i]: how many of a wave's n keys (n <= 64 NK) are above key[i], this
// lane's i-th.  kRankStep keys' reads are in flight at a time; 0 takes the
// place of those behind the last.
constexpr int kRankStep = 16;
template <int NK>
__device__ __forceinline__ void rank_keys(uint64_t *buf, int n, uint64_t (&key)[NK], int (&rank)[NK]) {
  const int lane = threadIdx.x & 63, padded = (n + kRankStep - 1) / kRankStep * kRankStep;
#pragma unroll
  for (int i = 0; i < NK; ++i) {
    const int at = lane + 64 * i;
    rank[i] = 0;
    if (at >= n && at < padded) buf[at] = 0;
  }
  wave_order();
#pragma unroll
  for (int i = 0; i < NK; ++i) key[i] = lane + 64 * i < n ? buf[lane + 64 * i] : 0;
  for (int j = 0; j < n; j += kRankStep) {
    uint64_t other[kRankStep];
#pragma unroll
    for (int i = 0; i < kRankStep; ++i) other[i] = buf[j + i];
#pragma unroll
    for (int i = 0; i < kRankStep; ++i)
#pragma unroll
      for (int l = 0; l < NK; ++l) rank[l] += other[i] > key[l];
  }
  wave_order();
}
template <int NK>
__device__ __forceinline__ void keep_by_rank(uint64_t *buf, int n, int k) {
  uint64_t key[NK];
  int rank[NK];
  rank_keys(buf, n, key, rank);
#pragma unroll
  for (int i = 0; i < NK; ++i)
    if ((int)(threadIdx.x & 63) + 64 * i < n && rank[i] < k) buf[rank[i]] = key[i];
  wave_order();
}

// The k largest of a wave's n keys (n <= kKeep) to the front of buf, in any
// order; returns how many there are.  `bits`: of an index.  Values below
// 2^LOW are all alike.
template <int LOW>
__device__ __forceinline__ int keep_largest(uint64_t *buf, int n, int k, int bits) {
  if (n <= k) return n;
  if (n <= 64) {
    keep_by_rank<1>(buf, n, k);
    return k;
  }
  if (n <= 128) {
    keep_by_rank<2>(buf, n, k);
    return k;
  }
  constexpr int NR = kKeep / 64;
  const int lane = threadIdx.x & 63;
  uint32_t hi[NR], lo[NR];
  wave_order();
#pragma unroll
  for (int i = 0; i < NR; ++i) {
    const uint64_t key = lane + 64 * i < n ? buf[lane + 64 * i] : 0;
    hi[i] = (uint32_t)(key >> 32) >> LOW;
    lo[i] = (uint32_t)key;
  }
  wave_order();
  const auto count = [&](auto f) {
    int cnt = 0;
#pragma unroll
    for (int i = 0; i < NR; ++i) cnt += __popcll(__ballot(f(i)));
    return cnt;
  };
  // The k-th value, bit by bit; or one that k keys reach, which is as good.
  // Then, if more do, the least index (counted down) among the equal ones.
  uint32_t v = 0, from = 0;
  int c = n;
  for (int b = 31 - LOW; b >= 0 && c != k; --b) {
    const uint32_t y = v | 1u << b;
    const int cy = count([&](int i) { return hi[i] >= y; });
    if (cy >= k) {
      v = y;
      c = cy;
    }
  }
  if (c != k) {
    const int above = count([&](int i) { return hi[i] > v; });
    from = ~0u << (bits - 1) << 1;
    for (int b = bits - 1; b >= 0 && c != k; --b) {
      const uint32_t y = from | 1u << b;
      const int cy = above + count([&](int i) { return hi[i] == v && lo[i] >= y; });
      if (cy >= k) {
        from = y;
        c = cy;
      }
    }
  }
  int at = 0;
#pragma unroll
  for (int i = 0; i < NR; ++i) {
    const bool keep = hi[i] > v || (hi[i] == v && lo[i] >= from);
    const uint64_t mask = __ballot(keep);
    // (the values' low bits are those of their sign: all 1 below 0)
    if (keep) buf[at + lanes_below(mask)] = (uint64_t)(hi[i] << LOW | (LOW && !(hi[i] >> (31 - LOW)) ? 0xffffu : 0u)) << 32 | lo[i];
    at += __popcll(mask);
  }
  wave_order();
  return at;
}

__device__ __forceinline__ uint64_t wave_min64(uint64_t v) {
#pragma unroll
  for (int off = 32; off; off >>= 1) {
    const uint64_t u = __shfl_xor(v, off, kWave);
    v = u < v ? u : v;
  }
  return v;
}

// A wave's candidates and the bound that they lie above.
template <typename T>
struct Candidates {
  static constexpr int LOW = sizeof(T) == 2 ? 16 : 0;
  uint64_t *buf;
  u32x4_t *noted;  // vectors and their numbers
  int *numbers;
  int n, vectors, k, bits;  // bits: of an index
  int ordered;     // a bound of an index below this is the lowest index of its value to come
  uint64_t bound;  // keys above it are wanted
  float least;     // vectors whose largest is this or more may hold one

  __device__ __forceinline__ void raise(uint64_t b) {
    if (b <= bound) return;
    bound = b;
    const uint32_t hi = (uint32_t)(b >> 32), lo = (uint32_t)b;
    least = value_of(lo != 0 && (int)~lo < ordered ? hi + 1 : hi);
  }
  __device__ __forceinline__ void put(float x, int v, bool valid) {
    const uint64_t key = key_of(x, v);
    const bool want = valid && x == x && key > bound;
    const uint64_t mask = __ballot(want);
    if (want) buf[n + lanes_below(mask)] = key;
    n += __popcll(mask);
  }
  __device__ __forceinline__ void note(float m, int v, u32x4_t x) {
    const bool want = m >= least;
    const uint64_t mask = __ballot(want);
    if (want) {
      const int at = vectors + lanes_below(mask);
      noted[at] = x;
      numbers[at] = v;
    }
    vectors += __popcll(mask);
  }
  // The noted vectors' logits that reach the bound, one of each vector at a
  // time; vector v begins at logit head + N v.
  __device__ __forceinline__ void look(int head, int end) {
    constexpr int N = Vec16<T>::N;
    const int lane = threadIdx.x & 63;
    wave_order();
#pragma unroll 1
    for (int i = 0; i < vectors; i += 64) {
      const int v = i + lane < vectors ? numbers[i + lane] : end;
      u32x4_t w{0, 0, 0, 0};
      uint32_t left = 0;
      if (v < end) {  // (behind the slice there are none)
        w = noted[i + lane];
        float f[N];
        Vec16<T>::open(w, f);
#pragma unroll
        for (int e = 0; e < N; ++e) left |= f[e] >= least ? 1u << e : 0u;
      }
#pragma unroll 1
      while (__ballot(left != 0)) {
        if (n > kKeep - 64) {
          n = keep_largest<LOW>(buf, n, k, bits);
          if (n == k) raise(wave_min64(lane < n ? buf[lane] : ~0ull));
        }
        const int e = __builtin_ctz(left | 0x80000000u) % N;
        uint32_t x;
        if constexpr (N == 8) {
          x = e < 4 ? (e < 2 ? w[0] : w[1]) : (e < 6 ? w[2] : w[3]);
          x = e & 1 ? x & 0xffff0000u : x << 16;
        } else {
          x = e < 2 ? (e < 1 ? w[0] : w[1]) : (e < 3 ? w[2] : w[3]);
        }
        put(__uint_as_float(x), head + N * v + e, left != 0);
        left &= left - 1;
      }
    }
    vectors = 0;
  }
};

// Results of a row by one wave: its sums, its token (-1: none) with the
// token's logit, and its m best keys in buf.
template <typename T, bool TOP>
__device__ __forceinline__ void put_row(const LogprobArgs &a, int64_t r, Sums s, int tok, float x_tok, uint64_t *buf,
                                        int m) {
  const int lane = threadIdx.x & 63;
  const T *x = (const T *)a.logits + r * a.stride;
  const float log_s = __builtin_amdgcn_logf(s.S) * kLn2;
  auto logprob = [&](float f) {
    if (s.S == 0.f) return -INFINITY;  // nothing but -infinity
    // (logits further apart than the largest number are scaled first)
    const float d = f - s.r, lp = d >= kLowest ? fmaf(d, a.scale, -log_s) : fmaf(f, a.scale, -a.scale * s.r) - log_s;
    return lp > 0.f ? 0.f : lp;
  };
  if (lane == 0) {
    if (a.entropy) {
      const float h = s.S == 0.f ? 0.f : fmaf(-a.scale, s.E / s.S, log_s);
      a.entropy[r] = h < 0.f ? 0.f : h;
    }
    if (a.logprob) {
      a.logprob[r] = tok >= 0 && tok < a.vocab ? logprob(x_tok) : 0.f;
      if ((tok < -1 || tok >= a.vocab) && a.err) set_err(a.err, SM_ERR_EINVAL);
    }
  }
  if constexpr (TOP) {
    uint64_t key[1];
    int rank[1];
    rank_keys(buf, m, key, rank);
    if (lane < m) {
      a.top_ids[r * a.k + rank[0]] = (int)~(uint32_t)key[0];
      if (a.top_logprobs) a.top_logprobs[r * a.k + rank[0]] = logprob(value_of((uint32_t)(key[0] >> 32)));
    }
    for (int64_t v0 = 0; m < a.k && v0 < a.vocab; v0 += 64) {  // fewer numbers than alternatives: NaN follow
      const float f = v0 + lane < a.vocab ? Elem<T>::load(x + v0 + lane) : 0.f;
      const uint64_t mask = __ballot(f != f);
      const int at = m + lanes_below(mask);
      if (f != f && at < a.k) {
        a.top_ids[r * a.k + at] = (int)v0 + lane;
        if (a.top_logprobs) a.top_logprobs[r * a.k + at] = f;
      }
      m += __popcll(mask);
    }
  }
}

template <class V>
__device__ __forceinline__ void put_shared(V *p, V v) {
  __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
template <class V>
__device__ __forceinline__ V get_shared(V *p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// W waves to a workgroup.
template <typename T, bool TOP, int W>
__global__ __launch_bounds__(64 * W) void logprobs_kernel(LogprobArgs a) {
  constexpr int N = Vec16<T>::N, LOW = Candidates<T>::LOW, THREADS = 64 * W, CHUNK = THREADS * kLpUnroll;
  __shared__ uint64_t keys[TOP ? W : 1][TOP ? kKeep : 1];
  __shared__ u32x4_t noted[TOP ? W : 1][TOP ? kNoted : 1];
  __shared__ int numbers[TOP ? W : 1][TOP ? kNoted : 1];
  __shared__ float w_max[W], w_r[W], w_S[W], w_E[W];
  __shared__ uint32_t w_bound[W];
  __shared__ int w_n[W], last;
  const int t = threadIdx.x, lane = t & 63, w = t >> 6;
  const int64_t r = blockIdx.x / a.slices;
  const int slice = blockIdx.x - (int)r * a.slices;
  const T *x = (const T *)a.logits + r * a.stride;
  // aligned vectors, and the few logits before and behind them
  const int head = min((int)((16 - (uintptr_t)x % 16) % 16 / sizeof(T)), a.vocab);
  const int nvec = (a.vocab - head) / N;
  const u32x4_t *xv = (const u32x4_t *)(x + head);
  const int begin = min(slice * a.per_slice, nvec), end = min(begin + a.per_slice, nvec);
  // The chunk at v0.  Two are held, the next one on its way while one is
  // worked on; the loads are unconditional (behind the slice's end its last
  // vector again), so that waiting for one chunk leaves the other in flight.
  u32x4_t even[kLpUnroll], odd[kLpUnroll];
  auto load = [&](u32x4_t (&cur)[kLpUnroll], int v0) {
#pragma unroll
    for (int u = 0; u < kLpUnroll; ++u)
      cur[u] = __builtin_nontemporal_load(xv + min(v0 + u * THREADS + t, end - 1));
  };
  auto fill = [&](u32x4_t (&cur)[kLpUnroll], int v0, uint32_t with) {  // behind the end
    if (v0 + CHUNK <= end) return;
#pragma unroll
    for (int u = 0; u < kLpUnroll; ++u)
      if (v0 + u * THREADS + t >= end) cur[u] = u32x4_t{with, with, with, with};
  };
  auto largest = [&](const float *f) {
    float m = f[0];
#pragma unroll
    for (int e = 1; e < N; ++e) m = fmaxf(m, f[e]);
    return m;
  };
  Sums s{kLowest, 0.f, 0.f};
  Candidates<T> top{keys[TOP ? w : 0], noted[TOP ? w : 0], numbers[TOP ? w : 0], 0, 0, a.k, 32 - __clz(a.vocab), head + nvec * N, 0, -INFINITY};
  float best = -INFINITY;  // this lane's largest
  // A bound below the slice's k-th largest: k / W of the largest of each wave's
  // lanes (few alternatives: k of one wave's) are the bound of its least one or
  // more; or of its vectors (reached(o): how many are o or more).
  const bool one_wave = a.k < W;
  const int want = one_wave ? a.k : (a.k + W - 1) / W;
  auto bound_of = [&](auto reached) {
    uint32_t b = 0;
    for (int bit = 31; bit >= 16; --bit)  // (the low bits are not worth their time)
      if (reached(b | 1u << bit) >= want) b |= 1u << bit;
    return b;
  };
  auto lanes_bound = [&]() {
    const uint32_t o = order_of(best);
    return bound_of([&](uint32_t b) { return __popcll(__ballot(o >= b)); });
  };
  auto use_bounds = [&]() {
    uint32_t b = one_wave ? 0 : ~0u;
#pragma unroll
    for (int i = 0; i < W; ++i) {
      const uint32_t o = __hip_atomic_load(w_bound + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
      b = one_wave ? max(b, o) : min(b, o);
    }
    b = max(b, 0x007fffffu);  // (-infinity's)
    top.raise((uint64_t)b << 32);
  };
  // the token's logit, long before it is used
  const int tok = a.logprob ? a.tokens[r] : -1;
  float x_tok = 0.f;
  if (begin < end) load(even, begin);
  if (t == 0 && tok >= 0 && tok < a.vocab) x_tok = Elem<T>::load(x + tok);
  if (begin < end) {
    fill(even, begin, Vec16<T>::kMinusInf);
    float m[kLpUnroll];
#pragma unroll
    for (int u = 0; u < kLpUnroll; ++u) {
      float f[N];
      Vec16<T>::open(even[u], f);
      m[u] = largest(f);
      best = fmaxf(best, m[u]);
    }
    const float mw = wave_max(best);
    uint32_t b = 0;
    if constexpr (TOP) {
      b = want <= kLanesWanted ? lanes_bound() : bound_of([&](uint32_t b) {
        int n = 0;
#pragma unroll
        for (int u = 0; u < kLpUnroll; ++u)  // (a vector of nothing but NaN has no largest: as -infinity)
          n += __popcll(__ballot(order_of(fmaxf(m[u], -INFINITY)) >= b));
        return n;
      });
    }
    if (lane == 0) {
      w_max[w] = mw;
      w_bound[w] = b;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < W; ++i) s.r = fmaxf(s.r, w_max[i]);
    if constexpr (TOP) use_bounds();
  }
  // adds a vector's logits to a chunk's sums, which join the row's together:
  // a sum of few terms at a time loses less
  auto add = [&](const float *f, Sums &to, bool clamp) {
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const float d = f[e] - to.r, p = __builtin_amdgcn_exp2f(d * a.c);
      to.S += p;
      to.E = fmaf(p, clamp ? fmaxf(d, kLowest) : d, to.E);
    }
  };
  if (slice == 0 && w == 0) {
    const int rest = a.vocab - head - nvec * N;  // (under two vectors with the head's)
    const int v = lane < head ? lane : a.vocab - rest + lane - head;
    float f[N];
#pragma unroll
    for (int e = 0; e < N; ++e) f[e] = -INFINITY;
    if (lane < head + rest) f[0] = Elem<T>::load(x + v);
    const float m = wave_max(f[0]);
    if ((m - s.r) * a.c > kLift) move_to(s, m, a.c);
    add(f, s, true);
    if constexpr (TOP) top.put(f[0], v, lane < head + rest);
  }
  bool clamp = false;  // whether the slice has shown -infinity
  auto chunk = [&](u32x4_t (&cur)[kLpUnroll], int v0, int seen) {
    // nothing behind the end: by a value of probability 0 (-infinity would have the chunk added again)
    fill(cur, v0, s.r > -1e38f ? Vec16<T>::kLowest : Vec16<T>::kMinusInf);
    Sums part{s.r, 0.f, 0.f};
    float m[kLpUnroll], all = -INFINITY;
    auto pass = [&](bool clamped) {
#pragma unroll
      for (int u = 0; u < kLpUnroll; ++u) {
        u32x4_t x = cur[u];
        if (clamped) asm("" : "+v"(x));  // (apart from the other pass, whose values would else be formed before the branch)
        float f[N];
        Vec16<T>::open(x, f);
        m[u] = largest(f);
        all = fmaxf(all, m[u]);
        add(f, part, clamped);
      }
    };
    if (clamp) pass(true);
    else pass(false);
    const bool odd = (TOP || !clamp) && __ballot(part.E != part.E) != 0, infinite = !clamp && odd;
    if constexpr (TOP) {
      // A maximum with a signaling NaN forgets what it was before: where there
      // may be one, the vectors' largest are taken again without any NaN.
      if (odd) {
        all = -INFINITY;
#pragma unroll
        for (int u = 0; u < kLpUnroll; ++u) {
          u32x4_t x = cur[u];
          asm("" : "+v"(x));  // (as above)
          float f[N];
          Vec16<T>::open(x, f);
          m[u] = -INFINITY;
#pragma unroll
          for (int e = 0; e < N; ++e) m[u] = f[e] > m[u] ? f[e] : m[u];
          all = fmaxf(all, m[u]);
        }
      }
    }
    if (infinite || __ballot((all - s.r) * a.c > kLift)) {
      clamp |= infinite;
      move_to(s, fmaxf(s.r, wave_max(all)), a.c);
      part = Sums{s.r, 0.f, 0.f};
#pragma unroll 1
      for (int u = 0; u < kLpUnroll; ++u) {
        float f[N];
        Vec16<T>::open(u == 0 ? cur[0] : u == 1 ? cur[1] : u == 2 ? cur[2] : cur[3], f);
        add(f, part, true);
      }
    }
    s.S += part.S;
    s.E += part.E;
    if constexpr (TOP) {
      if (v0 + CHUNK <= end) {
        best = fmaxf(best, all);
        if (seen > 1 && (seen & (seen - 1)) == 0) {
          const uint32_t b = lanes_bound();
          if (lane == 0) __hip_atomic_store(w_bound + w, b, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
          use_bounds();  // (another wave's may be an earlier one: a lower bound all the same)
        }
      }
      if (__ballot(all >= top.least)) {
#pragma unroll
        for (int u = 0; u < kLpUnroll; ++u) top.note(m[u], v0 + u * THREADS + t, cur[u]);
      }
    }
  };
  for (int v0 = begin, seen = 1; v0 < end; v0 += 2 * CHUNK, seen += 2) {
    load(odd, v0 + CHUNK);
    chunk(even, v0, seen);
    if constexpr (TOP)
      if (top.vectors > 64) top.look(head, end);
    load(even, v0 + 2 * CHUNK);
    if (v0 + CHUNK < end) chunk(odd, v0 + CHUNK, seen + 1);
    if constexpr (TOP)
      if (top.vectors > 64 || v0 + 2 * CHUNK >= end) top.look(head, end);
  }
  // Each wave's results, then the first one's of all waves; for a row of
  // several slices that twice, the second time of the slices' results.
#pragma unroll 1
  for (int stage = 0;; ++stage) {
    if (w == 0 || !(stage & 1)) {
      s = wave_sums(s, a.c);
      if constexpr (TOP) top.n = keep_largest<LOW>(top.buf, top.n, a.k, top.bits);
    }
    if (!(stage & 1)) {
      if (lane == 0) {
        w_r[w] = s.r;
        w_S[w] = s.S;
        w_E[w] = s.E;
        w_n[w] = top.n;
      }
      __syncthreads();
      if (w == 0) {
        s = Sums{lane < W ? w_r[lane] : kLowest, lane < W ? w_S[lane] : 0.f,
                 lane < W ? w_E[lane] : 0.f};
        if constexpr (TOP)
          for (int i = 1; i < W; ++i) {
            const int n = w_n[i];
            if (lane < n) top.buf[top.n + lane] = keys[i][lane];
            top.n += n;
          }
      }
      continue;
    }
    if (stage == 3 || a.slices == 1) {
      if (w == 0) put_row<T, TOP>(a, r, s, tok, x_tok, top.buf, top.n);
      return;
    }
    if (w == 0) {
      float *ps = (float *)(a.part_sums + r * a.slices + slice);
      if (lane < 3) put_shared(ps + lane, lane == 0 ? s.r : lane == 1 ? s.S : s.E);
      if constexpr (TOP) {
        if (lane < a.k) put_shared(a.part_keys + (r * a.slices + slice) * a.k + lane, lane < top.n ? top.buf[lane] : 0);
      }
      __builtin_amdgcn_s_waitcnt(0);  // in before the arrival counts
      if (lane == 0)
        last = __hip_atomic_fetch_add(a.counters + r * kCounterStep, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == a.slices - 1;
    }
    __syncthreads();
    if (!last) return;
    if (t == 0) put_shared(a.counters + r * kCounterStep, 0);
    s = Sums{kLowest, 0.f, 0.f};
    top.n = 0;
    if (t < a.slices) {
      float *ps = (float *)(a.part_sums + r * a.slices + t);
      s = Sums{get_shared(ps), get_shared(ps + 1), get_shared(ps + 2)};
    }
    if constexpr (TOP) {
      uint64_t *pk = a.part_keys + r * a.slices * a.k;
      for (int i = t - lane; i < a.slices * a.k; i += THREADS) {  // (kMostKeys: they fit)
        const uint64_t key = i + lane < a.slices * a.k ? get_shared(pk + i + lane) : 0;
        const uint64_t mask = __ballot(key != 0);
        if (key != 0) top.buf[top.n + lanes_below(mask)] = key;
        top.n += __popcll(mask);
      }
    }
  }
}

struct LogprobPlan {
  int slices, per_slice;
};

// Slices of a row: about kLpFill workgroups in all.  128,256 bf16 logits and
// 20 alternatives, us, with about 256, 512 and 1024 workgroups: 64 rows 14.6,
// 13.5, 15.4; 130 rows 19.4, 17.5, 19.0; 200 rows 23.0, 20.5, 21.1; 300 rows
// 27.6, 24.6, 24.4 (of 32,000 logits 12.7, 14.0, 13.9); 500 rows (one slice,
// one, two) 28.5, 28.4, 31.7.
constexpr int kLpFill = 512;
// Rows of up to kLpShort vectors are one wave's, longer ones where there are
// many rows: a wave alone has less to do once a row, and waits at no barrier.
// Four waves and one, us, bf16 logits, 20 alternatives:
//   9000 (1125 vectors) 1300 rows 15.9, 14.2; 5000 rows 44.1, 27.9
//   16,000 (2000)       1300 17.9, 18.6; 1536 19.7, 18.8; 5000 50.4, 42.0
//   32,000 (4000)       1536 25.9, 30.6; 1700 28.7, 31.1; 1850 32.8, 31.3; 5000 77.7, 72.0
//   50,257 (6282)       1536 36.8, 42.3; 1700 41.1, 42.4; 1850 44.6, 42.5; 8192 169, 156
//   128,256 (16,032)    2000 91, 95; 4096 179, 178 (two full rounds of 2048 waves; 201, 195 with likely
//                       tokens); 4150 204, 213; 6000 258, 278; 8192 346, 363
// (without alternatives one wave gains less, and loses up to 15% for 2000 to
// 8192 vectors.)  Four waves take 1024 vectors at a time: 66,000 logits, 8250
// vectors, would be one wave's by 9%, 65,000 and 70,000 are not.
constexpr int kLpShort = 1024;
constexpr int kLpMiddle = 2048, kLpManyMiddle = 1536;  // up to so many vectors: from this many rows on
constexpr int kLpLong = 8192, kLpManyLong = 1792;

static bool one_wave_rows(int rows, int nvec) {
  return nvec <= kLpShort || (nvec <= kLpMiddle && rows >= kLpManyMiddle) || (nvec <= kLpLong && rows >= kLpManyLong);
}

// (no row is cut beyond kLpFill rows, so its counter is within the first 64 KiB)
static_assert(kLpFill * kCounterStep * sizeof(int) <= 65536, "counters");

// Rows of a launch: its threads are counted in 32 bits, 256 a row at most.
constexpr int64_t kLpLaunchRows = 1 << 23;

static LogprobPlan plan_logprobs(int rows, int vocab, int k) {
  const int nvec = vocab / 4 + 1;  // (of fp32; bf16 rows have half as many)
  const int chunks = (nvec + kLpChunk - 1) / kLpChunk;
  int slices = rows > 0 && rows < kLpFill ? (kLpFill + rows / 2) / rows : 1;
  slices = slices < chunks ? slices : chunks;
  slices = slices < kMostSlices ? slices : kMostSlices;
  if (k > 0 && slices > kMostKeys / k) slices = kMostKeys / k;
  return LogprobPlan{slices < 1 ? 1 : slices, 0};
}

}  // namespace sm

using namespace sm;

SM_API size_t sm_token_logprobs_workspace_bytes(int rows, int vocab, int k) {
  if (rows < 0 || vocab < 1 || k < 0 || k > SM_MAX_TOP || k > vocab) return 0;
  const LogprobPlan p = plan_logprobs(rows, vocab, k);
  return 65536 + (p.slices > 1 ? (size_t)rows * p.slices * (16 + 8 * (size_t)k) : 0);
}

SM_API sm_status sm_token_logprobs(const void *logits, int64_t stride, int rows, int vocab, sm_dtype dt, float scale,
                                   const int32_t *tokens, float *logprob, float *entropy, int k, int32_t *top_ids,
                                   float *top_logprobs, void *ws, size_t ws_bytes, int32_t *err, hipStream_t stream) {
  if ((dt != SM_F32 && dt != SM_BF16) || rows < 0 || vocab < 1 || k < 0 || k > SM_MAX_TOP || k > vocab) return SM_EINVAL;
  const float c = (float)(scale * 1.4426950408889634);
  // (a chunk's terms p |d| are at most 2^kLift kLift ln 2 / scale = 44 / scale, for d below the reference at most
  // 1 / (e scale): from a scale of 1e-20 on 2^31 of them come to at most 1e31)
  if (!(scale >= 1e-20f) || !std::isfinite(c) || stride < vocab) return SM_EINVAL;
  if (rows == 0) return SM_OK;
  if (!logits || (logprob && !tokens) || (k > 0 && !top_ids) || (uintptr_t)ws % 16 != 0) return SM_EINVAL;
  if (!ws || ws_bytes < sm_token_logprobs_workspace_bytes(rows, vocab, k)) return SM_EINVAL;
  const int n = dt == SM_BF16 ? 8 : 4;
  LogprobPlan p = plan_logprobs(rows, vocab, k);
  const int nvec = vocab / n + 1, chunks = (nvec + kLpChunk - 1) / kLpChunk;
  p.per_slice = (chunks + p.slices - 1) / p.slices * kLpChunk;
  p.slices = (nvec + p.per_slice - 1) / p.per_slice;
  float4 *sums = (float4 *)((char *)ws + 65536);
  LogprobArgs a{logits, stride, rows, vocab, k, scale, c, tokens, logprob, entropy, top_ids, top_logprobs, err,
                      p.slices, p.per_slice, (int *)ws, sums, (uint64_t *)(sums + (size_t)rows * p.slices)};
  const bool bf = dt == SM_BF16;
  const bool short_row = p.slices == 1 && one_wave_rows(rows, nvec);
  const auto kernel =
      short_row ? (bf ? (k ? logprobs_kernel<uint16_t, true, 1> : logprobs_kernel<uint16_t, false, 1>)
                      : (k ? logprobs_kernel<float, true, 1> : logprobs_kernel<float, false, 1>))
                : (bf ? (k ? logprobs_kernel<uint16_t, true, kLpWaves> : logprobs_kernel<uint16_t, false, kLpWaves>)
                      : (k ? logprobs_kernel<float, true, kLpWaves> : logprobs_kernel<float, false, kLpWaves>));
  for (int64_t r = 0; r < rows; r += kLpLaunchRows) {
    a.rows = (int)std::min(rows - r, kLpLaunchRows);
    a.logits = row_at(logits, r, stride, 16 / n);
    a.tokens = (const int32_t *)row_at(tokens, r, 1, 4);
    a.logprob = (float *)row_at(logprob, r, 1, 4);
    a.entropy = (float *)row_at(entropy, r, 1, 4);
    a.top_ids = (int32_t *)row_at(top_ids, r, k, 4);
    a.top_logprobs = (float *)row_at(top_logprobs, r, k, 4);
    hipLaunchKernelGGL(kernel, dim3((unsigned)(a.rows * p.slices)), dim3(short_row ? 64 : 64 * kLpWaves), 0, stream, a);
    if (hipGetLastError() != hipSuccess) return SM_EHIP;
  }
  return SM_OK;
}
