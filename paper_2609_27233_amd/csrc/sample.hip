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
// workgroups, waves and atomics may add them as they come.  Of V tokens the
// roundings come to V x 2^-45 of the largest weight at most (2^-28 for 128,256,
// 2^-26 for the most that a row may have); as a rule, over 128,256, to 2^-37.
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
// where the filter ends, a k of thousands, logits hundreds apart, or all of them
// so far below the bins' origin that the histogram holds no mass) is cut by
// passes over the whole row, in `choose`, to the same result.
//
// Such a row is slow: one workgroup passes over it several times.  Us for 16
// rows of 128,256 bf16 logits: k = 50 22, 5000 687; p = 0.9 28, of nearly equal
// logits 960, of equal ones 506; p = 0.9 and min-p 1e-4 at T = 4 1020; k = 50000
// and p = 0.9 1190.  1024 rows: k = 50 162, 5000 1690; p = 0.9 269, of nearly
// equal logits 2650.  So is one whose first 512 logits lie more than 22 below the
// rest without being -infinity (a mask of -1e4 or of the type's lowest value):
// all of the rest falls into the first bin, and k = 50 takes 533, p = 0.9 1020
// (masked by -infinity 22 and 28).
//
// 1024 rows of 128,256 bf16 logits, mixed filters: scan 69 us, weigh 108,
// choose 23; all greedy, which are read once, 70 in all (scan 58 at 4.5 TB/s, 12
// of two launches that find nothing to do; 123 with their ties counted by
// weigh).  By filter: none 183, top-k 153, top-p 277, min-p 137; 400 rows of
// fp32 95, 94, 147, 83, greedy 50; 16 rows of bf16 14, 22, 31, 14, greedy 11.
// The vector ALU and the two reads bound it (20 and 37 instructions a logit; a
// read alone would take 39 us): LDS atomics and an exponential, and the nine
// products in double precision of a weight.  (Weights from a table of the bf16
// values in LDS: 222 for 207 in all, for the waves that its 32 KB displace.)  16
// rows: 6, 11 and 14 us, a chain of dependent reads and barriers.  Rows fewer at
// a time, or a slice's loads before the bins are known, took longer.
#include <algorithm>
#include <cmath>
#include <cstddef>
#include <type_traits>

#include "common.hpp"

namespace sm {

constexpr int kSampThreads = 256, kSampWaves = kSampThreads / 64;
constexpr int kPiece = 512;                    // tokens of a piece: 8 a lane
constexpr int kMostVocab = 1 << 19;            // 2^44 times this many is 2^63: a mass fits 64 bits
constexpr int kMostPieces = kMostVocab / kPiece;
constexpr int kInFlight = 4;                   // pieces that a wave loads at a time
constexpr int kUnit = 44;                      // a weight of 1 is 2^44
constexpr double kLeast = -46.0;               // exponents from here down weigh nothing (2^-45 and its half on)
constexpr double kLog2eD = 1.4426950408889634073599246810019;

// The histogram: bins of 1/23 in the logits, the first 512 above the largest
// of the row's first piece.
constexpr int kBins = 2048, kBinsAbove = 512;
constexpr float kBinsPerUnit = 16.f * 1.44269504f;
constexpr float kSharpest = 0.25f;             // temperatures below go by a list of all that weighs anything
constexpr int kList = 4096;                    // tokens that are cut in LDS
constexpr int kCutBins = 1024;

// What a row has in the workspace.  The first part is zero between calls.  The
// bins are read and cleared 16 bytes at a time.
struct alignas(16) RowState {
  uint32_t top;       // key of M
  uint32_t bad;       // a NaN
  uint32_t listed;    // tokens listed; more than kList: not all of them
  uint32_t unused;
  uint64_t mass;      // of all tokens (kMass); greedy: key of M << 32 | ~its first token
  alignas(16) uint32_t bins[kBins];
  // not cleared
  uint64_t pieces[kMostPieces];  // ties << 54 | mass
  uint64_t list[kList];          // key << 32 | token
};
static_assert(offsetof(RowState, bins) % 16 == 0 && sizeof(RowState) % 16 == 0, "16-byte accesses to the bins of any row");
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

// 2^t for t <= 0 in multiples of 2^-44, to nearest (so 0 from 2^-45 on), as the
// low bits of a double of 2^52 and that many; table: 2^(44 + j / 128).  t = k /
// 128 + r, |r| <= 2^-8, 2^r = e^(r ln 2) to its fourth power: the next term is
// below 2^-49.  The binary exponent goes into the table's entry.
constexpr uint64_t kZeroWeight = 0x4330000000000000ull;  // 2^52 as bits
__device__ __forceinline__ uint64_t weight_bits(double t, const double *table) {
  constexpr double ln2 = 0.69314718055994530941723212145818;
  constexpr double c1 = ln2, c2 = c1 * ln2 / 2, c3 = c2 * ln2 / 3, c4 = c3 * ln2 / 4;
  constexpr double magic = 6755399441055744.0;  // 1.5 x 2^52: a sum with it is a whole number in its low bits
  t = fmax(t, -100.0);                          // (and -infinity)
  const double sum = fma(t, 128.0, magic);
  const int k = (int)__double_as_longlong(sum);
  const double r = fma(sum - magic, -0.0078125, t);
  double p = fma(r, c4, c3);
  p = fma(r, p, c2);
  p = fma(r, p, c1);
  p = fma(r, p, 1.0);
  const double entry = table[k & 127];
  const double power = __hiloint2double(__double2hiint(entry) + ((k & ~127) << 13), __double2loint(entry));
  return __double_as_longlong(fma(power, p, 4503599627370496.0));
}
__device__ __forceinline__ uint64_t unit_weight(double t, const double *table) { return weight_bits(t, table) - kZeroWeight; }

// 2^(j / 128), rounded to double precision
__constant__ double kPowers[128] = {
    0x1.0000000000000p+0, 0x1.0163da9fb3335p+0, 0x1.02c9a3e778061p+0, 0x1.04315e86e7f85p+0,
    0x1.059b0d3158574p+0, 0x1.0706b29ddf6dep+0, 0x1.0874518759bc8p+0, 0x1.09e3ecac6f383p+0,
    0x1.0b5586cf9890fp+0, 0x1.0cc922b7247f7p+0, 0x1.0e3ec32d3d1a2p+0, 0x1.0fb66affed31bp+0,
    0x1.11301d0125b51p+0, 0x1.12abdc06c31ccp+0, 0x1.1429aaea92de0p+0, 0x1.15a98c8a58e51p+0,
    0x1.172b83c7d517bp+0, 0x1.18af9388c8deap+0, 0x1.1a35beb6fcb75p+0, 0x1.1bbe084045cd4p+0,
    0x1.1d4873168b9aap+0, 0x1.1ed5022fcd91dp+0, 0x1.2063b88628cd6p+0, 0x1.21f49917ddc96p+0,
    0x1.2387a6e756238p+0, 0x1.251ce4fb2a63fp+0, 0x1.26b4565e27cddp+0, 0x1.284dfe1f56381p+0,
    0x1.29e9df51fdee1p+0, 0x1.2b87fd0dad990p+0, 0x1.2d285a6e4030bp+0, 0x1.2ecafa93e2f56p+0,
    0x1.306fe0a31b715p+0, 0x1.32170fc4cd831p+0, 0x1.33c08b26416ffp+0, 0x1.356c55f929ff1p+0,
    0x1.371a7373aa9cbp+0, 0x1.38cae6d05d866p+0, 0x1.3a7db34e59ff7p+0, 0x1.3c32dc313a8e5p+0,
    0x1.3dea64c123422p+0, 0x1.3fa4504ac801cp+0, 0x1.4160a21f72e2ap+0, 0x1.431f5d950a897p+0,
    0x1.44e086061892dp+0, 0x1.46a41ed1d0057p+0, 0x1.486a2b5c13cd0p+0, 0x1.4a32af0d7d3dep+0,
    0x1.4bfdad5362a27p+0, 0x1.4dcb299fddd0dp+0, 0x1.4f9b2769d2ca7p+0, 0x1.516daa2cf6642p+0,
    0x1.5342b569d4f82p+0, 0x1.551a4ca5d920fp+0, 0x1.56f4736b527dap+0, 0x1.58d12d497c7fdp+0,
    0x1.5ab07dd485429p+0, 0x1.5c9268a5946b7p+0, 0x1.5e76f15ad2148p+0, 0x1.605e1b976dc09p+0,
    0x1.6247eb03a5585p+0, 0x1.6434634ccc320p+0, 0x1.6623882552225p+0, 0x1.68155d44ca973p+0,
    0x1.6a09e667f3bcdp+0, 0x1.6c012750bdabfp+0, 0x1.6dfb23c651a2fp+0, 0x1.6ff7df9519484p+0,
    0x1.71f75e8ec5f74p+0, 0x1.73f9a48a58174p+0, 0x1.75feb564267c9p+0, 0x1.780694fde5d3fp+0,
    0x1.7a11473eb0187p+0, 0x1.7c1ed0130c132p+0, 0x1.7e2f336cf4e62p+0, 0x1.80427543e1a12p+0,
    0x1.82589994cce13p+0, 0x1.8471a4623c7adp+0, 0x1.868d99b4492edp+0, 0x1.88ac7d98a6699p+0,
    0x1.8ace5422aa0dbp+0, 0x1.8cf3216b5448cp+0, 0x1.8f1ae99157736p+0, 0x1.9145b0b91ffc6p+0,
    0x1.93737b0cdc5e5p+0, 0x1.95a44cbc8520fp+0, 0x1.97d829fde4e50p+0, 0x1.9a0f170ca07bap+0,
    0x1.9c49182a3f090p+0, 0x1.9e86319e32323p+0, 0x1.a0c667b5de565p+0, 0x1.a309bec4a2d33p+0,
    0x1.a5503b23e255dp+0, 0x1.a799e1330b358p+0, 0x1.a9e6b5579fdbfp+0, 0x1.ac36bbfd3f37ap+0,
    0x1.ae89f995ad3adp+0, 0x1.b0e07298db666p+0, 0x1.b33a2b84f15fbp+0, 0x1.b59728de5593ap+0,
    0x1.b7f76f2fb5e47p+0, 0x1.ba5b030a1064ap+0, 0x1.bcc1e904bc1d2p+0, 0x1.bf2c25bd71e09p+0,
    0x1.c199bdd85529cp+0, 0x1.c40ab5fffd07ap+0, 0x1.c67f12e57d14bp+0, 0x1.c8f6d9406e7b5p+0,
    0x1.cb720dcef9069p+0, 0x1.cdf0b555dc3fap+0, 0x1.d072d4a07897cp+0, 0x1.d2f87080d89f2p+0,
    0x1.d5818dcfba487p+0, 0x1.d80e316c98398p+0, 0x1.da9e603db3285p+0, 0x1.dd321f301b460p+0,
    0x1.dfc97337b9b5fp+0, 0x1.e264614f5a129p+0, 0x1.e502ee78b3ff6p+0, 0x1.e7a51fbc74c83p+0,
    0x1.ea4afa2a490dap+0, 0x1.ecf482d8e67f1p+0, 0x1.efa1bee615a27p+0, 0x1.f252b376bba97p+0,
    0x1.f50765b6e4540p+0, 0x1.f7bfdad9cbe14p+0, 0x1.fa7c1819e90d8p+0, 0x1.fd3c22b8f71f1p+0,
};
__device__ __forceinline__ void fill_table(double *table) {
  if (threadIdx.x < 128) table[threadIdx.x] = kPowers[threadIdx.x] * (double)(1ull << kUnit);
}

// ---- sums ------------------------------------------------------------------
// Scans by lane permutations in the vector ALU: shifts by 1, 2, 4 and 8 within
// rows of 16 lanes, then each row's last lane to the rows behind it.  (Through
// LDS, as __shfl does it, a scan of 64 bits took 0.4 us of a call's chain.)
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t lane_moved(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xf, true);  // 0 where nothing moves in
}
template <int CTRL, int ROWS = 0xf>
__device__ __forceinline__ uint64_t moved(uint64_t v) {
  return (uint64_t)lane_moved<CTRL, ROWS>((uint32_t)(v >> 32)) << 32 | lane_moved<CTRL, ROWS>((uint32_t)v);
}
template <int CTRL, int ROWS = 0xf>
__device__ __forceinline__ float moved(float v) {
  return __uint_as_float(lane_moved<CTRL, ROWS>(__float_as_uint(v)));
}
template <typename V>
__device__ __forceinline__ V wave_scan(V v) {
  v += moved<0x111>(v);       // row_shr:1, 2, 4, 8
  v += moved<0x112>(v);
  v += moved<0x114>(v);
  v += moved<0x118>(v);
  v += moved<0x142, 0xa>(v);  // row_bcast:15 into rows 1 and 3
  v += moved<0x143, 0xc>(v);  // row_bcast:31 into rows 2 and 3
  return v;
}
__device__ __forceinline__ uint64_t last_lane(uint64_t v) {
  return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), 63) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}
__device__ __forceinline__ float last_lane(float v) {
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}
__device__ __forceinline__ uint32_t wave_max_u32(uint32_t v) {
  v = max(v, lane_moved<0x111, 0xf>(v));
  v = max(v, lane_moved<0x112, 0xf>(v));
  v = max(v, lane_moved<0x114, 0xf>(v));
  v = max(v, lane_moved<0x118, 0xf>(v));
  v = max(v, lane_moved<0x142, 0xa>(v));
  v = max(v, lane_moved<0x143, 0xc>(v));
  return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}
__device__ __forceinline__ uint64_t wave_sum64(uint64_t v) { return last_lane(wave_scan(v)); }
// Inclusive over the workgroup.  red: one value a wave, in turn two places, so
// that one barrier a scan does.
struct Red {
  uint64_t v[2][kSampWaves];
};
template <typename V>
__device__ __forceinline__ V block_scan(V v, Red &red, int &turn, V *total) {
  const int w = threadIdx.x >> 6;
  v = wave_scan(v);
  V *r = (V *)red.v[turn ^= 1];
  if ((threadIdx.x & 63) == 63) r[w] = v;
  __syncthreads();
  V before = 0, all = 0;
#pragma unroll
  for (int i = 0; i < kSampWaves; ++i) {
    if (i < w) before += r[i];
    all += r[i];
  }
  *total = all;
  return v + before;
}
// The least value over the workgroup of the threads that have one, kNone of
// none; values ascend with the thread.  (An atomic minimum of every lane's own
// value at one place would be taken lane by lane.)
constexpr int kNone = 0x7fffffff;
__device__ __forceinline__ int block_first(bool has, int value, Red &red, int &turn) {
  const int w = threadIdx.x >> 6;
  const uint64_t who = __ballot(has);
  int *r = (int *)red.v[turn ^= 1];
  const int first = __builtin_amdgcn_readlane(value, who ? __builtin_ctzll(who) : 0);
  if ((threadIdx.x & 63) == 0) r[w] = who ? first : kNone;
  __syncthreads();
  int least = kNone;
#pragma unroll
  for (int i = kSampWaves - 1; i >= 0; --i)
    if (r[i] != kNone) least = r[i];
  return least;
}

// ---- a row -----------------------------------------------------------------

// Tokens with keys above `tie`, and `ties` of those equal to it.
struct Kept {
  uint32_t tie;
  uint32_t ties;
};

enum Mode {
  kPlain,  // the pieces' masses, of the tokens that min_p keeps (greedy: `scan` has found the token)
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
  // (loaded at once: what is not given from where u is)
  const float u = a.u[r], t0 = (a.temperature ? a.temperature : a.u)[r], p0 = (a.top_p ? a.top_p : a.u)[r];
  const float m0 = (a.min_p ? a.min_p : a.u)[r];
  const int k0 = (a.top_k ? a.top_k : (const int32_t *)a.u)[r];
  const float t = a.temperature ? t0 : 1.f, p = a.top_p ? p0 : 1.f, m = a.min_p ? m0 : 0.f;
  const int k = a.top_k ? k0 : 0;
  Settings s;
  s.u = u;
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
    int p = p0 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (p >= p1) return;
    Eight f[kInFlight];
#pragma unroll
    for (int i = 0; i < kInFlight; ++i) f[i] = raw(min(p + i * kSampWaves, p1 - 1));
    while (true) {
#pragma unroll
      for (int i = 0; i < kInFlight; ++i) {
        g(f[i], p);
        if (p + kInFlight * kSampWaves < p1) f[i] = raw(p + kInFlight * kSampWaves);
        p += kSampWaves;
        if (p >= p1) return;
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
  __shared__ uint32_t bins[kBins + 64];  // and a place a lane for what is masked, so that no lane has to leave
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
    const auto fill = [&](auto of_masses) {
      row.each_piece(p0, p1, [&](const typename Row<T>::Eight &f, int) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float v = f[e];
          nan |= v != v;
          M = fmaxf(M, v);
          const float d = row.depth(v), b = floorf(fminf(d, (float)(kBins - 1)));
          uint32_t part = 1;
          if constexpr (of_masses) part = (uint32_t)fmaf(__builtin_amdgcn_exp2f((b - d) * slope), one, 0.5f);
          atomicAdd(&bins[v > -INFINITY ? (int)b : kBins + lane], part);
        }
      });
    };
    if (masses) fill(std::true_type());
    else fill(std::false_type());
    __syncthreads();
    for (int i = t; i < kBins; i += kSampThreads)
      if (bins[i]) atomicAdd(&st.bins[i], bins[i]);
  } else if (s.greedy) {
    int at = 0;  // the first token of M: a lane's ascend
    row.each_piece(p0, p1, [&](const typename Row<T>::Eight &f, int p) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float v = f[e];
        nan |= v != v;
        at = v > M ? p * kPiece + 8 * lane + e : at;
        M = v > M ? v : M;
      }
    });
    const float most = wave_max(M);
    const uint32_t first = wave_max_u32(M == most ? ~(uint32_t)at : 0u);
    if (lane == 0 && most > -INFINITY) atomicMax((unsigned long long *)&st.mass, (uint64_t)order_key(most) << 32 | first);
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
__device__ __forceinline__ Range end_bins(const RowState &st, const Settings &s, float top_depth, int vocab, Red &red, int &turn) {
  constexpr int N = kBins / kSampThreads;
  const int t = threadIdx.x;
  u32x4_t raw[N / 4];
#pragma unroll
  for (int i = 0; i < N / 4; ++i) raw[i] = *(const u32x4_t *)(st.bins + N * t + 4 * i);
  if (s.mode == kListK) {
    uint64_t n = 0, total;
#pragma unroll
    for (int i = 0; i < N; ++i) n += raw[i / 4][i % 4];
    uint64_t at = block_scan(n, red, turn, &total) - n;
    const bool here = at < (uint64_t)s.k && at + n >= (uint64_t)s.k;
    int b = 0;
#pragma unroll
    for (int i = N - 1; i >= 0; --i) {  // the first bin at which k are reached
      if (at + n >= (uint64_t)s.k) b = i;
      n -= raw[i / 4][i % 4];
    }
    const int last = block_first(here, N * t + b, red, turn);
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
  float at = block_scan(sum, red, turn, &total);
  if (!(total > 0.f)) return Range{kNone, kNone};
  const float slack = (0.5f / one + 2e-6f) * total, lo = s.p * total - slack, hi = s.p * total + slack;
  int b1 = kNone, b2 = kNone;
#pragma unroll
  for (int i = N - 1; i >= 0; --i) {
    if (at >= lo) b1 = N * t + i;
    if (at >= hi) b2 = N * t + i;
    at -= m[i];
  }
  b1 = block_first(b1 != kNone, b1, red, turn);
  b2 = block_first(b2 != kNone, b2, red, turn);
  return Range{b1, min(b2, kBins - 1)};
}

// tokens that a workgroup of `weigh` gathers before it takes their places in the row's list
constexpr int kSliceList = 1024;

template <typename T>
__global__ __launch_bounds__(kSampThreads) void sample_weigh_kernel(SampleArgs a) {
  __shared__ double table[128];
  __shared__ uint64_t list[kSliceList];
  __shared__ Red red;
  int turn = 0;
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
  if (!s.fine || s.greedy || st.bad || top == 0 || !(row.M < INFINITY)) return;
  row.c = s.c;
  fill_table(table);
  if (t == 0) listed = 0;
  Range range{0, -1};
  if (s.mode == kListK || s.mode == kMass) {
    row.set_origin();
    range = end_bins(st, s, row.depth(row.M), a.vocab, red, turn);
    if (range.first == kNone) {  // (masses that came to nothing)
      if (t == 0 && p0 == 0) atomicAdd(&st.listed, kList + 1);
      return;
    }
  }
  __syncthreads();
  // takes the marked ones of a lane's eight tokens into the list: one place in it a wave and piece
  const auto add = [&](const typename Row<T>::Eight &f, int p, const bool (&take)[8]) {
    int at[8], n = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint64_t who = __ballot(take[e]);
      at[e] = n + __builtin_amdgcn_mbcnt_hi((uint32_t)(who >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)who, 0));
      n += __popcll(who);
    }
    if (n == 0) return;
    int base = 0;
    if (lane == 0) base = atomicAdd(&listed, n);
    base = __builtin_amdgcn_readfirstlane(base);
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (take[e] && base + at[e] < kSliceList)
        list[base + at[e]] = (uint64_t)order_key(f[e]) << 32 | (uint32_t)(p * kPiece + 8 * lane + e);
  };
  const double lm = s.mode == kListM ? fmax(s.lm, kLeast) : s.lm;
  // a depth below the first lies in a bin above the range, one up to the second in it or above (the last bin's
  // logits may lie at an infinite depth)
  const float above_range = (float)range.first;
  const float in_range = range.last < kBins - 1 ? __uint_as_float(__float_as_uint((float)(range.last + 1)) - 1) : INFINITY;
  if (s.mode == kListK) {
    row.each_piece(p0, p1, [&](const typename Row<T>::Eight &f, int p) {
      bool take[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) take[e] = f[e] > -INFINITY && row.depth(f[e]) <= in_range;
      add(f, p, take);
    });
  } else if (s.mode == kListM) {
    row.each_piece(p0, p1, [&](const typename Row<T>::Eight &f, int p) {
      bool take[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) take[e] = f[e] > -INFINITY && row.exponent(f[e]) >= lm;
      add(f, p, take);
    });
  } else if (s.mode == kMass) {
    uint64_t S = 0;
    row.each_piece(p0, p1, [&](const typename Row<T>::Eight &f, int p) {
      uint64_t above = 0, all = 0;
      int n = 0;
      bool take[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint64_t m = weight_bits(row.exponent(f[e]), table);
        const float d = row.depth(f[e]);
        const bool over = d < above_range;
        all += m;
        above += over ? m : 0;
        n += over;
        take[e] = !over && d <= in_range && f[e] > -INFINITY;
      }
      S += all - 8 * kZeroWeight;
      above = wave_sum64(above - n * kZeroWeight);
      if (lane == 0) st.pieces[p] = above;
      add(f, p, take);
    });
    S = wave_sum64(S);
    if (lane == 0) atomicAdd((unsigned long long *)&st.mass, S);
  } else if (lm > -INFINITY) {
    row.each_piece(p0, p1, [&](const typename Row<T>::Eight &f, int p) {
      uint64_t sum = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const double ex = row.exponent(f[e]);
        if (ex >= lm) sum += unit_weight(ex, table);
      }
      sum = wave_sum64(sum);
      if (lane == 0) st.pieces[p] = sum;
    });
  } else {
    row.each_piece(p0, p1, [&](const typename Row<T>::Eight &f, int p) {
      uint64_t sum = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) sum += weight_bits(row.exponent(f[e]), table);
      sum = wave_sum64(sum - 8 * kZeroWeight);
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
  Red red;
  uint32_t lo[kSampWaves], hi[kSampWaves];
  uint64_t before, amount;       // mass (or count) above the bin, and in it
  int bin, left;
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
#pragma unroll 1
        for (int e = 0; e < 8; ++e) {
          float x = v[0];
#pragma unroll
          for (int i = 1; i < 8; ++i) x = e == i ? v[i] : x;
          if (x > -INFINITY) f(x, order_key(x), p * kPiece + 8 * (int)(threadIdx.x & 63) + e);
        }
      }
    }
  }
};

// The smallest start of the kept ones of these tokens, in descending order, at
// which `before` plus their amount (MASS: of their masses; else their number)
// reaches the target, or all of them.  All threads; returns the same in each.
// Rounds of 1024 bins over the keys from the largest down (of bf16 the upper
// halves, which are all there is to them): one for a list of bf16, two or
// three for fp32.  false: the target lies before these tokens or behind them, or
// there are none.
template <bool MASS, typename T>
__device__ __forceinline__ bool cut(const Row<T> &row, const Tokens<T> &tokens, Kept &kept, double lm, uint64_t before, uint64_t target,
                                 ChooseShared &sh, int &turn) {
  constexpr int DROP = 32 - 8 * sizeof(T);  // bits of a key that say nothing
  const int t = threadIdx.x, w = t >> 6;
  const auto amount = [&](float v) { return MASS ? unit_weight(row.exponent(v), sh.table) : (uint64_t)1; };
  const bool tie_in = kept.ties > 0 && row.exponent(value_of_key(kept.tie)) >= lm;
  const Kept was = kept;
  // ---- least and largest key ----
  uint32_t lo = 0xffffffffu, hi = 0;
  tokens.each([&](float v, uint32_t key, int) {
    if (key <= was.tie || row.exponent(v) < lm) return;
    lo = min(lo, key >> DROP);
    hi = max(hi, key >> DROP);
  });
  if (tie_in) lo = was.tie >> DROP;  // (the others are above it)
  hi = max(hi, tie_in ? was.tie >> DROP : 0u);
  hi = wave_max_u32(hi);
  lo = ~wave_max_u32(~lo);
  if ((t & 63) == 0) {
    sh.lo[w] = lo;
    sh.hi[w] = hi;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kSampWaves; ++i) {
    lo = min(lo, sh.lo[i]);
    hi = max(hi, sh.hi[i]);
  }
  if (hi == 0) return false;  // no tokens
  for (;;) {
    int shift = 0;
    while ((hi - lo) >> shift >= (uint32_t)kCutBins) ++shift;
    for (int i = t; i < kCutBins; i += kSampThreads) sh.mass[i] = sh.count[i] = 0;
    __syncthreads();
    // ---- amounts by bins ----
    tokens.each([&](float v, uint32_t key, int) {
      const uint32_t k = key >> DROP;
      if (key <= was.tie || k < lo || k > hi || row.exponent(v) < lm) return;
      const int b = (hi - k) >> shift;
      const uint64_t each = amount(v);
      // the commonest values of a wave's tokens are counted first: a bin takes one add of each, not one of every token
      bool left = true;
      for (int i = 0; i < 4 && left; ++i) {
        const uint32_t first = __builtin_amdgcn_readfirstlane(k);
        const uint64_t who = __ballot(k == first);
        if (k != first) continue;
        left = false;
        if ((t & 63) == __builtin_ctzll(who)) {
          atomicAdd(&sh.count[b], (uint32_t)__popcll(who));
          if constexpr (MASS) atomicAdd((unsigned long long *)&sh.mass[b], each * __popcll(who));
        }
      }
      if (!left) return;
      atomicAdd(&sh.count[b], 1u);
      if constexpr (MASS) atomicAdd((unsigned long long *)&sh.mass[b], each);
    });
    if (t == 0 && tie_in && was.tie >> DROP >= lo) {
      const int b = (hi - (was.tie >> DROP)) >> shift;
      atomicAdd(&sh.count[b], was.ties);
      if constexpr (MASS) atomicAdd((unsigned long long *)&sh.mass[b], was.ties * amount(value_of_key(was.tie)));
    }
    __syncthreads();
    uint64_t mine[kPer], sum = 0, total;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      mine[i] = MASS ? sh.mass[kPer * t + i] : sh.count[kPer * t + i];
      sum += mine[i];
    }
    const uint64_t end = block_scan(sum, sh.red, turn, &total) + before;
    total += before;
    if (before >= target && before > 0) return false;
    if (total < target) {
      if (MASS) return false;
      target = total;  // fewer than k: all of them
    }
    // the first bin at which the target is reached; one token at least
    const uint64_t aim = max(target, before + 1);
    if (end >= aim && end - sum < aim) {
      uint64_t at = end - sum;
      int b = 0;
#pragma unroll
      for (int i = 0; i < kPer; ++i)
        if (at < aim) {
          b = i;
          at += mine[i];
        }
      uint64_t in = mine[0];
#pragma unroll
      for (int i = 1; i < kPer; ++i) in = b == i ? mine[i] : in;
      sh.bin = kPer * t + b;
      sh.before = at - in;
      sh.amount = in;
    }
    __syncthreads();
    const int b = sh.bin;
    before = sh.before;
    const uint64_t in = sh.amount;
    const uint32_t n = sh.count[b];
    const uint32_t lower = hi - min(hi - lo, ((uint32_t)(b + 1) << shift) - 1), upper = hi - ((uint32_t)b << shift);
    if (shift == 0) {  // one value: its first few
      const uint64_t each = in / n, few = (aim - before + each - 1) / each;
      kept = Kept{upper << DROP, (uint32_t)min<uint64_t>(few, n)};
      if (DROP > 0 && !(kept.tie & 0x80000000u)) kept.tie |= (1u << DROP) - 1;  // (a negative number's bits are turned round)
      return true;
    }
    lo = lower;
    hi = upper;
    __syncthreads();
  }
}

template <typename T>
__global__ __launch_bounds__(kSampThreads) void sample_choose_kernel(SampleArgs a) {
  __shared__ ChooseShared sh;
  const int t = threadIdx.x;
  const int64_t r = blockIdx.x;
  Row<T> row(a, r);
  RowState &st = a.state[r];
  Settings s = settings_of(a, r);
  const uint32_t top = st.top;
  const int listed = (int)min(st.listed, kList + 1u);
  int turn = 0;
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
  if (s.greedy) {
    if (t == 0) {
      a.tokens[r] = (int)~(uint32_t)mass;
      if (a.logprob) a.logprob[r] = 0.f;
    }
    return;
  }
  // ---- the filters ----
  Kept kept{0, 0};  // (no finite logit has key 0)
  if (s.mode != kPlain) {
    // (a filter ends at a token: a list of none does not suffice)
    Tokens<T> tokens{row, sh, listed > 0 && listed <= kList ? listed : -1};
    if (s.k > 0) cut<false>(row, tokens, kept, -INFINITY, 0, (uint64_t)s.k, sh, turn);
    if (kept.ties > 0 && row.exponent(value_of_key(kept.tie)) < s.lm) kept.ties = 0;
    if (s.p < 1.f) {
      const auto reached = [&](uint64_t all) { return (uint64_t)ceil((double)s.p * (double)all); };
      for (;;) {
        uint64_t sum = 0, above = 0, all = mass;
        if (s.mode == kMass && tokens.listed >= 0) {
#pragma unroll
          for (int i = 0; i < kPer; ++i) sum += mine[i];
          block_scan(sum, sh.red, turn, &above);
        } else {
          tokens.each([&](float v, uint32_t key, int) {
            if (key > kept.tie && row.exponent(v) >= s.lm) sum += unit_weight(row.exponent(v), sh.table);
          });
          if (t == 0 && kept.ties > 0) sum += kept.ties * unit_weight(row.exponent(value_of_key(kept.tie)), sh.table);
          block_scan(sum, sh.red, turn, &all);
        }
        if (cut<true>(row, tokens, kept, s.lm, above, reached(all), sh, turn) || tokens.listed < 0) break;
        tokens.listed = -1;  // it ends elsewhere
        __syncthreads();
      }
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
  uint64_t ties_before = block_scan(ties, sh.red, turn, &unused) - ties, first_ties = ties_before;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const uint64_t n = mine[i] >> 54;
    mine[i] &= (1ull << 54) - 1;
    mine[i] += (ties_before >= kept.ties ? 0 : min(n, kept.ties - ties_before)) * each;
    ties_before += n;
    sum += mine[i];
  }
  const uint64_t start = block_scan(sum, sh.red, turn, &S) - sum;
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
  // ---- its token, by two a thread ----
  const int piece = sh.bin, first = piece * kPiece + 2 * t;
  const uint64_t goal = target - sh.before;
  int seen = sh.left;
  // the ties of the pieces before this one: `left` up to the first piece of its thread, the others looked at again
  if (kept.ties > 0 && piece % kPer != 0) {
    int n = 0;
    for (int i = piece / kPer * kPer * kPiece + t; i < piece * kPiece; i += kSampThreads)
      n += order_key(Elem<T>::load(row.x + i)) == kept.tie;
    block_scan((uint64_t)n, sh.red, turn, &unused);
    seen += (int)unused;
  }
  uint64_t m[2];
  int tied[2];
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const float v = first + e < row.vocab ? Elem<T>::load(row.x + first + e) : -INFINITY;
    const uint32_t key = order_key(v);
    const double ex = row.exponent(v);
    m[e] = v > -INFINITY && key > kept.tie && ex >= s.lm ? unit_weight(ex, sh.table) : 0;
    tied[e] = kept.ties > 0 && key == kept.tie;
  }
  const int rank = seen + (int)block_scan((uint64_t)(tied[0] + tied[1]), sh.red, turn, &unused) - tied[0] - tied[1];
  if (tied[0]) m[0] = rank < (int)kept.ties ? each : 0;
  if (tied[1]) m[1] = rank + tied[0] < (int)kept.ties ? each : 0;
  const uint64_t before = block_scan(m[0] + m[1], sh.red, turn, &unused) - m[0] - m[1];
  if (!(before <= goal && goal < before + m[0] + m[1])) return;
  const int token = first + (goal >= before + m[0]);
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
