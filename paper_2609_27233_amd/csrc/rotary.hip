// Rotary positions of rows of heads, and a layer's projected rows on their
// way into the paged cache (gfx950): rotary, kv_write_rotary.
//
// Every feature pair of a head is turned by position x frequency; the angles
// of a row are the same for all its heads.  Both calls read and write each
// row once and are bound by that traffic.  A workgroup takes a tile of rows
// and a range of heads: it forms the tile's cosines and sines in LDS (angle
// and reduction in double precision, then fp32); a thread keeps those of one
// row's 16-byte unit in registers and turns that unit of one head after
// another, several heads' loads in flight.  4096 bf16 rows of 64 heads of 128
// (134 MB) take 25.6 us, 5.2 TB/s, and a write of 39,328 rows of 32 + 8 + 8
// heads of 128 (967 MB) 199 us, 4.9 TB/s; a plain copy of 1 GiB reaches 5.1.
// Few rows are bound by latency (the slots, the angles, then the rows): 16
// rows 5 us.
//
// K rows go to token-major pages 16 bytes at a time.  V pages are dim-major,
// so V is transposed in registers: VEC rows (bf16 8, fp32 4) that fill an
// aligned group of a page's slots become 16-byte stores.  Tiles are cut where
// a 16-slot segment of a page begins, so a prompt's rows are stored whole
// wherever its sequence starts in the batch, and two neighbouring lanes fill
// 32 bytes of a page's row; single rows (a decode step) are stored an element
// at a time, which the layout of the pages asks for (39,328 rows of slots in
// no order: 539 us).
#include <algorithm>
#include <cmath>

#include "cache_meta.hpp"
#include "vec16.hpp"

namespace sm {

constexpr int kRotThreads = 256;
constexpr int kTileRows = 16;
constexpr int kMostRows = 2 * kTileRows - 1;  // of a tile cut by slots
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
  FastDiv per_head;         // by the units of a head
};

// Cosine and sine of the tile's rows, [row][pair]: the angle in turns is
// reduced to [-1/2, 1/2] in double precision and only then rounded to fp32, off
// by 1e-7 rad at most, as much as cosine and sine themselves are (a sine in
// double takes several times the instructions).
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

__device__ __forceinline__ float2 turned(float a, float b, float2 cs) {
  return make_float2(a * cs.x - b * cs.y, a * cs.y + b * cs.x);
}

// V features as they lie in memory: 16, 8, 4 or 2 bytes.
template <int BYTES> struct Raw;
template <> struct Raw<16> { typedef u32x4_t type; };
template <> struct Raw<8> { typedef uint32_t type __attribute__((ext_vector_type(2))); };
template <> struct Raw<4> { typedef uint32_t type; };
template <> struct Raw<2> { typedef uint16_t type; };
template <typename T, int V>
struct Piece {
  typedef typename Raw<V * sizeof(T)>::type raw;
  static __device__ __forceinline__ void open(raw r, float (&f)[V]) {
    T t[V];
    __builtin_memcpy(t, &r, sizeof r);
#pragma unroll
    for (int e = 0; e < V; ++e) f[e] = Elem<T>::load(t + e);
  }
  static __device__ __forceinline__ raw close(const float (&f)[V]) {
    T t[V];
#pragma unroll
    for (int e = 0; e < V; ++e) t[e] = Elem<T>::to_store(f[e]);
    raw r;
    __builtin_memcpy(&r, t, sizeof r);
    return r;
  }
};
template <> struct Piece<uint16_t, 8> {
  typedef u32x4_t raw;
  static __device__ __forceinline__ void open(raw r, float (&f)[8]) { Vec16<uint16_t>::open(r, f); }
  static __device__ __forceinline__ raw close(const float (&f)[8]) { return Vec16<uint16_t>::close(f); }
};

// Input that would fill the 256 MB of last-level cache with what is made of it
// is read past it (STREAM), as nothing reads it again.  Past it and plainly,
// beside what writes the rows and what reads the result, us:
//   about MiB         48          56          64          72          128         240
//   rotary, bf16, 32  17.4, 15.9  19.7, 20.9  21.2, 25.7  23.1, 26.4  41.9, 55.0  93, 104
//   write, bf16, 32+8 18.5, 20.1  25.0, 24.6  27.5, 28.3  25.1, 30.0  55.2, 64.0  105, 111
//   write, bf16, 28+4 21.9, 18.2  27.5, 23.8  27.3, 27.6  28.2, 33.4  52.5, 62.4  99, 108
//   write, fp32, 4+4  22.7, 20.7  25.7, 20.6  29.4, 26.0  31.6, 28.4  56.5, 59.7  96, 96
// (heads of 128, the last of 64: such rows, 3 KB, gain nothing below 80 MiB;
// fp32 writes of heads of 128 gain 8% and more from 56 on).  What the cache could not
// hold by itself is read plainly: 268 MB of fp32 rows 117 us past it, 111 so.
constexpr int64_t kStreamFrom = 64 << 20, kStreamTo = 256 << 20;

template <bool STREAM, typename R>
__device__ __forceinline__ R load_as(const void *p) {
  if constexpr (STREAM) return __builtin_nontemporal_load((const R *)p);
  else return *(const R *)p;
}

// A thread's unit: V features of a row's head that are turned with V more
// (half layout: the second half's; single features: a pair's other one), or
// among themselves, or behind the turned part, where they are copied.
template <typename T, bool HALF, int V>
struct Unit {
  static constexpr bool TWO = HALF || V == 1;
  static constexpr int NP = TWO ? V : V / 2;  // pairs
  int at, far;  // features; far 0: no second piece
  bool turning;
  float2 cs[NP];

  __device__ __forceinline__ void set(int j, int R, const float2 *row_cs) {
    const int units = TWO ? R / (2 * V) : R / V;
    turning = j < units;
    at = !turning ? R + (j - units) * V : HALF || !TWO ? j * V : 2 * j;
    far = !turning || !TWO ? 0 : HALF ? R / 2 : 1;
    if (turning)
#pragma unroll
      for (int e = 0; e < NP; ++e) cs[e] = row_cs[j * NP + e];
  }
  // Heads h, h + step, ... below h1: in(h), out(h) give a head's first
  // feature.  The loads are unconditional (the last head's again).
  template <bool STREAM, class In, class Out>
  __device__ __forceinline__ void run(int h, int h1, int step, In in, Out out) const {
    typedef Piece<T, V> P;
    typedef typename P::raw raw;
    constexpr int U = 4;
    for (; h < h1; h += U * step) {
      raw a[U], b[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const T *p = in(min(h + u * step, h1 - 1)) + at;
        a[u] = load_as<STREAM, raw>(p);
        if constexpr (TWO) b[u] = load_as<STREAM, raw>(p + far);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (h + u * step >= h1) break;
        T *p = out(h + u * step) + at;
        if (!turning) {
          *(raw *)p = a[u];
          continue;
        }
        float f[V], g[V];
        P::open(a[u], f);
        if constexpr (TWO) {
          P::open(b[u], g);
#pragma unroll
          for (int e = 0; e < V; ++e) {
            const float2 t = turned(f[e], g[e], cs[e]);
            f[e] = t.x;
            g[e] = t.y;
          }
          *(raw *)(p + far) = P::close(g);
        } else {
#pragma unroll
          for (int e = 0; e < V; e += 2) {
            const float2 t = turned(f[e], f[e + 1], cs[e / 2]);
            f[e] = t.x;
            f[e + 1] = t.y;
          }
        }
        *(raw *)p = P::close(f);
      }
    }
  }
};

// The units of `nr` rows over the workgroup: f(row, unit of the head, first
// head, step over the heads).  Lanes that are neighbours hold the units of a
// head, then BY_ROW those of the row's other heads (rows are read and written
// in long pieces), else those of the next rows (as pages hold them); with
// fewer units than threads, more threads share the heads.
template <bool BY_ROW, class F>
__device__ __forceinline__ void each_unit(int nr, const FastDiv &per_head, int heads, F f) {
  const int units = nr * (int)per_head.d;
  int share_log2 = 0;
  while (((BY_ROW && (int)per_head.d << share_log2 < 64) || units << share_log2 < kRotThreads) && 1 << share_log2 < heads)
    ++share_log2;
  for (int u = threadIdx.x; u < units << share_log2; u += kRotThreads) {
    if constexpr (BY_ROW) {
      const int rp = fdiv(u, per_head), part = rp & ((1 << share_log2) - 1);
      f(rp >> share_log2, u - rp * (int)per_head.d, part, 1 << share_log2);
    } else {
      const int part = share_log2 == 0 ? 0 : u / units, at = u - part * units, r = fdiv(at, per_head);
      f(r, at - r * (int)per_head.d, part, 1 << share_log2);
    }
  }
}

template <typename T, bool HALF, int V, bool STREAM>
__global__ __launch_bounds__(kRotThreads) void rotary_kernel(RopeArgs a, Rows x, int D, int heads_per) {
  extern __shared__ float2 cs[];  // [rows of a tile][R / 2]
  const int64_t r0 = (int64_t)blockIdx.x * kTileRows;
  const int nr = (int)min((int64_t)kTileRows, a.rows - r0);
  const int h0 = blockIdx.y * heads_per, h1 = min(h0 + heads_per, x.heads);
  fill_angles(a, (int)r0, nr, cs);
  __syncthreads();
  each_unit<true>(nr, a.per_head, h1 - h0, [&](int r, int j, int part, int share) {
    Unit<T, HALF, V> unit;
    unit.set(j, a.R, cs + r * (a.R / 2));
    const T *in = (const T *)x.in + (r0 + r) * x.in_stride;
    T *out = (T *)x.out + (r0 + r) * x.out_stride;
    unit.template run<STREAM>(h0 + part, h1, share, [&](int h) { return in + h * D; }, [&](int h) { return out + h * D; });
  });
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

// out[i] = element i of in[0 .. VEC-1]
__device__ __forceinline__ void transpose16(const u32x4_t (&in)[8], u32x4_t (&out)[8]) {  // bf16
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const uint32_t x = in[2 * w][i >> 1], y = in[2 * w + 1][i >> 1];
      out[i][w] = (i & 1) ? ((x >> 16) | (y & 0xffff0000u)) : ((x & 0xffffu) | (y << 16));
    }
}
__device__ __forceinline__ void transpose16(const u32x4_t (&in)[4], u32x4_t (&out)[4]) {  // fp32
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) out[i][j] = in[j][i];
}

// Head 0 of the page that holds slot s, and the slot in it.
template <typename T>
__device__ __forceinline__ T *page_of(T *pool, int s, const WriteArgs &w, int *in_page) {
  *in_page = s & ((1 << w.bs_log2) - 1);
  return pool + (((int64_t)(s >> w.bs_log2) * w.k.heads) << (w.bs_log2 + w.dh_log2));
}

template <typename T, bool HALF, bool STREAM>
__global__ __launch_bounds__(kRotThreads) void kv_write_kernel(RopeArgs a, WriteArgs w, int heads_per) {
  constexpr int VEC = 16 / sizeof(T);
  extern __shared__ float2 cs[];
  __shared__ int slot[kMostRows + 1], group[kMostRows + 1];
  const int t = threadIdx.x, lane = t & 63, D = 1 << w.dh_log2, bs = 1 << w.bs_log2;
  // The tile: from the first row at or past base that begins a 16-slot
  // segment, a run of its own or padding, to the next tile's first.  Each
  // wave looks at the slots of rows base - 1 .. base + 62.
  const int64_t base = (int64_t)blockIdx.x * kTileRows;
  const int64_t mine = base + lane - 1;
  int s = mine >= 0 && mine < a.rows ? w.slots[mine] : -1;
  const bool bad = s < -1 || s >= w.num_slots;
  if (bad) s = -1;
  const int before = __shfl_up(s, 1, kWave);
  const bool end = mine >= a.rows;
  const uint64_t first = __ballot(s < 0 || before != s - 1 || s % kTileRows == 0 || mine == 0 || end) >> 1;
  const uint64_t fill = __ballot(s < 0 || before != s - 1 || s % VEC == 0 || mine == 0 || end) >> 1;  // group starts
  const int b0 = __builtin_ctzll(first), b1 = kTileRows + __builtin_ctzll(first >> kTileRows);
  const int r0 = (int)(base + b0), nr = (int)min((int64_t)a.rows, base + b1) - r0;
  if (nr <= 0) return;
  const int h0 = blockIdx.y * heads_per, h1 = min(h0 + heads_per, w.q.heads + 2 * w.k.heads);
  const int me = lane - 1 - b0;  // this lane's row of the tile
  // groups of rows that fill consecutive slots of VEC aligned ones
  const uint64_t mask = fill >> b0 & ((1ull << nr) - 1);
  const int groups = __popcll(mask);
  if (t < 64 && me >= 0 && me < nr) {
    slot[me] = s;
    if (bad && h0 == 0) set_err(w.err, SM_ERR_EINVAL);
    if (mask >> me & 1) group[__popcll(mask & ((1ull << me) - 1))] = me;
  }
  if (t == 0) group[groups] = nr;
  if (h0 < w.q.heads + w.k.heads) fill_angles(a, r0, nr, cs);
  __syncthreads();
  // V: unit = (head, VEC dims, group), the groups of a segment side by side
  const int g0 = max(h0 - w.q.heads - w.k.heads, 0), g1 = h1 - w.q.heads - w.k.heads;
  if (g1 > g0) {
    const int dgs = D / VEC, units = (g1 - g0) * dgs * groups;
    const float inv = 1.f / groups;
    for (int u = t; u < units; u += kRotThreads) {
      const int hd = (int)((u + 0.5f) * inv), g = u - hd * groups;  // (exact below 2^21)
      const int h = g0 + hd / dgs, d0 = hd % dgs * VEC;
      const int f = group[g], n = group[g + 1] - f, sl = slot[f];
      const T *in = (const T *)w.v.in + (int64_t)(r0 + f) * w.v.in_stride + h * D + d0;
      u32x4_t v[VEC], vt[VEC];
#pragma unroll
      for (int i = 0; i < VEC; ++i) v[i] = load_as<STREAM, u32x4_t>(in + min(i, n - 1) * w.v.in_stride);
      if (sl < 0) continue;
      int at;
      T *out = page_of((T *)w.v_pool, sl, w, &at) + (((int64_t)h * D + d0) << w.bs_log2) + at;
      transpose16(v, vt);
      if (n == VEC) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) *(u32x4_t *)(out + (int64_t)i * bs) = vt[i];
      } else {
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
          const T *e = (const T *)&vt[i];
#pragma unroll
          for (int j = 0; j < VEC; ++j)
            if (j < n) out[(int64_t)i * bs + j] = e[j];
        }
      }
    }
  }
  const int hq1 = min(h1, w.q.heads), k0 = max(h0 - w.q.heads, 0), k1 = min(h1 - w.q.heads, w.k.heads);
  if (h0 >= w.q.heads + w.k.heads) return;
  if (hq1 > h0)
    each_unit<false>(nr, a.per_head, hq1 - h0, [&](int r, int j, int part, int share) {
      Unit<T, HALF, VEC> unit;
      unit.set(j, a.R, cs + r * (a.R / 2));
      const T *q = (const T *)w.q.in + (r0 + r) * w.q.in_stride;
      T *out = (T *)w.q.out + (r0 + r) * w.q.out_stride;
      unit.template run<STREAM>(h0 + part, hq1, share, [&](int h) { return q + h * D; }, [&](int h) { return out + h * D; });
    });
  if (k1 > k0)
    each_unit<false>(nr, a.per_head, k1 - k0, [&](int r, int j, int part, int share) {
      const int sl = slot[r];
      if (sl < 0) return;
      Unit<T, HALF, VEC> unit;
      unit.set(j, a.R, cs + r * (a.R / 2));
      const T *k = (const T *)w.k.in + (r0 + r) * w.k.in_stride;
      int at;
      T *page = page_of((T *)w.k_pool, sl, w, &at) + at * D;
      unit.template run<STREAM>(k0 + part, k1, share, [&](int h) { return k + h * D; },
               [&](int h) { return page + ((int64_t)h << (w.bs_log2 + w.dh_log2)); });
    });
}

// Rows or strides that 16 bytes do not divide: a feature at a time.
template <typename T, bool HALF>
__global__ __launch_bounds__(kRotThreads) void kv_write_any_kernel(RopeArgs a, WriteArgs w, int heads_per) {
  extern __shared__ float2 cs[];
  __shared__ int slot[kTileRows];
  const int64_t r0 = (int64_t)blockIdx.x * kTileRows;
  const int nr = (int)min((int64_t)kTileRows, a.rows - r0), t = threadIdx.x, D = 1 << w.dh_log2;
  const int h0 = blockIdx.y * heads_per, h1 = min(h0 + heads_per, w.q.heads + 2 * w.k.heads);
  if (t < nr) {
    const int s = w.slots[r0 + t];
    const bool bad = s < -1 || s >= w.num_slots;
    if (bad && h0 == 0) set_err(w.err, SM_ERR_EINVAL);
    slot[t] = bad ? -1 : s;
  }
  if (h0 < w.q.heads + w.k.heads) fill_angles(a, (int)r0, nr, cs);
  __syncthreads();
  const int hq1 = min(h1, w.q.heads), k0 = max(h0 - w.q.heads, 0), k1 = min(h1 - w.q.heads, w.k.heads);
  const int g0 = max(h0 - w.q.heads - w.k.heads, 0), g1 = h1 - w.q.heads - w.k.heads;
  int at;
  for (int r = 0; r < nr && g1 > g0; ++r) {
    if (slot[r] < 0) continue;
    const T *in = (const T *)w.v.in + (r0 + r) * w.v.in_stride;
    T *out = page_of((T *)w.v_pool, slot[r], w, &at) + at;
    for (int hd = g0 * D + t; hd < g1 * D; hd += kRotThreads) out[(int64_t)hd << w.bs_log2] = in[hd];
  }
  if (hq1 > h0)
    each_unit<true>(nr, a.per_head, hq1 - h0, [&](int r, int j, int part, int share) {
      Unit<T, HALF, 1> unit;
      unit.set(j, a.R, cs + r * (a.R / 2));
      const T *q = (const T *)w.q.in + (r0 + r) * w.q.in_stride;
      T *out = (T *)w.q.out + (r0 + r) * w.q.out_stride;
      unit.template run<false>(h0 + part, hq1, share, [&](int h) { return q + h * D; }, [&](int h) { return out + h * D; });
    });
  if (k1 > k0)
    each_unit<true>(nr, a.per_head, k1 - k0, [&](int r, int j, int part, int share) {
      if (slot[r] < 0) return;
      Unit<T, HALF, 1> unit;
      unit.set(j, a.R, cs + r * (a.R / 2));
      const T *k = (const T *)w.k.in + (r0 + r) * w.k.in_stride;
      T *page = page_of((T *)w.k_pool, slot[r], w, &at) + at * D;
      unit.template run<false>(k0 + part, k1, share, [&](int h) { return k + h * D; },
               [&](int h) { return page + ((int64_t)h << (w.bs_log2 + w.dh_log2)); });
    });
}

}  // namespace sm

using namespace sm;

// Rows of a launch: its threads are counted in 32 bits, 256 for 16 rows.
constexpr int64_t kLaunchRows = 1 << 24;

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

// Frequencies in turns per position, on the host in double precision:
// theta^(-j / P) as a power for every eighth pair times one for the pairs
// between (64 exponentials took 0.8 us of a small call's 7, 16 take 0.2; the
// product's rounding is a fraction of the exponentials' own).
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
  double step[8], base = 1;
  for (int i = 0; i < 8 && i < P; ++i) step[i] = std::exp(-ln_theta * i / P);
  for (int j = 0; j < P; ++j) {
    if (j % 8 == 0) base = std::exp(-ln_theta * j / P);
    double w = base * step[j % 8] / two_pi;  // turns per position
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

// Rows made in place lie where they are read.
static bool placed(const void *in, int64_t in_stride, const void *out, int64_t out_stride, int rows) {
  return in != out || in_stride == out_stride || rows == 1;
}

static bool aligned(const void *p, int64_t stride, int64_t bytes, int64_t es) {
  return (uintptr_t)p % bytes == 0 && stride * es % bytes == 0;
}

// Whether pieces of v features divide a head's turned part (half layout: each
// half of it) and the rest.
static bool divides(const sm_rope_params *p, int D, int v) {
  return (p->layout == SM_ROPE_HALF ? p->rot_dim / 2 : p->rot_dim) % v == 0 && (D - p->rot_dim) % v == 0;
}

// v: features of a piece
static RopeArgs rope_args(const sm_rope_params *p, int D, int v, int transpose) {
  RopeArgs a;
  set_turns(p, &a);
  a.R = p->rot_dim;
  a.sign = transpose ? -1 : 1;
  a.scale = p->attn_scale;
  a.per_head = make_fastdiv(p->rot_dim / (p->layout == SM_ROPE_HALF || v == 1 ? 2 * v : v) + (D - p->rot_dim) / v);
  return a;
}

// Heads per workgroup: enough workgroups for the device where there are few rows.
static int heads_per_wg(int heads, int64_t tiles) {
  int per = heads;
  while (per > 1 && tiles * ((heads + per - 1) / per) < 512) per = (per + 1) / 2;
  return per;
}

// Whether rows are read past the last-level cache.  Pieces that leave part of a
// 128-byte line for another load would have it fetched twice (halves of 64
// bytes: 108 us, not 87, for 65,536 rows of 24 heads of 64).
static bool streams(const RopeArgs &a, int D, int es, bool half, int heads) {
  const int64_t bytes = (int64_t)a.rows * heads * D * es;
  return bytes >= kStreamFrom && bytes < kStreamTo && D * es % 128 == 0 && (!half || a.R / 2 * es % 128 == 0);
}

template <typename T, int V>
static void launch_rotary(const RopeArgs &a, const Rows &x, int D, bool half, hipStream_t stream) {
  const int64_t tiles = ((int64_t)a.rows + kTileRows - 1) / kTileRows;
  const int per = heads_per_wg(x.heads, tiles);
  const dim3 grid((unsigned)tiles, (x.heads + per - 1) / per);
  const size_t lds = kTileRows * (a.R / 2) * sizeof(float2);
  auto kernel = half ? rotary_kernel<T, true, V, false> : rotary_kernel<T, false, V, false>;
  if constexpr (V * sizeof(T) == 16)
    if (streams(a, D, sizeof(T), half, x.heads)) kernel = half ? rotary_kernel<T, true, V, true> : rotary_kernel<T, false, V, true>;
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
  if (!x || !pos || !out || !placed(x, x_stride, out, out_stride, rows)) return SM_EINVAL;
  const int es = dt == SM_BF16 ? 2 : 4;
  int v = 16 / es;  // features of a piece: the most that divide the head and are aligned in every row
  while (v > 1 && !(divides(p, head_dim, v) && aligned(x, x_stride, v * es, es) && aligned(out, out_stride, v * es, es)))
    v /= 2;
  RopeArgs a = rope_args(p, head_dim, v, transpose);
  const bool half = p->layout == SM_ROPE_HALF;
  for (int64_t first = 0; first < rows; first += kLaunchRows) {
    a.pos = pos + first;
    a.rows = (int)std::min(rows - first, kLaunchRows);
    const Rows r{row_at(x, first, x_stride, es), row_at(out, first, out_stride, es), x_stride, out_stride, heads};
    if (dt == SM_BF16) {
      if (v == 8) launch_rotary<uint16_t, 8>(a, r, head_dim, half, stream);
      else if (v == 4) launch_rotary<uint16_t, 4>(a, r, head_dim, half, stream);
      else if (v == 2) launch_rotary<uint16_t, 2>(a, r, head_dim, half, stream);
      else launch_rotary<uint16_t, 1>(a, r, head_dim, half, stream);
    } else {
      if (v == 4) launch_rotary<float, 4>(a, r, head_dim, half, stream);
      else if (v == 2) launch_rotary<float, 2>(a, r, head_dim, half, stream);
      else launch_rotary<float, 1>(a, r, head_dim, half, stream);
    }
    if (hipGetLastError() != hipSuccess) return SM_EHIP;
  }
  return SM_OK;
}

template <typename T>
static void launch_write(const RopeArgs &a, const WriteArgs &w, bool half, bool wide, hipStream_t stream) {
  const int64_t tiles = ((int64_t)a.rows + kTileRows - 1) / kTileRows;
  const int heads = w.q.heads + 2 * w.k.heads, per = heads_per_wg(heads, tiles);
  const dim3 grid((unsigned)tiles, (heads + per - 1) / per);
  const size_t lds = kMostRows * (a.R / 2) * sizeof(float2);
  const bool past = streams(a, 1 << w.dh_log2, sizeof(T), half, heads);
  const auto kernel = !wide  ? (half ? kv_write_any_kernel<T, true> : kv_write_any_kernel<T, false>)
                      : past ? (half ? kv_write_kernel<T, true, true> : kv_write_kernel<T, false, true>)
                             : (half ? kv_write_kernel<T, true, false> : kv_write_kernel<T, false, false>);
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
  if (!pos || !slots || !k || !v) return SM_EINVAL;
  if (num_q_heads > 0 && (!q || !q_out || !placed(q, q_stride, q_out, q_out_stride, rows))) return SM_EINVAL;
  const int es = c->dtype == SM_BF16 ? 2 : 4;
  const bool wide = divides(p, D, 16 / es) && aligned(k, k_stride, 16, es) && aligned(v, v_stride, 16, es) &&
                    aligned(c->k_pool, 0, 16, es) && aligned(c->v_pool, 0, 16, es) &&
                    (num_q_heads == 0 || (aligned(q, q_stride, 16, es) && aligned(q_out, q_out_stride, 16, es)));
  RopeArgs a = rope_args(p, D, wide ? 16 / es : 1, 0);
  const int hkv = c->num_kv_heads;
  for (int64_t r = 0; r < rows; r += kLaunchRows) {
    a.pos = pos + r;
    a.rows = (int)std::min(rows - r, kLaunchRows);
    const WriteArgs w{Rows{row_at(q, r, q_stride, es), row_at(q_out, r, q_out_stride, es), q_stride, q_out_stride, num_q_heads},
                      Rows{row_at(k, r, k_stride, es), nullptr, k_stride, 0, hkv},
                      Rows{row_at(v, r, v_stride, es), nullptr, v_stride, 0, hkv},
                      slots + r, c->k_pool, c->v_pool, c->err, ca.bs_log2, ca.dh_log2, c->num_blocks * c->block_size};
    if (c->dtype == SM_BF16) launch_write<uint16_t>(a, w, p->layout == SM_ROPE_HALF, wide, stream);
    else launch_write<float>(a, w, p->layout == SM_ROPE_HALF, wide, stream);
    if (hipGetLastError() != hipSuccess) return SM_EHIP;
  }
  return SM_OK;
}
