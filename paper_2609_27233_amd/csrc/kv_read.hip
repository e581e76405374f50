// Cached entries read back as rows of K and V (gfx950): kv_read.
//
// Request i's rows are entries start[i], start[i] + 1, ... of its sequence, in
// the type that a row has when it is written: bf16 out of e4m3 pages (exact:
// every e4m3 value times its power of two is a bf16 number), the pages' own
// type otherwise.  A workgroup takes a tile of rows and a range of heads.  It
// finds each row's slot (request by a search in LDS, sequence, page) and cuts
// the tiles where a 16-slot segment of a page begins, as the write does: V
// pages are dim-major, and a thread takes one 16-byte piece of 8 (fp32: 4)
// features' slots, turns them round in registers and stores whole 16-byte
// pieces of rows.
//
// HBM bounds it: 39,328 entries of 8 heads x 128 out of e4m3 pages 57 us over
// several caches in turn (4.3 TB/s of values, exponents and rows), 41 over one
// whose pages stay in the last-level cache; out of bf16 pages 67.  A step's few
// rows take a launch, 5 us.
#include <algorithm>

#include "cache_meta.hpp"
#include "e4m3.hpp"
#include "vec16.hpp"

namespace sm {

constexpr int kReadThreads = 256;
constexpr int kReadTile = 16;
constexpr int kReadMost = 2 * kReadTile - 1;  // rows of a tile cut by slots
constexpr int kSlotNone = -2, kSlotZero = -1;  // a row that is not written; one that is zeroed

struct ReadArgs {
  CacheArgs c;
  const uint8_t *k_exp, *v_exp;
  const int32_t *seq_ids, *start, *row_offsets;
  int n, total_rows;
  int64_t first;  // row of the launch's first tile
  void *K, *V;
  int64_t k_stride, v_stride;
};

struct E4m3 { uint8_t byte; };

// What a page's type T is read as: rows of Out, VEC slots (and 16 / sizeof(T) features) to 16 bytes.
template <typename T> struct Paged { typedef T Out; static constexpr int SLOTS = 16 / sizeof(T), DIMS = SLOTS; };
template <> struct Paged<E4m3> { typedef uint16_t Out; static constexpr int SLOTS = 16, DIMS = 8; };

template <typename Out, bool WIDE>
__device__ __forceinline__ void store_piece(Out *to, u32x4_t v) {
  if constexpr (WIDE) {
    *(u32x4_t *)to = v;
  } else {
    Out e[16 / sizeof(Out)];
    __builtin_memcpy(e, &v, 16);
#pragma unroll
    for (int i = 0; i < (int)(16 / sizeof(Out)); ++i) to[i] = e[i];
  }
}

// in[d]: 16 bytes of feature d's slots -> out[i]: slot i's DIMS features in 16 bytes
template <typename T>
__device__ __forceinline__ void rows_of(const u32x4_t (&in)[Paged<T>::DIMS], u32x4_t bytes, u32x4_t (&out)[Paged<T>::SLOTS]) {
  if constexpr (sizeof(T) == 1) {
#pragma unroll
    for (int w = 0; w < 4; ++w) {  // four slots
      uint32_t lo[4], hi[4], tlo[4], thi[4];
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        lo[d] = in[d][w];
        hi[d] = in[4 + d][w];
      }
      transpose4(lo, tlo);
      transpose4(hi, thi);
#pragma unroll
      for (int i = 0; i < 4; ++i) out[4 * w + i] = e4m3_to_bf16(tlo[i], thi[i], exp_scale((bytes[w] >> (8 * i)) & 0xff));
    }
  } else if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const uint32_t x = in[2 * w][i >> 1], y = in[2 * w + 1][i >> 1];
        out[i][w] = (i & 1) ? ((x >> 16) | (y & 0xffff0000u)) : ((x & 0xffffu) | (y << 16));
      }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int d = 0; d < 4; ++d) out[i][d] = in[d][i];
  }
}

template <typename T, bool WIDE>
__global__ __launch_bounds__(kReadThreads) void kv_read_kernel(ReadArgs a, int heads_per) {
  typedef typename Paged<T>::Out Out;
  constexpr int SLOTS = Paged<T>::SLOTS, DIMS = Paged<T>::DIMS;
  __shared__ int offs[SM_MAX_REQUESTS + 1];
  __shared__ int slot[kReadMost + 1], group[kReadMost + 1];
  const int t = threadIdx.x, lane = t & 63, D = a.c.DH, bs_log2 = a.c.bs_log2, bs = 1 << bs_log2, H = a.c.Hkv;
  // ---- the offsets, whole, in order and within the rows ----
  int wrong = 0;
  for (int i = t; i <= a.n; i += kReadThreads) {
    const int o = a.row_offsets[i], next = i < a.n ? a.row_offsets[i + 1] : a.total_rows;
    wrong |= o < 0 || next < o || (i == 0 && o != 0);
    offs[i] = o;
  }
  if (__syncthreads_or(wrong)) {
    if (t == 0 && blockIdx.x == 0 && blockIdx.y == 0 && a.first == 0) set_err(a.c.err, SM_ERR_EINVAL);
    return;
  }
  // ---- slots of rows base - 1 .. base + 62, a row a lane, in every wave ----
  const int64_t base = a.first + (int64_t)blockIdx.x * kReadTile, mine = base + lane - 1;
  int s = kSlotNone, status = 0;
  if (mine >= 0 && mine < offs[a.n]) {
    int i = 0, end = a.n;  // the last request that begins at or before the row (those of no rows end there too)
    while (end - i > 1) {
      const int mid = (i + end) >> 1;
      if (offs[mid] <= mine) i = mid;
      else end = mid;
    }
    s = kSlotZero;
    const int id = a.seq_ids[i];
    if (id < 0 || id >= a.c.max_seqs) {
      status = SM_ERR_EINVAL;
    } else {
      const int64_t p = (a.start ? a.start[i] : 0) + (mine - offs[i]);
      const int L = a.c.lengths[id];
      if (p < 0 || p >= L || L > a.c.max_blocks << bs_log2) {
        status = SM_ERR_ERANGE;
      } else {
        const int blk = a.c.block_table[(int64_t)id * a.c.max_blocks + (p >> bs_log2)];
        if (blk < 0 || blk >= a.c.num_blocks) status = SM_ERR_EINVAL;
        else s = (blk << bs_log2) + (int)(p & (bs - 1));
      }
    }
  }
  const int before = __shfl_up(s, 1, kWave);
  const bool cut = s < 0 || before != s - 1 || mine == 0;
  const uint64_t first = __ballot(cut || s % kReadTile == 0) >> 1, fill = __ballot(cut || s % SLOTS == 0) >> 1;
  const int b0 = __builtin_ctzll(first), b1 = kReadTile + __builtin_ctzll(first >> kReadTile);
  const int64_t r0 = base + b0;
  const int nr = (int)(min((int64_t)a.total_rows, base + b1) - r0);
  if (nr <= 0) return;
  const int h0 = blockIdx.y * heads_per, h1 = min(h0 + heads_per, 2 * H);
  const int me = lane - 1 - b0;
  const uint64_t mask = fill >> b0 & ((1ull << nr) - 1);
  const int groups = __popcll(mask);
  if (t < 64 && me >= 0 && me < nr) {
    slot[me] = s;
    if (status && h0 == 0) set_err(a.c.err, status);
    if (mask >> me & 1) group[__popcll(mask & ((1ull << me) - 1))] = me;
  }
  if (t == 0) group[groups] = nr;
  __syncthreads();
  const u32x4_t zero = {0u, 0u, 0u, 0u};
  // ---- K: a lane 16 bytes of a page's row ----
  constexpr int PER = 16 / sizeof(T), OUTS = PER * (int)sizeof(Out) / 16;  // features; 16-byte pieces they become
  const int k1 = min(h1, H);
  if (a.K && k1 > h0) {
    const int lanes = D / PER, units = nr * (k1 - h0) * lanes;
    const float inv = 1.f / nr;
    for (int u = t; u < units; u += kReadThreads) {
      const int c = u & (lanes - 1), hr = u / lanes;
      const int hh = (int)((hr + 0.5f) * inv), r = hr - hh * nr, h = h0 + hh, sl = slot[r];  // (exact below 2^21)
      if (sl == kSlotNone) continue;
      Out *to = (Out *)a.K + (r0 + r) * a.k_stride + h * D + c * PER;
      u32x4_t v = zero;
      float scale = 1.f;
      if (sl >= 0) {
        const int64_t row = (((int64_t)(sl >> bs_log2) * H + h) << bs_log2) + (sl & (bs - 1));
        v = *(const u32x4_t *)((const T *)a.c.k_pool + row * D + c * PER);
        if constexpr (sizeof(T) == 1) scale = exp_scale(a.k_exp[row]);
      }
      if constexpr (OUTS == 2) {
        store_piece<Out, WIDE>(to, e4m3_to_bf16(v[0], v[1], scale));
        store_piece<Out, WIDE>(to + 8, e4m3_to_bf16(v[2], v[3], scale));
      } else {
        store_piece<Out, WIDE>(to, v);
      }
    }
  }
  // ---- V: a lane DIMS features of a group of slots ----
  const int g0 = max(h0 - H, 0), g1 = h1 - H;
  if (a.V && g1 > g0) {
    const int lanes = D / DIMS, units = (g1 - g0) * groups * lanes;
    const float inv = 1.f / groups;
    for (int u = t; u < units; u += kReadThreads) {
      const int c = u & (lanes - 1), hg = u / lanes;
      const int hh = (int)((hg + 0.5f) * inv), g = hg - hh * groups, h = g0 + hh;
      const int f = group[g], n = group[g + 1] - f, sl = slot[f];
      if (sl == kSlotNone) continue;
      Out *to = (Out *)a.V + (r0 + f) * a.v_stride + h * D + c * DIMS;
      if (sl < 0) {
        store_piece<Out, WIDE>(to, zero);
        continue;
      }
      const int64_t head = (int64_t)(sl >> bs_log2) * H + h;
      const int at = sl & (bs - 1) & ~(SLOTS - 1), skip = sl & (SLOTS - 1);
      const T *in = (const T *)a.c.v_pool + ((head * D + c * DIMS) << bs_log2) + at;
      u32x4_t v[DIMS], out[SLOTS], bytes = zero;
#pragma unroll
      for (int d = 0; d < DIMS; ++d) v[d] = *(const u32x4_t *)(in + ((int64_t)d << bs_log2));
      if constexpr (sizeof(T) == 1) bytes = *(const u32x4_t *)(a.v_exp + (head << bs_log2) + at);
      rows_of<T>(v, bytes, out);
#pragma unroll
      for (int i = 0; i < SLOTS; ++i)
        if (i >= skip && i < skip + n) store_piece<Out, WIDE>(to + (i - skip) * a.v_stride, out[i]);
    }
  }
}

}  // namespace sm

using namespace sm;

template <typename T>
static void launch_read(const ReadArgs &a, bool wide, int tiles, hipStream_t stream) {
  const int heads = 2 * a.c.Hkv;
  int per = heads;  // enough workgroups for the device where there are few rows
  while (per > 1 && (int64_t)tiles * ((heads + per - 1) / per) < 512) per = (per + 1) / 2;
  const dim3 grid(tiles, (heads + per - 1) / per);
  if (wide) hipLaunchKernelGGL((kv_read_kernel<T, true>), grid, dim3(kReadThreads), 0, stream, a, per);
  else hipLaunchKernelGGL((kv_read_kernel<T, false>), grid, dim3(kReadThreads), 0, stream, a, per);
}

SM_API sm_status sm_kv_read(const sm_paged_cache *c, const int32_t *seq_ids, const int32_t *start, const int32_t *row_offsets,
                            int n, int total_rows, void *K, int64_t k_stride, void *V, int64_t v_stride, hipStream_t stream) {
  ReadArgs a;
  if (!cache_ok(c, a.c, true) || n < 0 || n > SM_MAX_REQUESTS || total_rows < 0 || c->num_kv_heads > 1024) return SM_EINVAL;
  if ((int64_t)c->num_blocks * c->block_size > INT32_MAX) return SM_EINVAL;
  const int64_t width = (int64_t)c->num_kv_heads * c->head_dim;
  if ((K && k_stride < width) || (V && v_stride < width)) return SM_EINVAL;
  if ((uintptr_t)c->k_pool % 16 || (uintptr_t)c->v_pool % 16) return SM_EINVAL;
  if (n == 0 || total_rows == 0) return SM_OK;
  if (!seq_ids || !row_offsets || (!K && !V)) return SM_EINVAL;
  const int hkv = c->num_kv_heads, es = c->dtype == SM_F32 ? 4 : 2;
  const bool eight = c->dtype == SM_E4M3;
  a.k_exp = eight ? pool_exps((const uint8_t *)c->k_pool, c->num_blocks, hkv, c->block_size, c->head_dim) : nullptr;
  a.v_exp = eight ? pool_exps((const uint8_t *)c->v_pool, c->num_blocks, hkv, c->block_size, c->head_dim) : nullptr;
  a.seq_ids = seq_ids;
  a.start = start;
  a.row_offsets = row_offsets;
  a.n = n;
  a.total_rows = total_rows;
  a.K = K;
  a.V = V;
  a.k_stride = k_stride;
  a.v_stride = v_stride;
  const auto whole = [&](const void *p, int64_t stride) { return !p || ((uintptr_t)p % 16 == 0 && stride * es % 16 == 0); };
  const bool wide = whole(K, k_stride) && whole(V, v_stride);
  constexpr int64_t kLaunchRows = 1 << 24;  // a launch's threads are counted in 32 bits, 256 for 16 rows
  for (a.first = 0; a.first < total_rows; a.first += kLaunchRows) {
    const int tiles = (int)((std::min<int64_t>(total_rows - a.first, kLaunchRows) + kReadTile - 1) / kReadTile);
    if (eight) launch_read<E4m3>(a, wide, tiles, stream);
    else if (c->dtype == SM_BF16) launch_read<uint16_t>(a, wide, tiles, stream);
    else launch_read<float>(a, wide, tiles, stream);
    if (hipGetLastError() != hipSuccess) return SM_EHIP;
  }
  return SM_OK;
}
