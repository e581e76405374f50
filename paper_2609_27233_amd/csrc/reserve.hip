// Block tables, positions and slots of the rows that a step's requests are
// about to write (gfx950): kv_reserve.
//
// Metadata only: n lengths, the blocks that move between the table and the
// free stack, and 8 bytes per row.  One workgroup (request t on thread t)
// checks everything first, then moves the blocks at places fixed by prefix
// sums: the freed ones are pushed in reverse request order, highest logical
// block first, and the taken ones popped in request order, lowest first, so
// the state is the one of a rollback followed by an append.  The rows'
// positions and slots follow in the same launch, or for many rows in a
// second one over all compute units.
#include "cache_meta.hpp"

namespace sm {

struct ReserveArgs {
  const int32_t *seq_ids, *crop, *rows;
  int n, max_rows;
  int32_t *row_offsets, *pos, *slots;
};

// Inclusive prefix sum over kMetaThreads threads in 64 bits; `red` needs 16.
__device__ __forceinline__ int64_t scan64(int64_t v, int64_t *red, int64_t *total) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const int64_t u = __shfl_up(v, off, kWave);
    if (lane >= off) v += u;
  }
  __syncthreads();
  if (lane == 63) red[w] = v;
  __syncthreads();
  int64_t before = 0, tot = 0;
  for (int i = 0; i < kMetaThreads / 64; ++i) {
    if (i < w) before += red[i];
    tot += red[i];
  }
  *total = tot;
  return v + before;
}

// first i in [0, n) with ends[i] > x (x < ends[n - 1])
__device__ __forceinline__ int first_past(const int *ends, int n, int x) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (ends[mid] > x) hi = mid;
    else lo = mid + 1;
  }
  return lo;
}

struct ReserveShared {
  int64_t red[16];
  int ids[kMetaThreads];
  int keep[kMetaThreads];       // entries kept
  int row_end[kMetaThreads];    // inclusive prefix sums of the rows,
  int freed_end[kMetaThreads];  // of the blocks given back
  int taken_end[kMetaThreads];  // and of the blocks taken
  int fl_inval, fl_range, fl_stack, s_err, s_top;
};

// The position and slot of row r: of request i, which ends[] names.
__device__ __forceinline__ void put_row(const CacheArgs &c, const ReserveArgs &a, int r, int s, int p) {
  const int blk = c.block_table[(int64_t)s * c.max_blocks + (p >> c.bs_log2)];
  a.pos[r] = p;
  a.slots[r] = (blk << c.bs_log2) + (p & ((1 << c.bs_log2) - 1));
}

// The checks and the block moves; returns 0 when all of it was applied, else
// the error bit (uniform).
__device__ int reserve_meta(const CacheArgs &c, const ReserveArgs &a, ReserveShared &sh) {
  const int t = threadIdx.x;
  const bool active = t < a.n;
  const int s = active ? a.seq_ids[t] : -1, k = active && a.crop ? a.crop[t] : 0, m = active ? a.rows[t] : 0;
  sh.ids[t] = s;
  if (t == 0) {
    sh.fl_inval = sh.fl_range = sh.fl_stack = 0;
    sh.s_err = *c.err;
    sh.s_top = *c.free_top;
  }
  __syncthreads();
  if (sh.s_err != 0) return sh.s_err;  // sticky: the cache is frozen
  if (active && (k < 0 || m < 0 || !id_ok(sh.ids, t, s, c.max_seqs))) sh.fl_inval = 1;
  int64_t total_rows;
  const int64_t row_end = scan64(m < 0 ? 0 : m, sh.red, &total_rows);  // (its barriers: the flag is there)
  const int top = sh.s_top;
  if (sh.fl_inval || total_rows > a.max_rows || top < 0 || top > c.num_blocks) return SM_ERR_EINVAL;
  const int cap = c.max_blocks << c.bs_log2;
  int keep = 0, had = 0, kept = 0, want = 0;
  if (active) {
    const int L = c.lengths[s];
    if (L < 0 || L > cap || k > L || (int64_t)L - k + m > cap) {
      sh.fl_range = 1;
    } else {
      keep = L - k;
      had = blocks_for(L, c.bs_log2);
      kept = blocks_for(keep, c.bs_log2);
      want = blocks_for(keep + m, c.bs_log2);
    }
  }
  int64_t all_freed, all_taken;
  const int64_t freed_end = scan64(had - kept, sh.red, &all_freed);
  const int64_t taken_end = scan64(want - kept, sh.red, &all_taken);
  if (sh.fl_range || top + all_freed > c.num_blocks) return SM_ERR_ERANGE;
  if (all_taken > top + all_freed) return SM_ERR_ENOMEM;
  // (all sums are at most num_blocks from here)
  const int F = (int)all_freed, N = (int)all_taken;
  sh.keep[t] = keep;
  sh.row_end[t] = (int)row_end;
  sh.freed_end[t] = (int)freed_end;
  sh.taken_end[t] = (int)taken_end;
  __syncthreads();
  // every block that moves, and the partly filled page of a request's first
  // row, must name a real block
  // e-th block of the list that the pushes go through, the first request's first
  auto freed_cell = [&](int e, int *place) {
    const int i = first_past(sh.freed_end, a.n, e);
    const int at = e - (i ? sh.freed_end[i - 1] : 0), cnt = sh.freed_end[i] - (i ? sh.freed_end[i - 1] : 0);
    *place = top + F - sh.freed_end[i] + at;
    return c.block_table + (int64_t)sh.ids[i] * c.max_blocks + blocks_for(sh.keep[i], c.bs_log2) + cnt - 1 - at;
  };
  bool bad = false;
  for (int e = t; e < F; e += kMetaThreads) {
    int place;
    const int blk = *freed_cell(e, &place);
    bad |= blk < 0 || blk >= c.num_blocks;
  }
  for (int j = F + t; j < N; j += kMetaThreads) {
    const int blk = c.free_stack[top + F - 1 - j];
    bad |= blk < 0 || blk >= c.num_blocks;
  }
  if (active && m > 0 && (keep & ((1 << c.bs_log2) - 1)) != 0) {
    const int blk = c.block_table[(int64_t)s * c.max_blocks + (keep >> c.bs_log2)];
    bad |= blk < 0 || blk >= c.num_blocks;
  }
  if (bad) sh.fl_stack = 1;
  __syncthreads();
  if (sh.fl_stack) return SM_ERR_EINVAL;
  for (int e = t; e < F; e += kMetaThreads) {
    int place;
    int32_t *cell = freed_cell(e, &place);
    c.free_stack[place] = *cell;
    *cell = -1;
  }
  if (F) __syncthreads();  // (uniform)
  for (int j = t; j < N; j += kMetaThreads) {
    const int i = first_past(sh.taken_end, a.n, j);
    c.block_table[(int64_t)sh.ids[i] * c.max_blocks + blocks_for(sh.keep[i], c.bs_log2) + j -
                  (i ? sh.taken_end[i - 1] : 0)] = c.free_stack[top + F - 1 - j];
  }
  if (active) c.lengths[s] = keep + m;
  if (t == 0) *c.free_top = top + F - N;
  return 0;
}

// HERE: positions and slots in this launch too.
template <bool HERE>
__global__ __launch_bounds__(kMetaThreads) void reserve_kernel(CacheArgs c, ReserveArgs a) {
  __shared__ ReserveShared sh;
  const int t = threadIdx.x;
  const int bit = reserve_meta(c, a, sh);
  if (bit) {
    if (t == 0 && sh.s_err == 0) set_err(c.err, bit);
    for (int i = t; i <= a.n; i += kMetaThreads) a.row_offsets[i] = 0;
  } else {
    if (t == 0) a.row_offsets[0] = 0;
    if (t < a.n) a.row_offsets[t + 1] = sh.row_end[t];
  }
  if constexpr (HERE) {
    __syncthreads();  // the table's new cells
    const int total = bit || a.n == 0 ? 0 : sh.row_end[a.n - 1];
    for (int r = t; r < a.max_rows; r += kMetaThreads) {
      if (r < total) {
        const int i = first_past(sh.row_end, a.n, r);
        put_row(c, a, r, sh.ids[i], sh.keep[i] + r - (i ? sh.row_end[i - 1] : 0));
      } else {
        a.pos[r] = 0;
        a.slots[r] = -1;
      }
    }
  }
}

// Positions and slots of many rows, after reserve_kernel (whose offsets are
// all 0 where it failed).
constexpr int kRowThreads = 256, kRowsPerThread = 4;

__global__ __launch_bounds__(kRowThreads) void reserve_rows_kernel(CacheArgs c, ReserveArgs a) {
  __shared__ int ends[SM_MAX_REQUESTS];
  const int t = threadIdx.x;
  for (int i = t; i < a.n; i += kRowThreads) ends[i] = a.row_offsets[i + 1];
  __syncthreads();
  const int total = a.n ? ends[a.n - 1] : 0;
#pragma unroll
  for (int u = 0; u < kRowsPerThread; ++u) {
    const int64_t r = ((int64_t)blockIdx.x * kRowsPerThread + u) * kRowThreads + t;
    if (r >= a.max_rows) continue;
    if (r < total) {
      const int i = first_past(ends, a.n, (int)r);
      const int s = a.seq_ids[i];
      put_row(c, a, (int)r, s, c.lengths[s] - (ends[i] - (int)r));
    } else {
      a.pos[r] = 0;
      a.slots[r] = -1;
    }
  }
}

// Rows that the one workgroup places itself.
constexpr int kHereRows = 4096;

}  // namespace sm

using namespace sm;

SM_API sm_status sm_kv_reserve(const sm_paged_cache *c, const int32_t *seq_ids, const int32_t *crop, const int32_t *rows,
                               int n, int max_rows, int32_t *row_offsets, int32_t *pos, int32_t *slots,
                               hipStream_t stream) {
  CacheArgs a;
  if (!cache_ok(c, a) || n < 0 || n > SM_MAX_REQUESTS || n > c->max_seqs || max_rows < 0) return SM_EINVAL;
  if ((int64_t)c->num_blocks * c->block_size > INT32_MAX) return SM_EINVAL;
  if (!row_offsets || (n > 0 && (!seq_ids || !rows)) || (max_rows > 0 && (!pos || !slots))) return SM_EINVAL;
  const ReserveArgs r{seq_ids, crop, rows, n, max_rows, row_offsets, pos, slots};
  if (max_rows <= kHereRows) {
    hipLaunchKernelGGL(reserve_kernel<true>, dim3(1), dim3(kMetaThreads), 0, stream, a, r);
  } else {
    hipLaunchKernelGGL(reserve_kernel<false>, dim3(1), dim3(kMetaThreads), 0, stream, a, r);
    if (hipGetLastError() != hipSuccess) return SM_EHIP;
    const int per = kRowThreads * kRowsPerThread;
    hipLaunchKernelGGL(reserve_rows_kernel, dim3((unsigned)(((int64_t)max_rows + per - 1) / per)), dim3(kRowThreads), 0,
                       stream, a, r);
  }
  return hipGetLastError() == hipSuccess ? SM_OK : SM_EHIP;
}
