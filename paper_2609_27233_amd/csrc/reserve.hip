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
// second one over all compute units.  What bounds it is the chain of dependent
// reads (request, length, blocks, stores) and barriers, not its bytes: 16
// requests of a row each 3.4 us, 256 of four rows 4.9, and 16 prompts of 2458
// rows (354 KB) 7.1 and 3.0 for the two launches.
#include "cache_meta.hpp"

namespace sm {

struct ReserveArgs {
  const int32_t *seq_ids, *crop, *rows;
  int n, max_rows;
  int32_t *row_offsets, *pos, *slots;
};

// Sums that stay at 2^32 - 1 once they pass it: bad counts cannot wrap round
// to a small total.
__device__ __forceinline__ uint32_t sum_of(uint32_t a, uint32_t b) { return __builtin_elementwise_add_sat(a, b); }

// first i in [0, n) with ends[i] > x (x < ends[n - 1])
__device__ __forceinline__ int first_past(const uint32_t *ends, int n, uint32_t x) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (ends[mid] > x) hi = mid;
    else lo = mid + 1;
  }
  return lo;
}

constexpr int kHeld = 2048;  // blocks whose numbers stay in LDS
constexpr int kOwn = 4;      // and in a thread's registers

enum { kRows, kFreed, kTaken, kSums };

template <int NT>
struct ReserveShared {
  int table[2 * NT];           // sequence ids seen (hashed)
  int ids[NT], keep[NT];       // sequence, entries kept
  int tail[NT];                // the partly filled page that a request's first row goes to
  uint32_t end[kSums][NT];     // inclusive prefix sums of rows, blocks given back, blocks taken
  uint32_t waves[kSums][NT / 64];
  int freed[kHeld], taken[kHeld];
  int flags;                   // 1: bad argument, 2: out of range, 4: corrupt table or stack
};

// Whether another thread's request has put the same id into the table (2 NT
// places for NT ids: the search ends).
template <int NT>
__device__ __forceinline__ bool seen_before(int *table, int s) {
  for (uint32_t at = (uint32_t)s * 2654435761u >> (32 - __builtin_ctz(2 * NT));; at = (at + 1) & (2 * NT - 1)) {
    const int was = atomicCAS(&table[at], -1, s);
    if (was == -1) return false;
    if (was == s) return true;
  }
}

// By one workgroup, request t on thread t (n <= NT).  Dependent reads: the
// request and the cache's state, its length, the blocks concerned; a request
// whose page has room for its rows moves no block.  HERE: positions and slots
// in this launch too.
template <int NT, bool HERE>
__global__ __launch_bounds__(NT) void reserve_kernel(CacheArgs c, ReserveArgs a) {
  __shared__ ReserveShared<NT> sh;
  const int t = threadIdx.x, n = a.n, bs = 1 << c.bs_log2;
  const bool active = t < n;
  const int s = active ? a.seq_ids[t] : -1, k = active && a.crop ? a.crop[t] : 0, m = active ? a.rows[t] : 0;
  const int err = *c.err, top = *c.free_top;
  const bool known = s >= 0 && s < c.max_seqs;
  const int L = known ? c.lengths[s] : 0;
  sh.table[t] = sh.table[NT + t] = -1;
  if (t == 0) sh.flags = 0;
  __syncthreads();
  int flags = 0, keep = 0;
  uint32_t sum[kSums] = {};
  if (active) {
    if (!known || k < 0 || m < 0 || seen_before<NT>(sh.table, s)) flags = 1;
    if (L < 0 || L > c.max_blocks << c.bs_log2 || k > L || (int64_t)L - k + m > c.max_blocks << c.bs_log2) {
      flags |= 2;
    } else if (!flags) {
      keep = L - k;
      const int kept = blocks_for(keep, c.bs_log2);
      sum[kFreed] = blocks_for(L, c.bs_log2) - kept;
      sum[kTaken] = blocks_for(keep + m, c.bs_log2) - kept;
    }
    sum[kRows] = max(m, 0);
  }
  // inclusive prefix sums
#pragma unroll
  for (int off = 1; off < 64; off <<= 1)
#pragma unroll
    for (int q = 0; q < kSums; ++q) {
      const uint32_t u = __shfl_up(sum[q], off, kWave);
      if ((t & 63) >= off) sum[q] = sum_of(sum[q], u);
    }
  if ((t & 63) == 63)
#pragma unroll
    for (int q = 0; q < kSums; ++q) sh.waves[q][t >> 6] = sum[q];
  if (flags) atomicOr(&sh.flags, flags);
  __syncthreads();
  uint32_t all[kSums];
#pragma unroll
  for (int q = 0; q < kSums; ++q) {
    uint32_t before = 0, total = 0;
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) {
      if (w < t >> 6) before = sum_of(before, sh.waves[q][w]);
      total = sum_of(total, sh.waves[q][w]);
    }
    sh.end[q][t] = sum_of(before, sum[q]);
    all[q] = total;
  }
  flags = sh.flags;
  // (all values here are the same in every thread)
  int bit = 0;
  if (err != 0) bit = err;  // sticky: the cache is frozen
  else if (flags & 1 || all[kRows] > (uint32_t)a.max_rows || top < 0 || top > c.num_blocks) bit = SM_ERR_EINVAL;
  else if (flags & 2 || (uint64_t)top + all[kFreed] > (uint32_t)c.num_blocks) bit = SM_ERR_ERANGE;
  else if (all[kTaken] > (uint64_t)top + all[kFreed]) bit = SM_ERR_ENOMEM;
  if (!bit) {
    const int F = (int)all[kFreed], N = (int)all[kTaken];  // (at most num_blocks)
    sh.ids[t] = s;
    sh.keep[t] = keep;
    __syncthreads();
    // Every block that moves, and the partly filled page of a request's first
    // row, must be a real one.  The e-th block given back, the first request's
    // first and its highest logical block first, goes to place F - 1 - .. of
    // the stack above top: the last request is served first.
    auto given = [&](int e, int *place) {
      const int i = first_past(sh.end[kFreed], n, e);
      const int end = sh.end[kFreed][i], first = i ? sh.end[kFreed][i - 1] : 0;
      *place = F - end + e - first;
      return c.block_table + (int64_t)sh.ids[i] * c.max_blocks + blocks_for(sh.keep[i], c.bs_log2) + end - 1 - e;
    };
    bool bad = false;
    int own[kOwn], place[kOwn];
    int32_t *cell[kOwn];
#pragma unroll
    for (int u = 0; u < kOwn; ++u) {
      const int e = t + u * NT;
      if (e >= F) break;
      cell[u] = given(e, &place[u]);
      own[u] = *cell[u];
      bad |= own[u] < 0 || own[u] >= c.num_blocks;
    }
    for (int e = t + kOwn * NT; e < F; e += NT) {
      int p;
      const int blk = *given(e, &p);
      bad |= blk < 0 || blk >= c.num_blocks;
    }
    int popped[kOwn];  // those that lay on the stack before: pops F, F + 1, ...
#pragma unroll
    for (int u = 0; u < kOwn; ++u) {
      const int j = F + t + u * NT;
      popped[u] = j < N ? c.free_stack[top + F - 1 - j] : 0;
      bad |= popped[u] < 0 || popped[u] >= c.num_blocks;
    }
    for (int j = F + t + kOwn * NT; j < N; j += NT) {
      const int blk = c.free_stack[top + F - 1 - j];
      bad |= blk < 0 || blk >= c.num_blocks;
    }
    int tail = 0;
    if (active && m > 0 && (keep & (bs - 1)) != 0) {
      tail = c.block_table[(int64_t)s * c.max_blocks + (keep >> c.bs_log2)];
      bad |= tail < 0 || tail >= c.num_blocks;
    }
    sh.tail[t] = tail;
    if (bad) atomicOr(&sh.flags, 4);
    __syncthreads();
    if (sh.flags) {
      bit = SM_ERR_EINVAL;
    } else {
      // pushes
#pragma unroll
      for (int u = 0; u < kOwn; ++u) {
        if (t + u * NT >= F) break;
        c.free_stack[top + place[u]] = own[u];
        if (place[u] < kHeld) sh.freed[place[u]] = own[u];
        *cell[u] = -1;
      }
      for (int e = t + kOwn * NT; e < F; e += NT) {
        int p;
        int32_t *from = given(e, &p);
        const int blk = *from;
        c.free_stack[top + p] = blk;
        if (p < kHeld) sh.freed[p] = blk;
        *from = -1;
      }
      if (F) __syncthreads();  // (a cell given back may be taken again)
      // pops
      auto take = [&](int j, int blk) {
        const int i = first_past(sh.end[kTaken], n, j);
        c.block_table[(int64_t)sh.ids[i] * c.max_blocks + blocks_for(sh.keep[i], c.bs_log2) + j -
                      (i ? sh.end[kTaken][i - 1] : 0)] = blk;
        if (j < kHeld) sh.taken[j] = blk;
      };
      for (int j = t; j < min(F, N); j += NT) {
        const int p = F - 1 - j;
        take(j, p < kHeld ? sh.freed[p] : c.free_stack[top + p]);
      }
#pragma unroll
      for (int u = 0; u < kOwn; ++u)
        if (F + t + u * NT < N) take(F + t + u * NT, popped[u]);
      for (int j = F + t + kOwn * NT; j < N; j += NT) take(j, c.free_stack[top + F - 1 - j]);
      if (active) c.lengths[s] = keep + m;
      if (t == 0) *c.free_top = top + F - N;
    }
  }
  if (t == 0) {
    a.row_offsets[0] = 0;
    if (bit && err == 0) set_err(c.err, bit);
  }
  if (active) a.row_offsets[t + 1] = bit ? 0 : (int)sh.end[kRows][t];
  if constexpr (HERE) {
    __syncthreads();
    const int total = bit ? 0 : (int)all[kRows];
    for (int r = t; r < a.max_rows; r += NT) {
      int p = 0, slot = -1;
      if (r < total) {
        const int i = first_past(sh.end[kRows], n, r), kept = blocks_for(sh.keep[i], c.bs_log2);
        p = sh.keep[i] + r - (i ? (int)sh.end[kRows][i - 1] : 0);
        const int page = p >> c.bs_log2, j = page - kept + (i ? (int)sh.end[kTaken][i - 1] : 0);
        const int blk = page < kept  ? sh.tail[i]
                        : j < kHeld  ? sh.taken[j]
                                     : c.block_table[(int64_t)sh.ids[i] * c.max_blocks + page];
        slot = (blk << c.bs_log2) + (p & (bs - 1));
      }
      a.pos[r] = p;
      a.slots[r] = slot;
    }
  }
}

// Positions and slots of many rows, after reserve_kernel (whose offsets are
// all 0 where it failed).
constexpr int kRowThreads = 256;

__global__ __launch_bounds__(kRowThreads) void reserve_rows_kernel(CacheArgs c, ReserveArgs a) {
  __shared__ uint32_t ends[SM_MAX_REQUESTS];
  __shared__ int ids[SM_MAX_REQUESTS], last[SM_MAX_REQUESTS];  // last: the length with the rows
  const int t = threadIdx.x;
  const int64_t r = (int64_t)blockIdx.x * kRowThreads + t;
  for (int i = t; i < a.n; i += kRowThreads) {
    const int s = a.seq_ids[i], end = a.row_offsets[i + 1];
    ends[i] = end;
    ids[i] = s;
    last[i] = s >= 0 && s < c.max_seqs ? c.lengths[s] : 0;
  }
  __syncthreads();
  if (r >= a.max_rows) return;
  int p = 0, slot = -1;
  if (a.n && r < ends[a.n - 1]) {
    const int i = first_past(ends, a.n, (uint32_t)r);
    p = last[i] - ((int)ends[i] - (int)r);
    slot = (c.block_table[(int64_t)ids[i] * c.max_blocks + (p >> c.bs_log2)] << c.bs_log2) + (p & ((1 << c.bs_log2) - 1));
  }
  a.pos[r] = p;
  a.slots[r] = slot;
}

// Rows that the one workgroup places itself: 4096 rows of 4 requests 6.6 us
// so and 7.4 by the second launch, 8000 of 8 8.8 and 7.6.
constexpr int kHereRows = 4096;

template <int NT>
static sm_status launch_reserve(const CacheArgs &c, const ReserveArgs &a, hipStream_t stream) {
  if (a.max_rows <= kHereRows) {
    hipLaunchKernelGGL((reserve_kernel<NT, true>), dim3(1), dim3(NT), 0, stream, c, a);
  } else {
    hipLaunchKernelGGL((reserve_kernel<NT, false>), dim3(1), dim3(NT), 0, stream, c, a);
    if (hipGetLastError() != hipSuccess) return SM_EHIP;
    hipLaunchKernelGGL(reserve_rows_kernel, dim3((unsigned)(((int64_t)a.max_rows + kRowThreads - 1) / kRowThreads)),
                       dim3(kRowThreads), 0, stream, c, a);
  }
  return hipGetLastError() == hipSuccess ? SM_OK : SM_EHIP;
}

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
  // 1, 4, 8 or 16 waves by the rows that a thread places, us: 64 rows 3.5, 3.7,
  // 3.9, 4.9; 256 rows of 64 requests 5.1, 3.7, 3.9, 4.9; 512 of 128 with 4 and
  // more waves 4.4, 4.0, 5.0, 1024 of 256 6.1, 4.9, 5.2; 4000 of 16 with 8 and
  // more 8.1, 7.5.
  if (n <= 64 && max_rows <= 64) return launch_reserve<64>(a, r, stream);
  if (n <= 256 && max_rows <= 256) return launch_reserve<256>(a, r, stream);
  if (n <= 512 && max_rows <= 1024) return launch_reserve<512>(a, r, stream);
  return launch_reserve<kMetaThreads>(a, r, stream);
}
