// Prefill attention over the paged cache (gfx950): the kernels and their host
// side; the tiles they work by are in prefill_tiles.hpp.
#include "prefill_apart.hpp"

namespace sm {

template <int DH, int KS, bool EIGHT = false>
__global__ __launch_bounds__(kPfThreads, 2) void prefill_bf16(PrefillArgs a) {
  __shared__ __attribute__((aligned(16))) uint8_t lds[pf_lds_bytes<DH, KS, EIGHT>()];
  prefill_body<DH, KS, EIGHT>(a, pf_block(a), lds);
}

// For calls of few rows: blocks of KS = 4, but a request of up to kPfFewKeys
// keys is done sooner by the waves of its vectors alone than by four groups
// and their merge.  The length is known here only, so the choice is too.  Us
// alone and split, D = 128: one row of 32/8 heads 1 key 5.6, 6.7; 201 9.2,
// 9.5; 401 12.5, 12.0; 4097 78, 53; 64 rows of 8/8 heads 64 keys 6.1, 8.3; 264
// 11.3, 12.0; 364 12.5, 12.4; 564 16.0, 15.1.  D = 64, one row of 16/4: 201
// 6.9, 7.1; 301 7.6, 7.7; 401 9.3, 8.8.
constexpr int kPfFewKeys = 320;

template <int DH, bool EIGHT = false>
__global__ __launch_bounds__(kPfThreads, 2) void prefill_few_bf16(PrefillArgs a) {
  __shared__ __attribute__((aligned(16))) uint8_t lds[pf_lds_bytes<DH, 4, EIGHT>()];
  static_assert(pf_lds_bytes<DH, 1, EIGHT>() <= pf_lds_bytes<DH, 4, EIGHT>(), "one LDS for both");
  const PfBlock wg = pf_block(a);
  if (wg.L <= kPfFewKeys) prefill_body<DH, 1, EIGHT>(a, wg, lds);
  else prefill_body<DH, 4, EIGHT>(a, wg, lds);
}

template <int DH>
__global__ __launch_bounds__(kPfThreads, 2) void prefill_apart_e4m3(PrefillArgs a) {
  __shared__ __attribute__((aligned(16))) uint8_t lds[apart_lds_bytes<DH>()];
  prefill_apart_body<DH>(a, pf_block(a), lds);
}

}  // namespace sm

using namespace sm;

SM_API sm_status sm_prefill_attention(const sm_paged_cache *c, const int32_t *seq_ids, int n,
                                      const int32_t *q_offsets, int total_rows, const void *q, int num_q_heads,
                                      float scale, int max_rows, void *out, hipStream_t stream) {
  if (!c || n < 0 || max_rows < 0 || total_rows < 0) return SM_EINVAL;
  if (n == 0) return SM_OK;
  if (!seq_ids || !q_offsets || !q || !out || !c->k_pool || !c->v_pool || !c->block_table || !c->lengths ||
      !c->err)
    return SM_EINVAL;
  const bool eight = c->dtype == SM_E4M3;
  if ((c->dtype != SM_BF16 && !eight) || !(fabsf(scale) <= 3.0e38f)) return SM_EINVAL;  // a finite scale
  const int H = c->num_kv_heads, D = c->head_dim, bs = c->block_size;
  if (H <= 0 || num_q_heads <= 0 || num_q_heads % H != 0) return SM_EINVAL;
  const int G = num_q_heads / H;
  if (G > 16 || (D != 64 && D != 128)) return SM_EINVAL;
  if (bs < 16 || (bs & (bs - 1)) != 0 || c->max_blocks_per_seq <= 0 || c->max_blocks_per_seq > kPfMaxPages ||
      c->num_blocks <= 0 || c->max_seqs <= 0)
    return SM_EINVAL;
  if (n > 65535 || (uint64_t)H * bs * D * 2 > 0xffffffffull) return SM_EINVAL;
  PrefillArgs a = pf_args(c, q, num_q_heads, scale);
  a.seq_ids = seq_ids;
  a.q_offsets = q_offsets;
  a.out = (uint16_t *)out;
  a.n = n;
  a.total_rows = total_rows;
  a.max_rows = max_rows;
  const PrefillPlan plan = plan_prefill(n, H, G, total_rows, max_rows, (int64_t)c->max_blocks_per_seq * bs);
  const bool apart = eight && prefill_apart(n, H, G, total_rows, max_rows);
  const int ks = apart ? 8 : plan.splits;
  a.BQ = kPfVec / ks / G;
  const int nqb = max_rows > 0 ? (max_rows + a.BQ - 1) / a.BQ : 1;  // block 0 reports bad requests
  if ((int64_t)nqb * n * H > 0x7fffffff) return SM_EINVAL;
  a.nqb = nqb;
  const dim3 grid(nqb * n * H);
  const auto kernel = [&](auto dh, auto e) {
    constexpr int DH = decltype(dh)::value;
    constexpr bool EIGHT = decltype(e)::value;
    if constexpr (EIGHT)
      if (apart) return prefill_apart_e4m3<DH>;
    return plan.few  ? prefill_few_bf16<DH, EIGHT>
           : ks == 4 ? prefill_bf16<DH, 4, EIGHT>
           : ks == 2 ? prefill_bf16<DH, 2, EIGHT>
                     : prefill_bf16<DH, 1, EIGHT>;
  };
  const std::integral_constant<int, 128> d128{};
  const std::integral_constant<int, 64> d64{};
  const auto chosen = D == 128 ? (eight ? kernel(d128, std::true_type()) : kernel(d128, std::false_type()))
                               : (eight ? kernel(d64, std::true_type()) : kernel(d64, std::false_type()));
  hipLaunchKernelGGL(chosen, grid, dim3(kPfThreads), 0, stream, a);
  return hipGetLastError() == hipSuccess ? SM_OK : SM_EHIP;
}
