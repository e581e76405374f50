// Prefill attention of few query vectors over e4m3 pages (gfx950): the waves of
// a workgroup hold the same 32 vectors and take every eighth tile of 32 keys,
// each by itself.
//
// With no second wave at a tile LDS has nothing to share, and 8-bit values need
// no staging: a lane loads the bytes that its fragments of the two products
// are made of, 16 at a time, the next tile's while the current one is
// multiplied, and converts them in registers.  There is no barrier before the
// states are merged.  Two orders make the loads wide:
//   * S^T = K . Q^T sums over features in any order that both operands share:
//     lane half h2 has features h2 D / 2 and on, in chunks of 16.
//   * Row rho of the score block is the token at which register r of lane half
//     h2 has token 16 h2 + r: a half's 16 probabilities are a run of 16 tokens,
//     and so are its bytes of V, the 16 of one dim in a page.
// V's exponents go into the probabilities after their sum is taken and before
// they are rounded to bf16, the matrix cores' type beside V (2.2e-3 of the
// result's size with its own rounding of 1.65e-3).
//
// The two products and the softmax of a tile bound it: 0.7 PFLOP/s at 250 rows
// of 32/8 heads, D = 128, behind 8192 entries (54 us; with the loads left out
// 48, K's rows staged in LDS 57, two tiles ahead 55, the tiles in LDS shared by
// two waves, as for bf16 pages, 111).
#pragma once

#include "prefill_tiles.hpp"

namespace sm {

template <int DH>
constexpr int apart_lds_bytes() {
  return join_bytes<DH, kPfWaves, kPfWaves>() + kPfMaxPages * 4 + 16;
}

template <int DH>
__device__ __forceinline__ void prefill_apart_body(const PrefillArgs &a, const PfBlock &wg, uint8_t *lds) {
  constexpr int KEYS = 32, NKS = DH / 16, NRB = DH / 32, CH = DH / 32;  // CH: 16-byte chunks of half a row
  int *pages = (int *)(lds + join_bytes<DH, kPfWaves, kPfWaves>()), *bad_flag = pages + kPfMaxPages;
  const int g = wg.g, m = wg.m, L = wg.L;
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), c32 = lane & 31, h2 = lane >> 5;
  const int bs_log2 = a.bs_log2, bs = 1 << bs_log2;
  if (!wg.ok) {  // block 0 reports the request and zeroes its rows
    if (wg.qb != 0) return;
    if (tid == 0) set_err(a.err, SM_ERR_EINVAL);
    zero_rows<DH, kPfThreads>(a, wg, 0, m);
    return;
  }
  const int q_lo = wg.qb * a.BQ;
  if (q_lo >= m) return;
  const int nq = min(a.BQ, m - q_lo), pos0 = L - m + q_lo, kend = pos0 + nq;
  if (tid == 0) *bad_flag = 0;
  __syncthreads();
  const int npg = (kend + bs - 1) >> bs_log2;
  for (int p = tid; p < npg; p += kPfThreads) {
    int blk = a.block_table[(int64_t)wg.s * a.max_blocks + p];
    if (blk < 0 || blk >= a.num_blocks) {
      *bad_flag = 1;
      blk = 0;
    }
    pages[p] = blk;
  }
  __syncthreads();
  if (*bad_flag) {  // a corrupt block table: this block's rows are zero
    if (tid == 0) set_err(a.err, SM_ERR_EINVAL);
    zero_rows<DH, kPfThreads>(a, wg, q_lo, nq);
    return;
  }

  // vector c32 -> query head g G + c32 / BQ, row q_lo + c32 % BQ
  const int rr = c32 % a.BQ, hh = c32 / a.BQ;
  const bool vok = hh < a.G && rr < nq;
  const int vhead = g * a.G + (vok ? hh : 0), vrow = wg.r0 + q_lo + (vok ? rr : 0);
  const int vpos = vok ? pos0 + rr : -1;  // an idle vector sees no key
  u32x4_t qf[NKS];
  {
    const uint16_t *qp = a.q + ((int64_t)vrow * a.Hq + vhead) * DH + h2 * (DH / 2);
#pragma unroll
    for (int ks = 0; ks < NKS; ++ks) qf[ks] = vok ? *(const u32x4_t *)(qp + 8 * ks) ^ a.q_sign : u32x4_t{0u, 0u, 0u, 0u};
  }

  const uint64_t page_bytes = a.page_bytes;
  const uint8_t *kbase = (const uint8_t *)a.k_pool + (int64_t)g * bs * DH + h2 * (DH / 2);
  const uint8_t *vbase = (const uint8_t *)a.v_pool + (int64_t)g * bs * DH + ((int64_t)c32 << bs_log2);
  const uint32_t exp_page = (uint32_t)a.Hkv * bs;  // exponent bytes of a page
  const uint8_t *kebase = a.k_exp + g * bs, *vebase = a.v_exp + g * bs;
  const int krow = 16 * (c32 >> 2 & 1) + 4 * (c32 >> 3) + (c32 & 3);  // token of this lane's K row
  struct Tile {
    u32x4_t k[CH], v[NRB], ve;
    int ke;
  };
  auto fetch = [&](int t0, Tile &x) {
    const int kt = t0 + krow, kin = kt & (bs - 1), vt = t0 + 16 * h2, vin = vt & (bs - 1);
    const uint32_t kb = pages[kt < kend ? kt >> bs_log2 : 0], vb = pages[vt < kend ? vt >> bs_log2 : 0];
    const uint8_t *kp = kbase + kb * page_bytes + kin * DH, *vp = vbase + vb * page_bytes + vin;
#pragma unroll
    for (int c = 0; c < CH; ++c) x.k[c] = *(const u32x4_t *)(kp + 16 * c);
    x.ke = kebase[(uint64_t)kb * exp_page + kin];
#pragma unroll
    for (int rb = 0; rb < NRB; ++rb) x.v[rb] = *(const u32x4_t *)(vp + ((int64_t)(32 * rb) << bs_log2));
    x.ve = *(const u32x4_t *)(vebase + (uint64_t)vb * exp_page + vin);
  };

  f32x16_t o[NRB];
#pragma unroll
  for (int rb = 0; rb < NRB; ++rb)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[rb][e] = 0.f;
  float m_run = -INFINITY, l_run = 0.f;
  const float sl2 = a.scale_log2e;
  auto multiply = [&](int t0, Tile &x) {
    f32x16_t sc;
#pragma unroll
    for (int e = 0; e < 16; ++e) sc[e] = 0.f;
    const float kscale = exp_scale(x.ke);
#pragma unroll
    for (int ks = 0; ks < NKS; ++ks) {
      const u32x4_t kf = e4m3_to_bf16(x.k[ks / 2][2 * (ks & 1)], x.k[ks / 2][2 * (ks & 1) + 1], kscale);
      sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(kf), as_bf16x8(qf[ks]), sc, 0, 0, 0);
    }
    if (t0 + KEYS - 1 > pos0) {  // some vector sees part of the tile
      // entries past the last that is needed may hold anything
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int left = kend - (t0 + 16 * h2) - 4 * e;
        const uint32_t keep = left >= 4 ? ~0u : left <= 0 ? 0u : (1u << (8 * left)) - 1u;
        x.ve[e] &= keep;
#pragma unroll
        for (int rb = 0; rb < NRB; ++rb) x.v[rb][e] &= keep;
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) sc[r] = t0 + 16 * h2 + r <= vpos ? sc[r] : -INFINITY;
    }
    float mx = -INFINITY;
#pragma unroll
    for (int r = 0; r < 16; ++r) mx = fmaxf(mx, sc[r]);
    float a0, b0;
    swap32(mx, a0, b0);
    mx = fmaxf(a0, b0);
    const float ms = mx == -INFINITY ? -INFINITY : mx * sl2;
    const bool move = ms > m_run + 8.0f;
    const float m_new = move ? ms : m_run;
    const float mb = m_new == -INFINITY ? 0.f : m_new;
    if (__ballot(move) != 0) {
      const float alpha = move ? __builtin_amdgcn_exp2f(m_run - mb) : 1.f;
      l_run *= alpha;
#pragma unroll
      for (int rb = 0; rb < NRB; ++rb) o[rb] *= alpha;
    }
    m_run = m_new;
    float ps = 0.f;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      sc[r] = __builtin_amdgcn_exp2f(fmaf(sc[r], sl2, -mb));
      ps += sc[r];
      sc[r] *= exp_scale((x.ve[r / 4] >> (8 * (r % 4))) & 0xffu);
    }
    l_run += ps;
#pragma unroll
    for (int kst = 0; kst < 2; ++kst) {
      const u32x4_t pf{cvt_bf16x2(sc[8 * kst + 0], sc[8 * kst + 1]), cvt_bf16x2(sc[8 * kst + 2], sc[8 * kst + 3]),
                       cvt_bf16x2(sc[8 * kst + 4], sc[8 * kst + 5]), cvt_bf16x2(sc[8 * kst + 6], sc[8 * kst + 7])};
#pragma unroll
      for (int rb = 0; rb < NRB; ++rb)
        o[rb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(e4m3_to_bf16(x.v[rb][2 * kst], x.v[rb][2 * kst + 1], 1.f)),
                                                        as_bf16x8(pf), o[rb], 0, 0, 0);
    }
  };

  constexpr int STEP = KEYS * kPfWaves;
  Tile x, y;
  int t0 = KEYS * w;
  if (t0 < kend) fetch(t0, x);
  for (; t0 < kend; t0 += 2 * STEP) {
    if (t0 + STEP < kend) fetch(t0 + STEP, y);
    multiply(t0, x);
    if (t0 + STEP >= kend) break;
    if (t0 + 2 * STEP < kend) fetch(t0 + 2 * STEP, x);
    multiply(t0 + STEP, y);
  }
  float a0, b0;
  swap32(l_run, a0, b0);
  join_groups<DH, kPfWaves, kPfWaves, true>(lds, o, m_run, a0 + b0, min(kPfWaves, (kend + KEYS - 1) / KEYS), vok,
                                            a.out + ((int64_t)vrow * a.Hq + vhead) * DH);
}

}  // namespace sm
