// Attention over a quantised cache, rows whose sums left float32's range (internal).
//
// The other kinds keep a row's maximum where its first keys put it, and sum values times weights before they divide.  A row whose
// denominator then reaches 2^80 (its scores rise far above the first ones), or whose accumulators overflow (values that are large
// themselves, or times such weights), is taken again here, a wave to a row, in float32: with the maximum following, weights are 1 at most,
// and values are multiplied by 2^-25 of them, so that the sum of up to 2^25 keys is within the range of the values.  A key to a lane for the scores,
// D / 64 columns to a lane for the second product.  Slow (about a hundred times), and needed by next to no row: written for few registers,
// as it shares the kernel with the others.
#pragma once
#include "attn_mx.h"

namespace hs {

template <int FMT, int D>
__device__ __forceinline__ void attn_mx_follow(const MxAttnArgs& a, const MxItem& it, MxLds<D>& mem) {
  constexpr int ROW = mx_row_bytes(FMT, D), NS = D / MX_BLOCK, COLS = D / 64;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  float* const q = reinterpret_cast<float*>(mem.tiles) + wave * D;
  const int Rh = a.G * it.M, last_row = (it.blk0 + it.blk_n) * 32 < Rh ? (it.blk0 + it.blk_n) * 32 : Rh;
  const bool last_split = it.sp == it.n_sp - 1;
  const int k_lo = it.sp * it.pages * MX_PAGE, k_hi = last_split || k_lo + it.pages * MX_PAGE > it.L ? it.L : k_lo + it.pages * MX_PAGE;
  const int32_t* const table = a.pool.table + (int64_t)it.s * a.pool.max_blocks;
  // Columns of a NaN block among the item's values are NaN for every row, and those of a NaN or an infinity on its path for a row: no
  // reason to take it again.  What says so otherwise is what was written.
  if (threadIdx.x == 0) mem.nan_columns = 0u;
  mx_meet();
  for (int i = k_lo + (int)threadIdx.x; i < k_hi; i += MXA_THREADS) {
    const int page = table[i / MX_PAGE];
    const unsigned char* const s = a.pool.v_scales + ((((int64_t)(page < 0 || page >= a.pool.n_pages ? 0 : page) * a.pool.Hkv + it.g) * MX_PAGE) + (i & (MX_PAGE - 1))) * NS;
    unsigned nan = 0u;
#pragma unroll
    for (int t = 0; t < NS; ++t) nan |= s[t] == 255 ? 1u << t : 0u;
    if (nan != 0u) atomicOr(&mem.nan_columns, nan);
  }
  mx_meet();
  const unsigned nan_columns = mem.nan_columns;
  auto lost = [&](int r, const MxOwn& own) {
    unsigned beyond = 0u, odd = 0u;
    for (int w = (r >> 5) - it.blk0; w < MXA_WAVES; w += 1 << it.form) beyond |= mem.lost[w][0], odd |= mem.lost[w][1];  // (the waves of its row block)
    if ((beyond >> (r & 31)) & 1u) return true;
    if (((odd >> (r & 31)) & 1u) == 0u) return false;
    const int64_t row = (int64_t)(it.n0 + own.i) * a.Hq + own.h;
    const float* const rec = a.part + (it.rec0 + ((int64_t)own.i * a.Hq + own.h) * it.n_sp + it.sp) * (D + ATTN_REC_PAD);
    bool wrong[COLS];
#pragma unroll
    for (int c = 0; c < COLS; ++c) {
      const int d = COLS * lane + c;
      const float x = it.n_sp == 1 ? bf16_to_f32(static_cast<const bf16_t*>(a.o)[row * D + d]) : rec[d];
      wrong[c] = !(fabsf(x) < HS_INF) && ((nan_columns >> (d / MX_BLOCK)) & 1u) == 0u;
    }
    for (int j = last_split ? own.i : -1; j >= 0;) {
      const bf16_t* const v = static_cast<const bf16_t*>(a.v_tree) + (int64_t)(it.n0 + j) * a.v_stride + it.g * D;
#pragma unroll
      for (int c = 0; c < COLS; ++c) wrong[c] = wrong[c] && fabsf(bf16_to_f32(v[COLS * lane + c])) < HS_INF;
      const int up = a.parent[it.n0 + j];
      j = up < j ? up : -1;
    }
    bool any = false;
#pragma unroll
    for (int c = 0; c < COLS; ++c) any = any || wrong[c];
    return __ballot(any) != 0ull;
  };
  for (int r = it.blk0 * 32 + wave; r < last_row; r += MXA_WAVES) {
    const MxOwn own = mx_own(a, it, r);
    if (!lost(r, own)) continue;
    const bf16_t* const src = static_cast<const bf16_t*>(a.q) + (int64_t)(it.n0 + own.i) * a.q_stride + (int64_t)own.h * D;
#pragma unroll
    for (int c = 0; c < COLS; ++c) q[COLS * lane + c] = bf16_to_f32(src[COLS * lane + c]);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    float m = MXA_FLOOR, l = 0.f, acc[COLS];
#pragma unroll
    for (int c = 0; c < COLS; ++c) acc[c] = 0.f;
    auto raise = [&](float top) {
      const float up = fmaxf(m, top), alpha = exp2_fast(m - up);
      m = up;
      l *= alpha;
#pragma unroll
      for (int c = 0; c < COLS; ++c) acc[c] *= alpha;
    };
    for (int base = k_lo; base < k_hi; base += MX_PAGE) {  // (k_lo is a page's first token)
      int page = table[base / MX_PAGE];
      page = __builtin_amdgcn_readfirstlane(page < 0 || page >= a.pool.n_pages ? 0 : page);
      const int64_t at = ((int64_t)page * a.pool.Hkv + it.g) * MX_PAGE;
      const int left = k_hi - base < MX_PAGE ? k_hi - base : MX_PAGE;
      const int key = lane < left ? lane : left - 1;
      float dot = 0.f;
#pragma unroll 1
      for (int w = 0; w < ROW / 4; ++w) {  // a word of codes: four or eight elements
        constexpr int PER = 32 / Mx<FMT>::BITS;
        const unsigned codes = reinterpret_cast<const unsigned*>(a.pool.k_codes + (at + key) * ROW)[w];
        const float s = mx_scale(a.pool.k_scales[(at + key) * NS + w * PER / MX_BLOCK]);
        const uint4 e = mx_eight<FMT>(codes, 0u, s);
        const unsigned pair[4] = {e.x, e.y, e.z, e.w};
#pragma unroll
        for (int x = 0; x < PER / 2; ++x) {
          dot = __builtin_fmaf(__builtin_bit_cast(float, pair[x] << 16), q[w * PER + 2 * x], dot);
          dot = __builtin_fmaf(__builtin_bit_cast(float, pair[x] & 0xffff0000u), q[w * PER + 2 * x + 1], dot);
        }
      }
      const float score = lane < left ? dot * a.c2 : -HS_INF;
      raise(wave_max(score));
      const float p = exp2_fast(score - m);
      l += wave_sum(p);
#pragma unroll 1
      for (int j = 0; j < left; ++j) {
        const float pj = __shfl(p, j) * 0x1p-25f;
#pragma unroll
        for (int c = 0; c < COLS; ++c) {
          const int d = COLS * lane + c;
          const unsigned byte = a.pool.v_codes[(at + j) * ROW + d * Mx<FMT>::BITS / 8];
          const unsigned e = mx_pair<FMT, 0>(byte, mx_scale(a.pool.v_scales[(at + j) * NS + d / MX_BLOCK]));
          const bool odd = FMT == HS_MX_E2M1 && (d & 1) != 0;  // (two elements to a byte)
          acc[c] = __builtin_fmaf(pj, __builtin_bit_cast(float, odd ? e & 0xffff0000u : e << 16), acc[c]);
        }
      }
    }
    if (last_split) {
      for (int j = own.i; j >= 0;) {
        const bf16_t* const k = static_cast<const bf16_t*>(a.k_tree) + (int64_t)(it.n0 + j) * a.k_stride + it.g * D;
        const bf16_t* const v = static_cast<const bf16_t*>(a.v_tree) + (int64_t)(it.n0 + j) * a.v_stride + it.g * D;
        float dot = 0.f;
#pragma unroll
        for (int c = 0; c < COLS; ++c) dot = __builtin_fmaf(bf16_to_f32(k[COLS * lane + c]), q[COLS * lane + c], dot);
        const float score = wave_sum(dot) * a.c2;
        raise(score);
        const float p = exp2_fast(score - m);
        l += p;
#pragma unroll
        for (int c = 0; c < COLS; ++c) acc[c] = __builtin_fmaf(p * 0x1p-25f, bf16_to_f32(v[COLS * lane + c]), acc[c]);
        const int up = a.parent[it.n0 + j];
        j = up < j ? up : -1;
      }
    }
    const int64_t row = (int64_t)(it.n0 + own.i) * a.Hq + own.h;
    const float inv = mx_inverse(l, it.n_sp == 1) * 0x1p25f;
    if (it.n_sp == 1) {
#pragma unroll
      for (int c = 0; c < COLS; ++c) static_cast<bf16_t*>(a.o)[row * D + COLS * lane + c] = f32_to_bf16(acc[c] * inv);
      if (a.lse != nullptr && lane == 0) a.lse[row] = (m + __log2f(l)) * MXA_LN2;
    } else {
      float* const rec = a.part + (it.rec0 + ((int64_t)own.i * a.Hq + own.h) * it.n_sp + it.sp) * (D + ATTN_REC_PAD);
#pragma unroll
      for (int c = 0; c < COLS; ++c) rec[COLS * lane + c] = acc[c] * inv;
      if (lane == 0) {
        rec[D] = m;
        rec[D + 1] = l;
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }
}

}  // namespace hs
