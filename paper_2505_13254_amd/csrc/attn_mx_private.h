// Attention over a quantised cache, work items of one or two row blocks: every wave by itself (internal).
//
// Wave w works for row block w % R on every (8 / R)-th 32 keys of the item's split, alone: its keys go from memory into its
// registers, its softmax state is its own, and the waves of a row block meet once, at the end.
//
// K needs no LDS: which 8 elements of a row a lane's operand register holds is free as long as Q's agree, so a lane
// loads 16 bytes of codes of its own key and converts them in place.  V is converted in the order it is
// loaded, written to the wave's 8 KB of LDS and fetched from there with the transposing read.
//
// A row's maximum stays that of the wave's first 32 keys: weights above one cost no precision (P, sums and accumulators are
// floating point) until a denominator reaches 2^40 (a score 27 above the first ones, or a NaN); the wave then takes its
// keys again, with the maximum following.  So neither a block's maximum nor a rescaling is computed in almost every step.
#pragma once
#include <type_traits>

#include "attn_mx.h"

namespace hs {

template <int FMT, int D, int R>
__device__ __forceinline__ void attn_mx_private(const MxAttnArgs& a, const MxItem& it, MxLds<D>& mem) {
  constexpr int W = MXA_WAVES / R;       // ways: waves that share a row block's keys
  constexpr int NK = D / 16;             // matrix instructions of a 32-key score block
  constexpr int NT = D / 32;
  constexpr int ROW = mx_row_bytes(FMT, D);
  constexpr int EPC = 16 * 8 / Mx<FMT>::BITS;  // elements of a 16-byte chunk of codes
  constexpr int SPC = EPC / 8;                 // matrix instructions that it feeds
  constexpr int KC = NK / SPC;                 // chunks of a K row that a lane holds
  constexpr int CPR = ROW / 16;                // chunks of a row
  constexpr int VC = 32 * CPR / 64;            // V chunks of a lane and 32 keys
  constexpr int NS = D / MX_BLOCK;             // scale bytes of a row
  constexpr int TILE = 32 * D * 2;             // a wave's V tile
  char* const lds = mem.tiles;
  auto& den = mem.den;
  int* const par = mem.par;
  int2* const hops = mem.hops;

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 31, half = lane >> 5;
  const int rb = wave % R, way = wave / R;
  const int Rh = a.G * it.M;
  const int row_base = (it.blk0 + rb) * 32;
  const bool active = rb < it.blk_n;
  const int r_own = row_base + col < Rh ? row_base + col : Rh - 1;
  const int i_own = r_own / a.G, h_own = it.g * a.G + (r_own - i_own * a.G);
  const int64_t L = it.L;
  const bool last_split = it.sp == it.n_sp - 1;
  const int64_t k_lo = (int64_t)it.sp * it.pages * MX_PAGE;
  const int64_t k_hi = last_split ? L : k_lo + (int64_t)it.pages * MX_PAGE;
  const int n_blocks = (int)((k_hi - k_lo + 31) >> 5);  // 32-key blocks of the prefix part

  if (last_split) mx_stage_tree(a, it, par, hops);

  MxState<D> st;
  st.clear();
  char* const tile = lds + wave * TILE;
  if (active) {
    // ---- Q: element order of step kk as K's (see below)
    bf16x8 qf[NK];
    {
      const bf16_t* const src = static_cast<const bf16_t*>(a.q) + (int64_t)(it.n0 + i_own) * a.q_stride + (int64_t)h_own * D;
#pragma unroll
      for (int kk = 0; kk < NK; ++kk)
        qf[kk] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const uint4*>(src + (kk / SPC) * 2 * EPC + half * EPC + (kk % SPC) * 8));
    }
    // ---- V^T fragments: the transposing read returns, to lane l of a 16-lane group, element l % 4 of the 8-byte pieces
    // addressed by lanes l / 4 + {0, 4, 8, 12} of the group
    const int tr_a = lane & 3, tr_j = (lane >> 2) & 3, tr_dh = (lane >> 4) & 1;
    auto second = [&](const uint4& p0, const uint4& p1) {
      const bf16x8 b0 = __builtin_bit_cast(bf16x8, p0), b1 = __builtin_bit_cast(bf16x8, p1);
#pragma unroll
      for (int k2 = 0; k2 < 2; ++k2)
#pragma unroll
        for (int tt = 0; tt < NT; ++tt) {
          bf16x8 vf;
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const int key = 16 * k2 + 8 * x + 4 * half + tr_j;
            const char* const p = tile + v_at<D>(key, 4 * tt + 2 * tr_dh + (tr_a >> 1)) + (tr_a & 1) * 8;
            const shortx4 got = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4_ptr)p);
            const bf16x4 four = __builtin_bit_cast(bf16x4, got);
#pragma unroll
            for (int e = 0; e < 4; ++e) vf[4 * x + e] = four[e];
          }
          st.acc[tt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, k2 == 0 ? b0 : b1, st.acc[tt], 0, 0, 0);
        }
    };
    const floatx16 zero = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};

    // ---- prefix: 32-key blocks way, way + W, ... of the split
    const int32_t* const table = a.pool.table + (int64_t)it.s * a.pool.max_blocks + (k_lo >> 6);
    const int mine = n_blocks > way ? (n_blocks - way + W - 1) / W : 0;
    int page_of = 0;  // lane j: the page of this wave's block j of the present 64
    uint4 kc[KC], vc[VC];
    unsigned ks = 0, vs[VC];
    auto request = [&](int j) {
      if ((j & 63) == 0) {
        const int b = way + (j + lane) * W;
        int p = b < n_blocks ? table[b >> 1] : 0;
        page_of = p < 0 || p >= a.pool.n_pages ? 0 : p;  // (a page outside the pool would be a caller's error)
      }
      const int b = way + j * W;
      const int page = __builtin_amdgcn_readlane(page_of, j & 63);
      const int64_t base = ((int64_t)page * a.pool.Hkv + it.g) * MX_PAGE;
      const int s0 = (b & 1) * 32;
      const int last = (int)(k_hi - k_lo - (int64_t)b * 32) - 1;  // last key of the block that exists (>= 0)
      const int kr = s0 + (col < last ? col : last);              // (keys behind it repeat it; masked)
      const unsigned char* const kp = a.pool.k_codes + (base + kr) * ROW + half * 16;
#pragma unroll
      for (int n = 0; n < KC; ++n) kc[n] = *reinterpret_cast<const uint4*>(kp + n * 32);
      const unsigned char* const sp = a.pool.k_scales + (base + kr) * NS;
      if constexpr (NS == 4) ks = *reinterpret_cast<const unsigned*>(sp);
      else ks = *reinterpret_cast<const unsigned short*>(sp);
#pragma unroll
      for (int n = 0; n < VC; ++n) {
        const int id = n * 64 + lane, key = id / CPR, c = id % CPR;
        const int64_t vr = base + s0 + (key < last ? key : last);
        vc[n] = *reinterpret_cast<const uint4*>(a.pool.v_codes + vr * ROW + c * 16);
        vs[n] = a.pool.v_scales[vr * NS + c * EPC / MX_BLOCK];
      }
    };
    auto step = [&](int j, auto safe) {
      constexpr bool SAFE = decltype(safe)::value;
      if (SAFE) request(j);
      floatx16 S = zero;
#pragma unroll
      for (int n = 0; n < KC; ++n) {
        // chunk n of a half-wave: elements 2 EPC n + EPC half ..
        const unsigned byte = FMT == HS_MX_E4M3 ? ks >> (8 * n) : ks >> (8 * (2 * n + half));
        const float s = mx_scale(byte & 255u);
        const unsigned w[4] = {kc[n].x, kc[n].y, kc[n].z, kc[n].w};
#pragma unroll
        for (int e = 0; e < SPC; ++e) {
          const uint4 f = FMT == HS_MX_E4M3 ? mx_eight<FMT>(w[(2 * e) & 3], w[(2 * e + 1) & 3], s) : mx_eight<FMT>(w[e & 3], 0u, s);
          S = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, f), qf[n * SPC + e], S, 0, 0, 0);
        }
      }
#pragma unroll
      for (int n = 0; n < VC; ++n) {
        const int id = n * 64 + lane, key = id / CPR, c = id % CPR;
        const float s = mx_scale(vs[n]);
        const unsigned w[4] = {vc[n].x, vc[n].y, vc[n].z, vc[n].w};
#pragma unroll
        for (int e = 0; e < SPC; ++e)
          *reinterpret_cast<uint4*>(tile + v_at<D>(key, c * SPC + e)) =
              FMT == HS_MX_E4M3 ? mx_eight<FMT>(w[(2 * e) & 3], w[(2 * e + 1) & 3], s) : mx_eight<FMT>(w[e & 3], 0u, s);
      }
      if (!SAFE && j + 1 < mine) request(j + 1);
      const int left = (int)(k_hi - k_lo - (int64_t)(way + j * W) * 32);  // keys of this block
      if (left < 32) {
#pragma unroll
        for (int v = 0; v < 16; ++v) S[v] = 8 * (v >> 2) + 4 * half + (v & 3) < left ? S[v] : -HS_INF;
      }
      uint4 p0, p1;
      if constexpr (SAFE) {
        st.softmax(S, a.c2, p0, p1);
      } else {
        if (j == 0) st.start(S, a.c2);
        st.exp_half(S, a.c2, 0, p0, st.l);
        st.exp_half(S, a.c2, 1, p1, st.l);
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // the tile is read by other lanes than wrote it
      second(p0, p1);
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    };
    if (mine > 0) {
      request(0);
      for (int j = 0; j < mine; ++j) step(j, std::false_type{});
      if (st.over(st.l)) {  // the first block's maximum did not hold: again, with the maximum following
        st.clear();
        for (int j = 0; j < mine; ++j) step(j, std::true_type{});
      }
    }

    // ---- the tree's own rows, block by block from the last that a row of this wave can see to the first
    if (last_split) {
      const int r_top = row_base + 31 < Rh ? row_base + 31 : Rh - 1;
      int cur = i_own;
      for (int b = (r_top / a.G) >> 5; b >= 0; --b) {
        const unsigned word = mx_path_word(hops, cur, b);
        if (b % W != way || __ballot(word != 0u) == 0ull) continue;
        const int last = it.M - 1 - 32 * b;  // >= 0
        const int kr = it.n0 + 32 * b + (col < last ? col : last);
        const bf16_t* const kp = static_cast<const bf16_t*>(a.k_tree) + (int64_t)kr * a.k_stride + it.g * D;
        floatx16 S = zero;
#pragma unroll
        for (int kk = 0; kk < NK; ++kk) {
          const uint4 f = *reinterpret_cast<const uint4*>(kp + (kk / SPC) * 2 * EPC + half * EPC + (kk % SPC) * 8);
          S = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, f), qf[kk], S, 0, 0, 0);
        }
        constexpr int TC = 32 * (D / 8) / 64;
        const bf16_t* const vb = static_cast<const bf16_t*>(a.v_tree) + (int64_t)(it.n0 + 32 * b) * a.v_stride + it.g * D;
        ushort2v most = {0, 0};
#pragma unroll
        for (int n = 0; n < TC; ++n) {
          const int id = n * 64 + lane, key = id / (D / 8), c = id % (D / 8);
          const uint4 w = *reinterpret_cast<const uint4*>(vb + (key < last ? key : last) * a.v_stride + c * 8);
          note_bits(most, w);
          *reinterpret_cast<uint4*>(tile + v_at<D>(key, c)) = w;
        }
        const bool odd = __ballot(has_odd(most)) != 0ull;
        if (odd)
          for (int n = 0; n < TC; ++n) {
            const int id = n * 64 + lane;
            uint4* const at = reinterpret_cast<uint4*>(tile + v_at<D>(id / (D / 8), id % (D / 8)));
            *at = without_odd(*at);
          }
#pragma unroll
        for (int v = 0; v < 16; ++v) S[v] = (word >> (8 * (v >> 2) + 4 * half + (v & 3))) & 1u ? S[v] : -HS_INF;
        uint4 p0, p1;
        st.softmax(S, a.c2, p0, p1);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        second(p0, p1);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if (odd) st.add_odd(vb, a.v_stride, last < 31 ? last + 1 : 32, word, half);
      }
    }
    st.l = half_sum(st.l);
    if (half == 0) {
      den[wave][0][col] = st.m;
      den[wave][1][col] = st.l;
    }
  }
  __syncthreads();  // every wave has its sums (and no tile is read any more)

  // ---- the ways of a row block meet: each leaves its accumulators, scaled to the common maximum, and adds up its share
  // of the columns
  float top = MXA_FLOOR, total = 0.f;
  if (active) {
#pragma unroll
    for (int x = 0; x < W; ++x) top = fmaxf(top, den[x * R + rb][0][col]);
#pragma unroll
    for (int x = 0; x < W; ++x) total += den[x * R + rb][1][col] * exp2_fast(den[x * R + rb][0][col] - top);
    const float mine = exp2_fast(st.m - top);
    float4* const to = reinterpret_cast<float4*>(lds) + wave * (NT * 4 * 64) + lane;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int b = 0; b < 4; ++b)
        to[(t * 4 + b) * 64] = make_float4(st.acc[t][4 * b] * mine, st.acc[t][4 * b + 1] * mine, st.acc[t][4 * b + 2] * mine, st.acc[t][4 * b + 3] * mine);
  }
  __syncthreads();
  if (!active || row_base + col >= Rh) return;
  const int64_t out_row = (int64_t)(it.n0 + i_own) * a.Hq + h_own;
  float* const rec = a.part + (it.rec0 + ((int64_t)i_own * a.Hq + h_own) * it.n_sp + it.sp) * (D + ATTN_REC_PAD);
  const float inv = 1.f / total;
  for (int x = way; x < NT * 4; x += W) {
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int y = 0; y < W; ++y) {
      const float4 f = reinterpret_cast<const float4*>(lds)[(y * R + rb) * (NT * 4 * 64) + x * 64 + lane];
      sum.x += f.x, sum.y += f.y, sum.z += f.z, sum.w += f.w;
    }
    mx_write4(a, it.n_sp == 1, out_row, rec, 8 * x + 4 * half, sum, inv);  // (column 32 (x / 4) + 8 (x % 4) + 4 half)
  }
  if (way == 0 && half == 0) {
    if (it.n_sp == 1) {
      if (a.lse != nullptr) a.lse[out_row] = (top + __log2f(total)) * MXA_LN2;
    } else {
      rec[D] = top;
      rec[D + 1] = total;
    }
  }
}

}  // namespace hs
