// Attention over a quantised cache, work items of one or two row blocks: every wave by itself (internal).
//
// Wave w works for row block w % R (R = 1 or 2) on every (8 / R)-th 32 keys of the item's split, alone: its keys go from memory into its
// registers, its softmax state is its own, and the waves of a row block meet once, at the end.
//
// K needs no LDS: which 8 elements of a row a lane's operand register holds is free as long as Q's agree, so a lane
// loads 16 bytes of codes of its own key and converts them in place.  V is converted in the order it is
// loaded, written to the wave's 8 KB of LDS and fetched from there with the transposing read.
//
// A row's maximum stays that of the tree's rows and the wave's first 32 keys: neither a block's maximum nor a rescaling is
// computed in almost every step.  Weights above one cost no precision (P, sums and accumulators are floating point) until
// a denominator reaches 2^80 (a score 55 above the first ones) or an accumulator overflows: attn_mx_follow then takes the row.
#pragma once
#include <type_traits>

#include "attn_mx.h"

namespace hs {

// Returns whether all rows' sums stayed in range (mem.lost: which did not); rows that did not are written, but wrong.
template <int FMT, int D, int R>
__device__ __forceinline__ bool attn_mx_private(const MxAttnArgs& a, const MxItem& it, MxLds<D>& mem) {
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
  const MxOwn own = mx_own(a, it, row_base + col < Rh ? row_base + col : Rh - 1);
  const bool last_split = it.sp == it.n_sp - 1;
  const int k_lo = it.sp * it.pages * MX_PAGE, k_hi = last_split || k_lo + it.pages * MX_PAGE > it.L ? it.L : k_lo + it.pages * MX_PAGE;
  const int keys = k_hi > k_lo ? k_hi - k_lo : 0;  // of the prefix part
  const int n_blocks = (keys + 31) >> 5;

  // ---- what the first steps wait for is requested first, all of it: the pages, the tree's parents, Q, a block of the tree
  const int32_t* const table = a.pool.table + (int64_t)it.s * a.pool.max_blocks + (k_lo >> 6);
  const int mine = active && n_blocks > way ? (n_blocks - way + W - 1) / W : 0;
  auto pages_from = [&](int j) {  // lane l: the page of this wave's block j + l
    const int b = way + (j + lane) * W, p = table[b < n_blocks ? b >> 1 : 0];
    return p < 0 || p >= a.pool.n_pages ? 0 : p;  // (a page outside the pool would be a caller's error)
  };
  int page_of = mine > 0 ? pages_from(0) : 0;
  MxParents parents = {};
  MxPath path = {0u, 0u, own.i};
  const bool small = it.M <= 64;
  if (last_split) parents = mx_request_parents(a, it);
  char* const q_lds = lds + MXA_WAVES * TILE + rb * 32 * MX_Q_ROW<D>;
  static_assert(MXA_WAVES * TILE + 2 * 32 * MX_Q_ROW<D> <= (int)sizeof(mem.tiles), "Q behind the V tiles");
  if (active) mx_stage_q<D>(a, it, row_base, q_lds, way * 64 + lane, W * 64);

  // ---- prefix: 32-key blocks way, way + W, ... of the split
  uint4 kc[KC], vc[VC];
  unsigned ks = 0, vs[VC];
  // (keys behind the last of a block repeat it; they are masked.  Scalar bases, 32 bits to a lane.)
  // The loop's requests are unconditional (behind the last block it again): a wait can then count the younger ones, where a
  // branch around them makes it a wait for all.
  int64_t base = 0;
  unsigned last = 0;
  int page_j = 0;
  auto request_k = [&](int j) {
    const int b = way + j * W;
    base = ((int64_t)__builtin_amdgcn_readlane(page_of, j - page_j) * a.pool.Hkv + it.g) * MX_PAGE + (b & 1) * 32;
    last = (unsigned)(keys - b * 32 < 32 ? keys - b * 32 - 1 : 31);
    const unsigned kr = (unsigned)col < last ? (unsigned)col : last;
    mx_mem kp = (mx_mem)(a.pool.k_codes + base * ROW), kp_s = (mx_mem)(a.pool.k_scales + base * NS);
    asm volatile("" : "+s"(kp), "+s"(kp_s));
#pragma unroll
    for (int n = 0; n < KC; ++n) kc[n] = mx_load16(kp + (kr * ROW + half * 16 + n * 32));
    if constexpr (NS == 4) ks = *reinterpret_cast<const __attribute__((address_space(1))) unsigned*>(kp_s + kr * NS);
    else ks = *reinterpret_cast<const __attribute__((address_space(1))) unsigned short*>(kp_s + kr * NS);
  };
  auto request_v = [&]() {  // of the block that request_k was called for last
    mx_mem vp = (mx_mem)(a.pool.v_codes + base * ROW), vp_s = (mx_mem)(a.pool.v_scales + base * NS);
    asm volatile("" : "+s"(vp), "+s"(vp_s));
#pragma unroll
    for (int n = 0; n < VC; ++n) {
      const unsigned id = n * 64 + lane, key = id / CPR, c = id % CPR, vr = key < last ? key : last;
      vc[n] = mx_load16(vp + (vr * ROW + c * 16));
      vs[n] = vp_s[vr * NS + c * EPC / MX_BLOCK];
    }
  };
  // The tree's own rows go straight into LDS, those of a small tree from here: they take no registers on the way.  Lane l's 16 bytes come to lie
  // behind lane l - 1's, so each lane fetches the piece whose place that is.
  constexpr int TC = 32 * (D / 8) / 64;
  char* const tile = lds + wave * TILE;
  auto request_tree = [&](const void* rows, int64_t stride, int b, char* to) {
    const int end = it.M - 1 - 32 * b;  // >= 0; rows behind the last repeat it
    int ln = lane;
    asm volatile("" : "+v"(ln));  // (no address of these is kept in registers from block to block)
    const bf16_t* const from = static_cast<const bf16_t*>(rows) + (int64_t)(it.n0 + 32 * b) * stride + it.g * D;
#pragma unroll
    for (int n = 0; n < TC; ++n) {
      const int id = n * 64 + ln, key = id / (D / 8), c = (v_at<D>(key, id % (D / 8)) - key * (2 * D)) >> 4;
      mx_to_lds(from + (key < end ? key : end) * stride + c * 8, to + n * 1024);
    }
  };
  const int top_blk = last_split ? mx_own(a, it, row_base + 31 < Rh ? row_base + 31 : Rh - 1).i >> 5 : -1;
  // (block b is the way's whose number is W - 1 - b % W: at most one, where the tree has two)
  const int tree_first = W - 1 - way;
  const bool has_tree = active && small && tree_first <= top_blk;
  char* const tree_k = lds + MXA_WAVES * TILE + 2 * 32 * MX_Q_ROW<D> + (rb * 2 + (tree_first & 1)) * TILE;  // (behind Q)
  static_assert(MXA_WAVES * TILE + 2 * 32 * MX_Q_ROW<D> + 4 * TILE <= (int)sizeof(mem.tiles), "tree rows behind Q");
  if (has_tree) {
    request_tree(a.k_tree, a.k_stride, tree_first, tree_k);
    request_tree(a.v_tree, a.v_stride, tree_first, tile);
  }
  if (last_split && !small) mx_stage_tree(it, parents, par, hops);
  if (mine > 0) {
    request_k(0);
  }
  mx_meet();  // Q is there
  if (last_split && small) mx_small_paths(parents.a, it.M, own.i, path);

  MxState<D> st;
  st.clear();
  if (active) {
    bf16x8 qf[NK];  // element order of step kk as K's (see below)
#pragma unroll
    for (int kk = 0; kk < NK; ++kk)
      qf[kk] = *reinterpret_cast<const bf16x8*>(q_lds + col * MX_Q_ROW<D> + ((kk / SPC) * 2 * EPC + half * EPC + (kk % SPC) * 8) * 2);
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

    bool fresh = true;  // no scores yet
    auto step = [&](int j, auto first) {
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
      request_k(j + 1 < mine ? j + 1 : j);
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
      request_v();
      const int left = keys - (way + j * W) * 32;  // keys of this block
      if (left < 32) {
#pragma unroll
        for (int v = 0; v < 16; ++v) S[v] = 8 * (v >> 2) + 4 * half + (v & 3) < left ? S[v] : -HS_INF;
      }
      if constexpr (decltype(first)::value) {
        if (fresh) st.start(S, a.c2);
        else st.move(S, a.c2, HS_INF);
      }
      uint4 p0, p1;
      st.exp_half(S, a.c2, 0, p0, st.l);
      st.exp_half(S, a.c2, 1, p1, st.l);
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // the tile is read by other lanes than wrote it
      second(p0, p1);
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    };
    // ---- the tree's own rows, block by block (of large trees from the last that a row of this wave can see to the first), dealt to the
    // ways from the last one on, which has the fewest keys
    auto tree_block = [&](int b, unsigned word, floatx16 S) {
      const int last = it.M - 1 - 32 * b;  // >= 0
      const int ln = lane;
      const bf16_t* const vb = static_cast<const bf16_t*>(a.v_tree) + (int64_t)(it.n0 + 32 * b) * a.v_stride + it.g * D;
      ushort2v most = {0, 0};
#pragma unroll
      for (int n = 0; n < TC; ++n) note_bits(most, *reinterpret_cast<const uint4*>(tile + n * 1024 + ln * 16));
      const bool odd = __ballot(has_odd(most)) != 0ull;
      if (odd)
        for (int n = 0; n < TC; ++n) {
          const int id = n * 64 + ln;
          uint4* const at = reinterpret_cast<uint4*>(tile + id * 16);
          *at = without_odd(*at);
        }
#pragma unroll
      for (int v = 0; v < 16; ++v) S[v] = (word >> (8 * (v >> 2) + 4 * half + (v & 3))) & 1u ? S[v] : -HS_INF;
      uint4 p0, p1;
      if (fresh) st.start(S, a.c2);
      fresh = false;
      st.softmax(S, a.c2, p0, p1);
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      second(p0, p1);
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      if (odd) st.add_odd(vb, a.v_stride, last < 31 ? last + 1 : 32, word, half);
    };
    // (piece of a K row that step kk multiplies, and the step, are those of the cache's keys)
    auto piece = [&](int kk) { return (kk / SPC) * 2 * SPC + half * SPC + kk % SPC; };
    if (has_tree) {
      const unsigned word = tree_first == 0 ? path.lo : path.hi;
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // the tree's rows are there
      if (__ballot(word != 0u) != 0ull) {
        floatx16 S = zero;
#pragma unroll
        for (int kk = 0; kk < NK; ++kk)
          S = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const bf16x8*>(tree_k + v_at<D>(col, piece(kk))), qf[kk], S, 0, 0, 0);
        tree_block(tree_first, word, S);
      }
    } else if (!small) {
      for (int b = top_blk; b >= 0; --b) {
        const unsigned word = mx_path_word(false, hops, path, b);
        if (W - 1 - b % W != way || __ballot(word != 0u) == 0ull) continue;
        request_tree(a.v_tree, a.v_stride, b, tile);
        const int end = it.M - 1 - 32 * b;
        int ln = lane;
        asm volatile("" : "+v"(ln));
        const int lc = ln & 31, lh = ln >> 5;
        const bf16_t* const kp = static_cast<const bf16_t*>(a.k_tree) + (int64_t)(it.n0 + 32 * b + (lc < end ? lc : end)) * a.k_stride + it.g * D;
        floatx16 S = zero;
#pragma unroll
        for (int kk = 0; kk < NK; ++kk) {
          const uint4 f = *reinterpret_cast<const uint4*>(kp + 8 * ((kk / SPC) * 2 * SPC + lh * SPC + kk % SPC));
          S = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, f), qf[kk], S, 0, 0, 0);
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // V is there
        tree_block(b, word, S);
      }
    }
    if (mine > 0) request_v();
    if (mine > 0) step(0, std::true_type{});
    for (int j = 1; j < mine;) {
      if (j > 1) page_of = pages_from(page_j = j);
      for (const int stop = page_j + 63; j < mine && j < stop; ++j) step(j, std::false_type{});  // (the last one requests page_j + 63)
    }
  }
  const float sum = half_sum(st.l);
  st.note_lost(false, sum, wave, lane, mem.lost);  // (an inactive wave has zeros)
  if (half == 0) {
    den[wave][0][col] = st.m;
    den[wave][1][col] = sum;
  }
  mx_meet();  // every wave has its sums (and no tile is read any more)
  const bool held = mx_none_lost<D>(mem);

  // ---- the ways of a row block meet: each leaves its accumulators, scaled to the common maximum, and adds up its share
  // of the columns
  float top = MXA_FLOOR, total = 0.f;
  if (active) {
#pragma unroll
    for (int x = 0; x < W; ++x) top = fmaxf(top, den[x * R + rb][0][col]);
#pragma unroll
    for (int x = 0; x < W; ++x) total += den[x * R + rb][1][col] * exp2_fast(den[x * R + rb][0][col] - top);
    const float mine = exp2_fast(st.m - top) * mx_inverse(total, it.n_sp == 1);
    float4* const to = reinterpret_cast<float4*>(lds) + wave * (NT * 4 * 64) + lane;
    if (row_base + col < Rh)
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int b = 0; b < 4; ++b)
        to[(t * 4 + b) * 64] = make_float4(st.acc[t][4 * b] * mine, st.acc[t][4 * b + 1] * mine, st.acc[t][4 * b + 2] * mine, st.acc[t][4 * b + 3] * mine);
  }
  mx_meet();
  if (!active || row_base + col >= Rh) return held;
  const int64_t out_row = (int64_t)(it.n0 + own.i) * a.Hq + own.h;
  float* const rec = a.part + (it.rec0 + ((int64_t)own.i * a.Hq + own.h) * it.n_sp + it.sp) * (D + ATTN_REC_PAD);
  for (int x = way; x < NT * 4; x += W) {
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int y = 0; y < W; ++y) {
      const float4 f = reinterpret_cast<const float4*>(lds)[(y * R + rb) * (NT * 4 * 64) + x * 64 + lane];
      sum.x += f.x, sum.y += f.y, sum.z += f.z, sum.w += f.w;
    }
    mx_write4(a, it.n_sp == 1, out_row, rec, 8 * x + 4 * half, sum);  // (column 32 (x / 4) + 8 (x % 4) + 4 half)
  }
  if (way == 0 && half == 0) {
    if (it.n_sp == 1) {
      if (a.lse != nullptr) a.lse[out_row] = (top + __log2f(total)) * MXA_LN2;
    } else {
      rec[D] = top;
      rec[D + 1] = total;
    }
  }
  return held;
}

}  // namespace hs
