// Attention over a quantised cache, work items of three to eight row blocks: the waves share the keys (internal).
//
// A tile of 64 keys is read and converted to bfloat16 once, by all waves together, into LDS, where each wave fetches its
// fragments.  Every wave has a row block of 32; with W = 2 two waves share a block, each with one 32-key block of every tile.
//
// A tile passes through four stages: its codes are on their way into registers (three tiles ahead), they are converted and
// written to one of three LDS buffers while the tile before is being multiplied, a barrier, and its two 32-key blocks are
// multiplied.  A block's steps are two windows of matrix instructions, its scores and its second product, and each
// window also takes half of a block's exponentials, of the block whose scores are there already, so that the matrix and the
// vector pipes of a wave have independent work:
//     scores of the second block of t    | exponentials of the first block, second half | tile t + 1 is converted
//     product of the first block of t    | of the second block, first half
//     barrier (tile t + 1 is there)
//     scores of the first block of t + 1 | of the second block of t, second half
//     product of the second block of t   | of the first block of t + 1, first half
// (W = 2: one block a tile, two windows.)  The tree's own rows before, and the partial page behind them, go through the
// same buffers without that overlap: they are a few tiles.
//
// A row's maximum stays that of the tree's rows and its first 32 keys, as in the other kind.
#pragma once
#include <type_traits>

#include "attn_mx.h"

namespace hs {

// Returns whether all rows' sums stayed in range (mem.lost: which did not); rows that did not are written, but wrong.
template <int FMT, int D, int W>
__device__ __forceinline__ bool attn_mx_shared(const MxAttnArgs& a, const MxItem& it, MxLds<D>& mem) {
  constexpr int NK = D / 16, NT = D / 32, STEPS = NK / 2, EPS = 4 / STEPS;
  constexpr int ROW = mx_row_bytes(FMT, D);
  constexpr int SPC = 16 / Mx<FMT>::BITS;      // 16-byte pieces of bfloat16 that a 16-byte chunk of codes becomes
  constexpr int CPR = ROW / 16;                // chunks of a row
  constexpr int CH = MX_PAGE * CPR;            // chunks of a tile of K (or V)
  constexpr bool BOTH = CH == MXA_THREADS;     // a thread has a chunk of K and one of V; otherwise one of either
  constexpr int NS = D / MX_BLOCK;
  constexpr int EPC = 128 / Mx<FMT>::BITS;
  constexpr int KR = mxs_k_row(D), VR = mxs_v_row(D);
  constexpr int KT = MX_PAGE * KR, VT = MX_PAGE * VR, KB = KT / 2, VB = VT / 2;  // a buffer, and a 32-key block of it
  constexpr int BLOCKS = MXA_WAVES / W;        // row blocks of a workgroup
  char* const lds = mem.tiles;
  auto& den = mem.den;
  int* const par = mem.par;
  int2* const hops = mem.hops;
  int& odd_lds = mem.odd;
  char* const lds_k = lds;
  char* const lds_v = lds + MXS_BUF * KT;

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 31, half = lane >> 5;
  const int rb = wave % BLOCKS, way = wave / BLOCKS;
  const int Rh = a.G * it.M;
  const int row_base = (it.blk0 + rb) * 32;
  const bool active = rb < it.blk_n;
  // (the lane's row is found again where it is needed, which the empty statement keeps the compiler from doing once ahead of
  // the loops, where there are no registers to keep it in)
  auto own = [&]() {
    int c = col;
    asm volatile("" : "+v"(c));
    return mx_own(a, it, row_base + c < Rh ? row_base + c : Rh - 1);  // (rows behind the last repeat it)
  };
  const bool last_split = it.sp == it.n_sp - 1;
  const int k_lo = it.sp * it.pages * MX_PAGE, k_hi = last_split || k_lo + it.pages * MX_PAGE > it.L ? it.L : k_lo + it.pages * MX_PAGE;
  const int keys = k_hi > k_lo ? k_hi - k_lo : 0;  // of the prefix part
  const int n_full = keys / MX_PAGE;

  // ---- a thread's part of a tile of codes
  const int32_t* const table = a.pool.table + (int64_t)it.s * a.pool.max_blocks + (k_lo >> 6);
  const bool is_v = !BOTH && wave >= MXA_WAVES / 2;
  const int chunk = BOTH ? tid : tid & (MXA_THREADS / 2 - 1);
  const bool moves = chunk < CH;               // (half of the threads of a 2 KB tile have nothing)
  const int c_row = moves ? chunk / CPR : 0, c_at = moves ? chunk % CPR : 0;
  const int code_off = c_row * ROW + c_at * 16, scale_off = c_row * NS + c_at * EPC / MX_BLOCK;
  const unsigned char* const my_codes = is_v ? a.pool.v_codes : a.pool.k_codes;
  const unsigned char* const my_scales = is_v ? a.pool.v_scales : a.pool.k_scales;
  struct Raw {
    uint4 k, v;
    unsigned ks, vs;
  };
  auto pages_from = [&](int t) {  // lane l: the page of tile t + l
    const int p = keys > 0 ? table[(t + lane) * MX_PAGE < keys ? t + lane : t] : 0;
    return p < 0 || p >= a.pool.n_pages ? 0 : p;  // (a page outside the pool would be a caller's error)
  };
  int page_of = pages_from(0), page_base = 0;  // (moved on outside of the loop over the tiles: see every_tile)
  auto page_at = [&](int t) { return __builtin_amdgcn_readlane(page_of, t - page_base); };
  auto load = [&](int t, int rows, Raw& r) {  // (rows behind the last repeat it; they are masked)
    const int64_t base = ((int64_t)page_at(t) * a.pool.Hkv + it.g) * MX_PAGE;
    const unsigned back = c_row < rows ? 0u : (unsigned)(c_row - (rows - 1));
    const unsigned co = (unsigned)code_off - back * ROW, so = (unsigned)scale_off - back * NS;  // (a scalar base and a lane's 32 bits)
    // (the statements keep the page's address in scalar registers: added to a lane's address ahead of the loop it takes
    // two registers to a tensor)
    mx_mem kc = (mx_mem)(my_codes + base * ROW), ks = (mx_mem)(my_scales + base * NS);
    asm volatile("" : "+s"(kc), "+s"(ks));
    r.k = mx_load16(kc + co);
    r.ks = ks[so];
    if constexpr (BOTH) {
      mx_mem vc = (mx_mem)(a.pool.v_codes + base * ROW), vs = (mx_mem)(a.pool.v_scales + base * NS);
      asm volatile("" : "+s"(vc), "+s"(vs));
      r.v = mx_load16(vc + co);
      r.vs = vs[so];
    }
  };
  // piece e of a chunk as bfloat16 into its place of a buffer
  char* const my_k = lds_k + c_row * KR + c_at * SPC * 16;
  char* const my_v = lds_v + c_row * VR + c_at * SPC * 16;
  auto put = [&](const uint4& codes, unsigned byte, char* to, int e) {
    const unsigned w[4] = {codes.x, codes.y, codes.z, codes.w};
    *reinterpret_cast<uint4*>(to + 16 * e) =
        FMT == HS_MX_E4M3 ? mx_eight<FMT>(w[(2 * e) & 3], w[(2 * e + 1) & 3], mx_scale(byte)) : mx_eight<FMT>(w[e & 3], 0u, mx_scale(byte));
  };
  constexpr int PIECES = BOTH ? 2 * SPC : SPC;
  char* const my_one = is_v ? my_v : my_k;
  const int my_step = is_v ? VT : KT;
  auto put_piece = [&](const Raw& r, int slot, int x) {  // x: 0 .. PIECES - 1
    if constexpr (BOTH) {
      if (x >= SPC) put(r.v, r.vs, my_v + slot * VT, x - SPC);
      else put(r.k, r.ks, my_k + slot * KT, x);
    } else if (moves) {
      put(r.k, r.ks, my_one + slot * my_step, x);
    }
  };
  auto meet = [&]() { mx_meet(); };

  // ---- what the first steps wait for is requested first, all of it: the pages, the tree's parents and its last tile, Q, three
  // tiles of codes
  constexpr int PER = MX_PAGE * (D / 8) / MXA_THREADS;  // 16-byte pieces of K (and of V) of a tree tile to a thread
  static_assert(PER <= 2, "two pieces");
  const int row_last = (it.blk0 + it.blk_n) * 32 <= Rh ? (it.blk0 + it.blk_n) * 32 - 1 : Rh - 1;
  const int tree_top = last_split ? mx_own(a, it, row_last).i / MX_PAGE : -1;  // the last tile that a row of this workgroup sees
  uint4 k0, v0, k1, v1;  // (an array is given memory here, not registers)
  auto load_tree = [&](int t) {
    const int left = it.M - t * MX_PAGE;  // >= 1 rows of this tile exist; rows behind them repeat the last
    const bf16_t* const kb = static_cast<const bf16_t*>(a.k_tree) + (int64_t)(it.n0 + t * MX_PAGE) * a.k_stride + it.g * D;
    const bf16_t* const vb = static_cast<const bf16_t*>(a.v_tree) + (int64_t)(it.n0 + t * MX_PAGE) * a.v_stride + it.g * D;
    int x = tid;
    asm volatile("" : "+v"(x));  // (no address of these is kept in registers through the pages)
    auto one = [&](int id, uint4& k, uint4& v) {
      const int key = id / (D / 8), c = id % (D / 8), r = key < left ? key : left - 1;
      k = *reinterpret_cast<const uint4*>(kb + r * a.k_stride + 8 * c);
      v = *reinterpret_cast<const uint4*>(vb + r * a.v_stride + 8 * c);
    };
    one(x, k0, v0);
    if constexpr (PER == 2) one(x + MXA_THREADS, k1, v1);
  };
  MxParents parents = {};
  MxPath path = {0u, 0u, 0};
  const bool small = it.M <= 64;
  if (last_split) {
    parents = mx_request_parents(a, it);
    load_tree(tree_top);
  }
  // ---- Q (B operand): element 16 kk + 8 half + j of step kk; by way of the wave's part of the tile buffers
  char* const q_lds = lds + wave * 32 * MX_Q_ROW<D>;
  static_assert(MXA_WAVES * 32 * MX_Q_ROW<D> <= (int)sizeof(mem.tiles), "room for Q");
  if (active) mx_stage_q<D>(a, it, row_base, q_lds, lane, 64);
  bf16x8 qf[NK];
  if (last_split && !small) mx_stage_tree(it, parents, par, hops);
  if (tid == 0) odd_lds = 0;
  Raw ra, rb_, rc;
  if (n_full > 0) {
    load(0, MX_PAGE, ra);
    load(n_full > 1 ? 1 : 0, MX_PAGE, rb_);
    load(n_full > 2 ? 2 : n_full - 1, MX_PAGE, rc);
  }

  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
  for (int kk = 0; kk < NK; ++kk) qf[kk] = *reinterpret_cast<const bf16x8*>(q_lds + col * MX_Q_ROW<D> + 32 * kk + 16 * half);
  meet();  // (the buffers are free)
  MxState<D> st;
  st.clear();
  const float c2 = a.c2;
  const floatx16 zero = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};

  // ---- fragments: addresses of the first block of buffer 0
  const int tr_a = lane & 3, tr_j = (lane >> 2) & 3, tr_dh = (lane >> 4) & 1;
  // (W = 2: of the wave's own block, b is 0)
  const char* const kl = lds_k + (W == 2 ? way * KB : 0) + col * KR + half * 16;
  const char* const vl = lds_v + (W == 2 ? way * VB : 0) + (4 * half + tr_j) * VR + tr_dh * 32 + tr_a * 8;
  auto ldk = [&](int slot, int b, int kk) { return *reinterpret_cast<const bf16x8*>(kl + slot * KT + b * KB + kk * 32); };
  auto ldv = [&](int slot, int b, int f) {  // f = NT k2 + tt: keys 16 k2 .. of a block
    bf16x8 vf;
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const shortx4 got = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4_ptr)(vl + slot * VT + b * VB + (16 * (f / NT) + 8 * x) * VR + (f % NT) * 64));
      const bf16x4 four = __builtin_bit_cast(bf16x4, got);
#pragma unroll
      for (int e = 0; e < 4; ++e) vf[4 * x + e] = four[e];
    }
    return vf;
  };
  struct None {
    __device__ __forceinline__ void operator()(int) const {}
  };
  // Scores of block b of a buffer, with half h of S_in's exponentials and a step's share of `more`.
  auto win_qk = [&](int slot, int b, floatx16& S_out, const floatx16& S_in, int h, uint4& P, auto more) {
    unsigned w[4];
    bf16x8 f0 = ldk(slot, b, 0), f1 = ldk(slot, b, 1);
#pragma unroll
    for (int j = 0; j < STEPS; ++j) {
      bf16x8 n0 = f0, n1 = f1;
      if (j + 1 < STEPS) {
        n0 = ldk(slot, b, 2 * j + 2);
        n1 = ldk(slot, b, 2 * j + 3);
      }
      S_out = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f0, qf[2 * j], j == 0 ? zero : S_out, 0, 0, 0);
#pragma unroll
      for (int e = EPS * j; e < EPS * (j + 1); ++e) {
        const floatx2 p = st.exps(S_in, c2, 4 * h + e);
        st.l += p[0] + p[1];
        w[e] = __builtin_bit_cast(unsigned, __builtin_convertvector(p, bf16x2));
      }
      S_out = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f1, qf[2 * j + 1], S_out, 0, 0, 0);
      more(j);
      __builtin_amdgcn_sched_barrier(0);
      f0 = n0;
      f1 = n1;
    }
    P = make_uint4(w[0], w[1], w[2], w[3]);
  };
  // Product of block b of a buffer with P = (P0, P1); with EXP, half h of S_in's exponentials.
  auto win_pv = [&](int slot, int b, const uint4& P0, const uint4& P1, const floatx16& S_in, int h, uint4& P, auto with_exp) {
    constexpr bool EXP = decltype(with_exp)::value;
    const bf16x8 b0 = __builtin_bit_cast(bf16x8, P0), b1 = __builtin_bit_cast(bf16x8, P1);
    unsigned w[4];
    bf16x8 f0 = ldv(slot, b, 0), f1 = ldv(slot, b, 1);
#pragma unroll
    for (int j = 0; j < STEPS; ++j) {
      bf16x8 n0 = f0, n1 = f1;
      if (j + 1 < STEPS) {
        n0 = ldv(slot, b, 2 * j + 2);
        n1 = ldv(slot, b, 2 * j + 3);
      }
      st.acc[(2 * j) % NT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f0, 2 * j < NT ? b0 : b1, st.acc[(2 * j) % NT], 0, 0, 0);
      if (EXP) {
#pragma unroll
        for (int e = EPS * j; e < EPS * (j + 1); ++e) {
          const floatx2 p = st.exps(S_in, c2, 4 * h + e);
          st.l += p[0] + p[1];
          w[e] = __builtin_bit_cast(unsigned, __builtin_convertvector(p, bf16x2));
        }
      }
      st.acc[(2 * j + 1) % NT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f1, 2 * j + 1 < NT ? b0 : b1, st.acc[(2 * j + 1) % NT], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
      f0 = n0;
      f1 = n1;
    }
    if (EXP) P = make_uint4(w[0], w[1], w[2], w[3]);
  };
  const std::true_type YES{};
  const std::false_type NO{};
  auto scores = [&](int slot, int b) {
    floatx16 S = zero;
#pragma unroll
    for (int kk = 0; kk < NK; ++kk) S = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ldk(slot, b, kk), qf[kk], S, 0, 0, 0);
    return S;
  };

  // ---- the tree's own rows, the full pages, the partial page
  auto block = [&](int b, const floatx16& S) {
    const int slot = 0;
    uint4 p0, p1;
    st.softmax(S, c2, p0, p1);
    const bf16x8 b0 = __builtin_bit_cast(bf16x8, p0), b1 = __builtin_bit_cast(bf16x8, p1);
#pragma unroll
    for (int f = 0; f < NK; ++f) st.acc[f % NT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ldv(slot, b, f), f < NT ? b0 : b1, st.acc[f % NT], 0, 0, 0);
  };
  // Tile t + 1 of buffer S1 is converted from r, tile t + 4 requested into it (the last tile again behind the end).
  auto next_tile = [&](int t, Raw& r) { load(t + 4 < n_full ? t + 4 : n_full - 1, MX_PAGE, r); };
  auto convert = [&](const Raw& r, int slot, int j) {  // a step's share
#pragma unroll
    for (int x = 0; x < PIECES; ++x)
      if (x * STEPS / PIECES == j) put_piece(r, slot, x);
  };
  // f(t, buffer of t, registers of tile t + 1) for every full tile but the last
  auto every_tile = [&](auto f) {
    int t = 0;
    while (t + 3 < n_full) {
      // 57 tiles request up to the 62nd from here.  (With the look-up of the pages in the loop, under a branch, the waits for a tile
      // could not count the younger ones.)
      if (t > 0) page_of = pages_from(page_base = t);
      for (const int stop = t + 57; t + 3 < n_full && t < stop; t += 3) {  // (the buffers spelled out: every LDS address is a register plus an immediate)
        f(t, std::integral_constant<int, 0>{}, rb_);
        f(t + 1, std::integral_constant<int, 1>{}, rc);
        f(t + 2, std::integral_constant<int, 2>{}, ra);
      }
    }
    if (t + 1 < n_full) {
      f(t, std::integral_constant<int, 0>{}, rb_);
      if (++t + 1 < n_full) {
        f(t, std::integral_constant<int, 1>{}, rc);
        ++t;
      }
    }
    return t;
  };
  if (tree_top >= 0) {
    path.cur = own().i;
    if (small) mx_small_paths(parents.a, it.M, path.cur, path);
    bool fresh = true;
    for (int t = tree_top; t >= 0; --t) {  // (a small tree is one tile)
      const int left = it.M - t * MX_PAGE;
      ushort2v most = {0, 0};
      meet();  // (the buffer's last readers are done)
      int own_id = tid;
      asm volatile("" : "+v"(own_id));
      auto put_one = [&](int id, const uint4& k, const uint4& v) {
        const int key = id / (D / 8), c = id % (D / 8);
        note_bits(most, v);
        *reinterpret_cast<uint4*>(lds_k + key * KR + c * 16) = k;
        *reinterpret_cast<uint4*>(lds_v + key * VR + c * 16) = without_odd(v);
      };
      put_one(own_id, k0, v0);
      if constexpr (PER == 2) put_one(own_id + MXA_THREADS, k1, v1);
      if (has_odd(most)) odd_lds = 1;
      if (t > 0) load_tree(t - 1);
      meet();
      if (active) {
        for (int x = 0; x < 2; ++x) {
          const int b = small ? x : 1 - x;
          const unsigned word = mx_path_word(small, hops, path, 2 * t + b);
          if (W == 2 && b != way) continue;
          if (__ballot(word != 0u) == 0ull) continue;
          floatx16 S = scores(0, W == 2 ? 0 : b);
#pragma unroll
          for (int v = 0; v < 16; ++v) S[v] = (word >> (8 * (v >> 2) + 4 * half + (v & 3))) & 1u ? S[v] : -HS_INF;
          if (fresh) st.start(S, c2);
          fresh = false;
          block(W == 2 ? 0 : b, S);
          if (odd_lds != 0) {
            const bf16_t* const vb = static_cast<const bf16_t*>(a.v_tree) + (int64_t)(it.n0 + t * MX_PAGE + 32 * b) * a.v_stride + it.g * D;
            st.add_odd(vb, a.v_stride, left - 32 * b < 32 ? left - 32 * b : 32, word, half);
          }
        }
      }
    }
    meet();
  }
  if (n_full > 0) {
#pragma unroll
    for (int x = 0; x < PIECES; ++x) put_piece(ra, 0, x);
    load(n_full > 3 ? 3 : n_full - 1, MX_PAGE, ra);
    meet();
    if (active) {
      floatx16 sA, sB;
      uint4 pa, pb, pc;
      sA = scores(0, 0);
      st.move(sA, c2, HS_INF);  // the maximum of the whole pass over the full tiles
      st.exp_half(sA, c2, 0, pa, st.l);
      const int last = every_tile([&](int t, auto slot, Raw& r) {
        const int S0 = slot, S1 = (S0 + 1) % MXS_BUF;
        if constexpr (W == 1) {
          win_qk(S0, 1, sB, sA, 1, pb, [&](int j) { convert(r, S1, j); });
          next_tile(t, r);
          win_pv(S0, 0, pa, pb, sB, 0, pc, YES);
          meet();
          win_qk(S1, 0, sA, sB, 1, pb, None{});
          win_pv(S0, 1, pc, pb, sA, 0, pa, YES);
        } else {
#pragma unroll
          for (int j = 0; j < STEPS; ++j) convert(r, S1, j);
          next_tile(t, r);
          meet();
          win_qk(S1, 0, sB, sA, 1, pb, None{});
          win_pv(S0, 0, pa, pb, sB, 0, pc, YES);
          sA = sB;
          pa = pc;
        }
      });
      const int s0 = last % MXS_BUF;
      if constexpr (W == 1) {
        win_qk(s0, 1, sB, sA, 1, pb, None{});
        win_pv(s0, 0, pa, pb, sB, 0, pc, YES);
        st.exp_half(sB, c2, 1, pb, st.l);
        win_pv(s0, 1, pc, pb, sB, 0, pa, NO);
      } else {
        st.exp_half(sA, c2, 1, pb, st.l);
        win_pv(s0, 0, pa, pb, sA, 0, pc, NO);
      }
    } else {  // no rows: this wave only moves tiles
      every_tile([&](int t, auto slot, Raw& r) {
        const int S1 = (slot + 1) % MXS_BUF;
#pragma unroll
        for (int j = 0; j < STEPS; ++j) convert(r, S1, j);
        next_tile(t, r);
        meet();
      });
    }
  }
  // (before the partial page, which may move a maximum: scaled down, a sum that has left its range could pass for one within it)
  const bool over = st.l >= MX_LIMIT;
  if (keys > n_full * MX_PAGE) {
    const int rest = keys - n_full * MX_PAGE;
    load(n_full, rest, ra);
    meet();  // (the buffer's last readers are done)
#pragma unroll
    for (int x = 0; x < PIECES; ++x) put_piece(ra, 0, x);
    meet();
    if (active) {
      for (int b = 0; b < 2; ++b) {
        if (W == 2 ? b != way : false) continue;
        if (32 * b >= rest) continue;
        floatx16 S = scores(0, W == 2 ? 0 : b);
#pragma unroll
        for (int v = 0; v < 16; ++v) S[v] = 32 * b + 8 * (v >> 2) + 4 * half + (v & 3) < rest ? S[v] : -HS_INF;
        block(W == 2 ? 0 : b, S);
      }
    }
  }
  float top = st.m, total = half_sum(st.l);
  st.note_lost(over, total, wave, lane, mem.lost);
  st.l = total;
  meet();
  const bool held = mx_none_lost<D>(mem);

  // ---- out
  if constexpr (W == 2) {  // each way of a row block hands over the columns that the other one writes
    if (half == 0) {
      den[wave][0][col] = st.m;
      den[wave][1][col] = st.l;
    }
    meet();  // (no tile is read any more)
    const int other = wave ^ BLOCKS;
    const float m2 = den[other][0][col];
    top = fmaxf(st.m, m2);
    float mine = exp2_fast(st.m - top);
    total = st.l * mine + den[other][1][col] * exp2_fast(m2 - top);
    mine *= mx_inverse(total, it.n_sp == 1);
    floatx16 keep[NT / 2];
    float4* const to = reinterpret_cast<float4*>(lds) + wave * (NT / 2 * 4 * 64) + lane;
    const float4* const from = reinterpret_cast<const float4*>(lds) + other * (NT / 2 * 4 * 64) + lane;
#pragma unroll
    for (int t = 0; t < NT / 2; ++t) {
      keep[t] = way == 0 ? st.acc[t] : st.acc[NT / 2 + t];
      const floatx16 give = way == 0 ? st.acc[NT / 2 + t] : st.acc[t];
#pragma unroll
      for (int b = 0; b < 4; ++b)
        to[(t * 4 + b) * 64] = make_float4(give[4 * b] * mine, give[4 * b + 1] * mine, give[4 * b + 2] * mine, give[4 * b + 3] * mine);
    }
    meet();
#pragma unroll
    for (int t = 0; t < NT / 2; ++t)
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        const float4 f = from[(t * 4 + b) * 64];
        keep[t][4 * b] = keep[t][4 * b] * mine + f.x, keep[t][4 * b + 1] = keep[t][4 * b + 1] * mine + f.y;
        keep[t][4 * b + 2] = keep[t][4 * b + 2] * mine + f.z, keep[t][4 * b + 3] = keep[t][4 * b + 3] * mine + f.w;
      }
    meet();
    if (!active) return held;
    mx_write_half<D>(a, it, row_base, way, keep, 1.f, q_lds, lane);
  } else {
    if (!active) return held;
    const float inv = mx_inverse(total, it.n_sp == 1);
    mx_write_half<D>(a, it, row_base, 0, st.acc, inv, q_lds, lane);
    mx_write_half<D>(a, it, row_base, 1, st.acc + NT / 2, inv, q_lds, lane);
  }
  if (row_base + col >= Rh || way != 0 || half != 0) return held;
  const MxOwn o = own();
  if (it.n_sp == 1) {
    if (a.lse != nullptr) a.lse[(int64_t)(it.n0 + o.i) * a.Hq + o.h] = (top + __log2f(total)) * MXA_LN2;
  } else {
    float* const rec = a.part + (it.rec0 + ((int64_t)o.i * a.Hq + o.h) * it.n_sp + it.sp) * (D + ATTN_REC_PAD);
    rec[D] = top;
    rec[D + 1] = total;
  }
  return held;
}

}  // namespace hs
