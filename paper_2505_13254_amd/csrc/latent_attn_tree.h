// Absorbed attention over latents on the matrix cores: layouts, and one 32-key tile's work (internal).
//
// bfloat16, R = 512, Dr = 64.  A token is 1152 bytes that are key and value at once: S^T = K Q^T, O^T += V^T P^T with V the first 512
// columns of K, by v_mfma_f32_32x32x16_bf16 (a lane has a query, its registers the keys or the columns: softmax reductions stay inside a
// lane and its other half, and P is born in the layout that the second product takes).
//
// A workgroup has four waves, one to a SIMD with all of its 512 registers: 32 queries a wave take 144 registers for Q and 256 for O.  Rows (a
// sequence's tree row and head) are dealt in groups of 128.  What a group's waves share depends on how many 32-row blocks it has:
//   RB = 4 (65 .. 128 rows)  a block each, every key; the scores of the next tile run beside the softmax of this one
//   RB = 2 (33 .. 64)        two waves a block, each with one half of every 64-key page
//   RB = 1 (up to 32)        four waves a block: a half of the page and a half of the columns (scores computed twice)
// The latter two are bound by the stream of pages, not by what the waves do.
//
// LDS: a ring of four 32-key tiles, which global_load_lds fills.  A tile lies as in memory, but for the order of the eight 16-byte chunks of every
// 128 bytes: with G the number of a 128-byte group from the page's start (row r, group k of it: 9 r + k), chunk c stands at c ^ f(G), f(G) = bits 1, 2, 3 of G
// as bits 2, 1, 0.  16 rows of one chunk (a K fragment's read) and four rows of 64 bytes (a transposing V read) then lie in
// different banks, and the source address of a lane is the same for every load of a wave.
#pragma once
#include "latent_attn.h"

namespace hs {

typedef __bf16 lt_bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 lt_bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 lt_bf16x2 __attribute__((ext_vector_type(2)));
typedef float lt_floatx16 __attribute__((ext_vector_type(16)));
typedef float lt_floatx2 __attribute__((ext_vector_type(2)));
typedef short lt_shortx4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) lt_shortx4* lt_lds_s4;
typedef unsigned short lt_ushort2 __attribute__((ext_vector_type(2)));

constexpr int LT_THREADS = 256;
constexpr int LT_R = 512, LT_DR = 64;
constexpr int LT_ROW = 2 * (LT_R + LT_DR);
constexpr int LT_TILE = 32 * LT_ROW, LT_PAGE = 64 * LT_ROW;
constexpr int LT_LOADS = LT_TILE / 1024 / 4;  // to a wave, for a tile
constexpr int LT_GROUP = 128;                 // rows of a work item
constexpr int LT_NK = (LT_R + LT_DR) / 16;    // steps of the first product
constexpr int LT_MAX_TREE = 1024;
constexpr float LT_FLOOR = -3e38f;
constexpr float LT_RISE = 24.f;               // octaves that a score may rise above the reference
constexpr float LT_LN2 = 0.6931471805599453f, LT_LOG2E = 1.4426950408889634f;

__host__ __device__ __forceinline__ unsigned lt_key(unsigned G) { return ((G >> 1) & 1) << 2 | ((G >> 2) & 1) << 1 | ((G >> 3) & 1); }
// Byte of 16-byte chunk c (0 .. 71) of row r of a page.
__device__ __forceinline__ unsigned lt_at(unsigned r, unsigned c) {
  const unsigned G = 9 * r + (c >> 3);
  return G * 128 + 16 * ((c & 7) ^ lt_key(G));
}

__device__ __forceinline__ float2 lt_halves(float x) {  // this lane's value in the lower and in the upper half-wave
  const unsigned u = __builtin_bit_cast(unsigned, x);
  const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  const unsigned lo = r[0], hi = r[1];
  return make_float2(__builtin_bit_cast(float, lo), __builtin_bit_cast(float, hi));
}
__device__ __forceinline__ float lt_half_max(float x) {
  const float2 h = lt_halves(x);
  return fmaxf(h.x, h.y);
}
__device__ __forceinline__ float lt_half_sum(float x) {
  const float2 h = lt_halves(x);
  return h.x + h.y;
}

__device__ __forceinline__ void lt_meet() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// A wave's nine loads of a tile (1 KB each, every fourth of its 36): from `from` (the tile, uniform) + `off` (the lane's place, see the head of
// this file) to `to`, both moved to the wave's first load.  The caller waits for them with vmcnt.
// once: nobody else reads the pages.  The loads then carry the non-temporal hint.
__device__ __forceinline__ void lt_fetch(const char* from, unsigned off, unsigned to, bool once) {
  unsigned saved;
#define LT_LOAD(HINT) "global_load_lds_dwordx4 %1, %3" HINT "\n\t"
#define LT_NEXT(HINT) "s_add_u32 m0, m0, 0x1000\n\tv_add_u32 %1, 0x1000, %1\n\t" LT_LOAD(HINT)
#define LT_FETCH(HINT)                                                                                                                            \
  asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %2\n\ts_nop 0\n\t" LT_LOAD(HINT) LT_NEXT(HINT) LT_NEXT(HINT) LT_NEXT(HINT) LT_NEXT(HINT) LT_NEXT(HINT) \
                   LT_NEXT(HINT) LT_NEXT(HINT) LT_NEXT(HINT) "s_mov_b32 m0, %0"                                                                     \
               : "=&s"(saved), "+v"(off)                                                                                                          \
               : "s"(to), "s"(from)                                                                                                               \
               : "memory", "scc")
  if (once) LT_FETCH(" nt");
  else LT_FETCH("");
#undef LT_FETCH
#undef LT_NEXT
#undef LT_LOAD
}
static_assert(LT_LOADS == 9, "lt_fetch");
// 16 bytes of each lane's own address, lane l's to the wave's `to` + 16 l.
__device__ __forceinline__ void lt_fetch_one(const void* from, unsigned to) {
  unsigned saved;
  asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, off\n\ts_mov_b32 m0, %0" : "=&s"(saved) : "s"(to), "v"(from) : "memory");
}

// Step i of a score chain, in ordinary registers.  (As builtins the chain's results go to the accumulation registers, of which O takes all 256: sixteen of O's
// then live in memory, and a load from there waits for every tile on its way.)  Steps of one chain may follow each other at once; the last one waits until
// anything may read the result (twelve wait states behind a matrix instruction of eight passes), in the same statement.  (The two wait states ahead: k or q may come straight from a
// vector instruction.)
__device__ __forceinline__ void lt_step(lt_floatx16& S, const lt_bf16x8& k, const lt_bf16x8& q, int i) {
  if (i == 0) asm volatile("s_nop 1\n\tv_mfma_f32_32x32x16_bf16 %0, %1, %2, 0" : "=&v"(S) : "v"(k), "v"(q));
  else asm volatile("s_nop 1\n\tv_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+v"(S) : "v"(k), "v"(q));
}
__device__ __forceinline__ void lt_last(lt_floatx16& S, const lt_bf16x8& k, const lt_bf16x8& q) {
  asm volatile("s_nop 1\n\tv_mfma_f32_32x32x16_bf16 %0, %1, %2, %0\n\ts_nop 11" : "+v"(S) : "v"(k), "v"(q));
}
// 32 queries of a wave (col: the lane's), over NB blocks of 32 columns of the values from the wave's first one on.
template <int NB>
struct LtState {
  lt_bf16x8 q[LT_NK];  // element 16 i + 8 half + j of step i
  lt_floatx16 acc[NB]; // O^T: column 32 t + 8 (v / 4) + 4 half + v % 4
  float m, l, seen;    // reference of the scores (octaves), sum of the weights relative to it (of this half-wave's keys), largest score
  unsigned k_row, k_in;  // the first group of the lane's K row of a tile, and the byte of its chunk within a group
  unsigned v_row, v_in;  // of its V rows (the wave's first column on)

  __device__ __forceinline__ void clear(float reference) {
    m = seen = reference;
    l = 0.f;
#pragma unroll
    for (int t = 0; t < NB; ++t)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[t][v] = 0.f;
  }
  __device__ __forceinline__ void start(int lane, int first_block) {
    const unsigned half = lane >> 5, col = lane & 31;
    k_row = 9 * col;
    k_in = 16 * half;
    const unsigned a = lane & 3, j = (lane >> 2) & 3, dh = (lane >> 4) & 1, r0 = 4 * half + j;
    v_row = 9 * r0 + first_block / 2;
    v_in = 16 * (2 * dh + (a >> 1)) + 8 * (a & 1);
  }
  // The place of the lane's chunk in a group (found again for every tile: there are no registers to keep them in).
  __device__ __forceinline__ static unsigned place(unsigned G, unsigned in) { return (G << 7) + (in ^ (((__builtin_bitreverse32(G) >> 28) & 7u) << 4)); }
  // Chunk 2 i + half of the lane's K row; at: its place in group i / 4.
  __device__ __forceinline__ static lt_bf16x8 key(const char* lds, unsigned tile, unsigned at, int i) {
    return *reinterpret_cast<const lt_bf16x8*>(lds + ((at ^ (32u * (i & 3))) + tile));
  }
  // V^T of block t, keys 16 k2 .. of a tile.
  __device__ __forceinline__ lt_bf16x8 value(char* lds, unsigned tile, unsigned at, int t, int k2) const {
    lt_bf16x8 f;
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const lt_shortx4 got = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lt_lds_s4)(lds + ((at ^ (64u * (t & 1) | 16u * x)) + tile) + 9216 * x + 18432 * k2));
      const lt_bf16x4 four = __builtin_bit_cast(lt_bf16x4, got);
#pragma unroll
      for (int e = 0; e < 4; ++e) f[4 * x + e] = four[e];
    }
    return f;
  }
  __device__ __forceinline__ lt_floatx16 scores(const char* lds, unsigned tile) const {
    lt_floatx16 S;
    unsigned row = k_row, at;
    asm volatile("" : "+v"(row));
    constexpr int AHEAD = 4;
    lt_bf16x8 f[AHEAD];
    at = place(row, k_in);
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) f[i] = key(lds, tile, at, i);
#pragma unroll
    for (int i = 0; i < LT_NK; ++i) {
      if (i + 1 < LT_NK) lt_step(S, f[i % AHEAD], q[i], i);
      else lt_last(S, f[i % AHEAD], q[i]);
      const int n = i + AHEAD;
      if (n < LT_NK) {
        if ((n & 3) == 0) at = place(row + (n >> 2), k_in);
        f[i % AHEAD] = key(lds, tile, at, n);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    return S;
  }
  // A row's reference is the largest score of the first tile in which it sees a key, and stays: a weight may be as large as 2^LT_RISE.  `seen` is the
  // largest score so far; where it has risen further, the item is done again with it as the reference.
  __device__ __forceinline__ void refer(float top, float c2) {
    const float up = lt_half_max(top) * c2;
    seen = fmaxf(seen, up);
    m = m == LT_FLOOR ? seen : m;
  }
  __device__ __forceinline__ float top_of(const lt_floatx16& S) const {
    float top = fmaxf(S[0], S[1]);
#pragma unroll
    for (int v = 2; v < 16; ++v) top = fmaxf(top, S[v]);
    return top;
  }
  __device__ __forceinline__ unsigned pair(const lt_floatx16& S, float c2, int e) {  // weights 2 e, 2 e + 1
    const lt_floatx2 p = {exp2_fast(__builtin_fmaf(S[2 * e], c2, -m)), exp2_fast(__builtin_fmaf(S[2 * e + 1], c2, -m))};
    l += p[0] + p[1];
    return __builtin_bit_cast(unsigned, __builtin_convertvector(p, lt_bf16x2));
  }
  // A tile by itself: its scores (masked ones at -infinity) are S.
  __device__ __forceinline__ void take(char* lds, unsigned tile, const lt_floatx16& S, float c2) {
    refer(top_of(S), c2);
    uint4 P0, P1;
    P0.x = pair(S, c2, 0), P0.y = pair(S, c2, 1), P0.z = pair(S, c2, 2), P0.w = pair(S, c2, 3);
    P1.x = pair(S, c2, 4), P1.y = pair(S, c2, 5), P1.z = pair(S, c2, 6), P1.w = pair(S, c2, 7);
    product(lds, tile, P0, P1);
  }
  __device__ __forceinline__ void product(char* lds, unsigned tile, const uint4& P0, const uint4& P1) {
    const lt_bf16x8 b0 = __builtin_bit_cast(lt_bf16x8, P0), b1 = __builtin_bit_cast(lt_bf16x8, P1);
    // steps: pairs of blocks in one 128-byte group, the lower 16 keys of both, then the upper ones
    unsigned row = v_row;
    asm volatile("" : "+v"(row));
    lt_bf16x8 f[4];
    unsigned at = place(row, v_in);
#pragma unroll
    for (int x = 0; x < 4; ++x) f[x] = value(lds, tile, at, x & 1, x >> 1);
#pragma unroll
    for (int x = 0; x < 2 * NB; ++x) {
      const int t = 2 * (x >> 2) + (x & 1), k2 = (x >> 1) & 1;
      acc[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[x & 3], k2 == 0 ? b0 : b1, acc[t], 0, 0, 0);
      const int n = x + 4;
      if (n < 2 * NB) {
        if ((n & 3) == 0) at = place(row + (n >> 2), v_in);
        f[x & 3] = value(lds, tile, at, 2 * (n >> 2) + (n & 1), (n >> 1) & 1);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  // The scores of tile `next` beside the softmax of S (tile by tile, RB = 4), whose weights become P0, P1.
  __device__ __forceinline__ void ahead(const char* lds, unsigned next, const lt_floatx16& S, lt_floatx16& N, float c2, uint4& P0, uint4& P1) {
    constexpr int AHEAD = 4;
    unsigned row = k_row, at;
    asm volatile("" : "+v"(row));
    at = place(row, k_in);
    lt_bf16x8 f[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) f[i] = key(lds, next, at, i);
    float top = S[0];
    unsigned w[8];
#pragma unroll
    for (int i = 0; i < LT_NK; ++i) {
      if (i + 1 < LT_NK) lt_step(N, f[i % AHEAD], q[i], i);
      else lt_last(N, f[i % AHEAD], q[i]);
      const int n = i + AHEAD;
      if (n < LT_NK) {
        if ((n & 3) == 0) at = place(row + (n >> 2), k_in);
        f[i % AHEAD] = key(lds, next, at, n);
      }
      if (i < 5) {
#pragma unroll
        for (int v = 3 * i + 1; v < 3 * i + 4; ++v) top = fmaxf(top, S[v]);
      }
      if (i == 5) refer(top, c2);
      if (i >= 8 && i < 32 && (i - 8) % 3 == 0) w[(i - 8) / 3] = pair(S, c2, (i - 8) / 3);
      __builtin_amdgcn_sched_barrier(0);
    }
    P0 = make_uint4(w[0], w[1], w[2], w[3]);
    P1 = make_uint4(w[4], w[5], w[6], w[7]);
  }
};

}  // namespace hs
