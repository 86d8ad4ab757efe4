// Absorbed attention over latents on the matrix cores: layouts, and one 32-key tile's work (internal).
//
// bfloat16, R = 512, Dr = 64.  A token is 1152 bytes that are key and value at once: S^T = K Q^T, O^T += V^T P^T with V the first 512
// columns of K, by v_mfma_f32_32x32x16_bf16 (a lane has a query, its registers the keys or the columns: softmax reductions stay inside a
// lane and its other half, and P is born in the layout that the second product takes).
//
// A workgroup has four waves, one to a SIMD with all of its 512 registers: 32 queries a wave take 144 registers for Q and 256 for O.  Rows (a
// sequence's tree row and head) are dealt in groups of 128, or of 64 or 32 where a call has few items.  What a group's waves share depends on how many 32-row blocks it has:
//   RB = 4 (65 .. 128 rows)  a block each, every key; the scores of the next tile run beside the softmax of this one
//   RB = 2 (33 .. 64)        two waves a block, each with one half of every 64-key page
//   RB = 1 (up to 32)        four waves a block: a half of the page and a half of the columns (scores computed twice)
// The latter two are bound by the stream of pages, not by what the waves do.
// Measured: RB = 4, 4 x 97 rows of 64 heads on 8192 tokens, 1.06 to 1.1 PFLOP/s, the chip's power (a product of 8192^3 by the library: 1.22); RB = 1, 64 rows of
// 16 heads on 4451 pages, 5.1 TB/s over the whole call (a kernel that only reads: 6.4); one row of 16 heads on 2048 tokens 12 us, of which 4 until the last workgroup starts,
// 6 until Q and the first page are there, and 4 for two pages.
//
// LDS: a ring of four 32-key tiles, which global_load_lds fills.  A tile is its rows' latents, 1024 bytes each, and behind them their rotary parts, 128 bytes
// each.  16-byte chunk c of row r stands at c ^ lt_key(r) among a latent's, at c ^ (r / 2 mod 8) among a rotary part's: 16 rows of one chunk (a K fragment's
// read) and four rows of 64 bytes (a transposing V read) lie in different banks.  The key takes four bits, so that the place of every fragment is one of eight
// patterns, an exclusive or each, plus an immediate; fragments are taken pattern by pattern (the order of a product's steps is free).
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
constexpr float LT_FLOOR = -__FLT_MAX__;  // no score yet
constexpr float LT_RISE = 24.f;               // octaves that a weight may rise above the reference's
constexpr float LT_LN2 = 0.6931471805599453f, LT_LOG2E = 1.4426950408889634f;

constexpr int LT_ROT = 32 * 2 * LT_R;  // where a tile's rotary parts begin
__host__ __device__ __forceinline__ unsigned lt_key(unsigned r) { return (r & 3) << 2 | ((r >> 2) & 3); }
// Row and chunk (0 .. 71) of the 16 bytes at 16 * id of a page in the ring (two tiles).
__device__ __forceinline__ void lt_what(unsigned id, unsigned* row, unsigned* chunk) {
  const unsigned tile = id >= LT_TILE / 16 ? 1 : 0, x = id - tile * (LT_TILE / 16), y = x - LT_ROT / 16;
  const unsigned r = x < LT_ROT / 16 ? x >> 6 : y >> 3;
  *row = 32 * tile + r;
  *chunk = x < LT_ROT / 16 ? (x & 63) ^ lt_key(r) : 64 + ((y & 7) ^ ((r >> 1) & 7));
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

// A wave's nine loads of a tile, 1 KB each: the latents of rows w, w + 4, .. and the rotary parts of rows 8 w .. 8 w + 7 (w: the wave).  from: the tile's first
// row; off: the lane's place in row w (16 (lane ^ lt_key(w)) + 1152 w); rot: in the rotary parts of its row (lt_rot_off).  to, to_rot: the wave's first places
// in LDS.  The caller waits for them with vmcnt.  once: nobody else reads the pages.  The loads then carry the non-temporal hint.
__device__ __forceinline__ unsigned lt_rot_off(int lane, int wave) {
  const unsigned r = 8 * wave + (lane >> 3);
  return LT_ROW * r + 2 * LT_R + 16 * ((lane & 7) ^ ((r >> 1) & 7));
}
__device__ __forceinline__ void lt_fetch(const char* from, unsigned off, unsigned rot, unsigned to, unsigned to_rot, bool once) {
  unsigned saved;
#define LT_LOAD(HINT) "global_load_lds_dwordx4 %1, %3" HINT "\n\t"
#define LT_NEXT(KEY, HINT) "s_add_u32 m0, m0, 0x1000\n\tv_add_u32 %1, 0x1200, %1\n\tv_xor_b32 %1, " KEY ", %1\n\t" LT_LOAD(HINT)
#define LT_FETCH(HINT)                                                                                                                                       \
  asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %5\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %4, %3" HINT "\n\ts_mov_b32 m0, %2\n\ts_nop 0\n\t" LT_LOAD(HINT)        \
                   LT_NEXT("16", HINT) LT_NEXT("48", HINT) LT_NEXT("16", HINT) LT_NEXT("48", HINT) LT_NEXT("16", HINT) LT_NEXT("48", HINT) LT_NEXT("16", HINT) \
                       "s_mov_b32 m0, %0"                                                                                                                    \
               : "=&s"(saved), "+v"(off)                                                                                                                     \
               : "s"(to), "s"(from), "v"(rot), "s"(to_rot)                                                                                                   \
               : "memory", "scc")
  if (once) LT_FETCH(" nt");
  else LT_FETCH("");
#undef LT_FETCH
#undef LT_NEXT
#undef LT_LOAD
}
static_assert(LT_LOADS == 9, "lt_fetch");
// 16 bytes at `off` behind an address, lane l's to the wave's `to` + 16 l.
__device__ __forceinline__ void lt_fetch_row(const char* from, unsigned off, unsigned to) {
  unsigned saved;
  asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %3\n\ts_mov_b32 m0, %0" : "=&s"(saved) : "s"(to), "v"(off), "s"(from) : "memory");
}
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
  float m, l, seen;    // reference of the scores (products, not scaled yet), sum of the weights relative to it (of this half-wave's keys), largest score
  unsigned k_at, r_at, v_at;  // the lane's places in a tile: of its K row's first chunk, of its rotary part's, of its V rows' (the wave's first column on)

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
    k_at = 1024 * col + 16 * (half ^ lt_key(col));
    r_at = LT_ROT + 128 * col + 16 * (half ^ ((col >> 1) & 7));
    const unsigned a = lane & 3, j = (lane >> 2) & 3, dh = (lane >> 4) & 1, r0 = 4 * half + j;
    v_at = 1024 * r0 + 16 * ((2 * dh + (a >> 1)) ^ lt_key(r0)) + 8 * (a & 1) + 64 * first_block;
  }
  // Step n of the first product: chunks 2 i + half, i = step(n), of the lane's K row (the same i for n = 4 m .. 4 m + 3 but for multiples of eight).
  __device__ __forceinline__ static constexpr int step(int n) { return n < 32 ? 8 * (n & 3) + (n >> 2) : n; }
  struct Keys {
    const char* lds;
    unsigned k, r, at;
    __device__ __forceinline__ lt_bf16x8 operator()(int n) {
      if (n >= 32) at = r ^ (32u * (n - 32));
      else if ((n & 3) == 0) at = k ^ (32u * (n >> 2));
      return *reinterpret_cast<const lt_bf16x8*>(lds + at + (n < 32 ? 256 * (n & 3) : 0));
    }
  };
  __device__ __forceinline__ Keys keys(const char* lds, unsigned tile) const {
    Keys k = {lds, k_at + tile, r_at + tile, 0u};
    asm volatile("" : "+v"(k.k), "+v"(k.r));  // (found again for every tile: there are no registers to keep all patterns in)
    return k;
  }
  // Fragment x of the second product: block t = block(x) of the wave's columns, keys 16 k2 .. of a tile, k2 = (x / 2) % 2.
  __device__ __forceinline__ static constexpr int block(int x) { return 4 * (2 * ((x >> 2) % (NB / 8)) + (x & 1)) + (x >> 2) / (NB / 8); }
  struct Values {
    char* lds;
    unsigned v, at0, at1;
    __device__ __forceinline__ lt_bf16x8 operator()(int x) {
      const int t = block(x), k2 = (x >> 1) & 1;
      if (x % (NB / 2) == 0) at0 = v ^ (64u * (t & 3)), at1 = v ^ (64u * (t & 3) | 32u);
      lt_bf16x8 f;
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        const lt_shortx4 got = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lt_lds_s4)(lds + (y ? at1 : at0) + 256 * (t >> 2) + 8192 * y + 16384 * k2));
        const lt_bf16x4 four = __builtin_bit_cast(lt_bf16x4, got);
#pragma unroll
        for (int e = 0; e < 4; ++e) f[4 * y + e] = four[e];
      }
      return f;
    }
  };
  __device__ __forceinline__ lt_floatx16 scores(const char* lds, unsigned tile) const {
    lt_floatx16 S;
    constexpr int AHEAD = 4;
    Keys key = keys(lds, tile);
    lt_bf16x8 f[AHEAD];
#pragma unroll
    for (int n = 0; n < AHEAD; ++n) f[n] = key(n);
#pragma unroll
    for (int n = 0; n < LT_NK; ++n) {
      if (n + 1 < LT_NK) lt_step(S, f[n % AHEAD], q[step(n)], n);
      else lt_last(S, f[n % AHEAD], q[step(n)]);
      if (n + AHEAD < LT_NK) f[n % AHEAD] = key(n + AHEAD);
      __builtin_amdgcn_sched_barrier(0);
    }
    return S;
  }
  // A row's reference is the largest score of the first tile in which it sees a key, and stays: a weight may be as large as 2^LT_RISE.  `seen` is the
  // largest score so far; where it has risen further, the item is done again with it as the reference.
  __device__ __forceinline__ void refer(float top) {
    seen = fmaxf(seen, lt_half_max(top));
    m = m == LT_FLOOR ? seen : m;
  }
  __device__ __forceinline__ float top_of(const lt_floatx16& S) const {
    float top = fmaxf(S[0], S[1]);
#pragma unroll
    for (int v = 2; v < 16; ++v) top = fmaxf(top, S[v]);
    return top;
  }
  __device__ __forceinline__ bool rose(float c2) const { return (seen - m) * c2 > LT_RISE; }
  // Weights 2 e, 2 e + 1.  (The difference comes first, here and in the merges: of scores as large as 2^30 octaves a scaled reference is off by the rounding of a product, more
  // octaves than float32 has, and a fused multiplication would keep them: weights would be infinite, or all zero.  Still larger ones have no octaves in float32.)
  __device__ __forceinline__ unsigned pair(const lt_floatx16& S, float c2, int e) {
    const lt_floatx2 p = {exp2_fast((S[2 * e] - m) * c2), exp2_fast((S[2 * e + 1] - m) * c2)};
    l += p[0] + p[1];
    return __builtin_bit_cast(unsigned, __builtin_convertvector(p, lt_bf16x2));
  }
  // A tile by itself: its scores (masked ones at -infinity) are S.
  __device__ __forceinline__ void take(char* lds, unsigned tile, const lt_floatx16& S, float c2) {
    refer(top_of(S));
    uint4 P0, P1;
    P0.x = pair(S, c2, 0), P0.y = pair(S, c2, 1), P0.z = pair(S, c2, 2), P0.w = pair(S, c2, 3);
    P1.x = pair(S, c2, 4), P1.y = pair(S, c2, 5), P1.z = pair(S, c2, 6), P1.w = pair(S, c2, 7);
    product(lds, tile, P0, P1);
  }
  __device__ __forceinline__ void product(char* lds, unsigned tile, const uint4& P0, const uint4& P1) {
    const lt_bf16x8 b0 = __builtin_bit_cast(lt_bf16x8, P0), b1 = __builtin_bit_cast(lt_bf16x8, P1);
    Values value = {lds, v_at + tile, 0u, 0u};
    asm volatile("" : "+v"(value.v));
    lt_bf16x8 f[4];
#pragma unroll
    for (int x = 0; x < 4; ++x) f[x] = value(x);
#pragma unroll
    for (int x = 0; x < 2 * NB; ++x) {
      acc[block(x)] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[x & 3], (x >> 1) & 1 ? b1 : b0, acc[block(x)], 0, 0, 0);
      if (x + 4 < 2 * NB) f[x & 3] = value(x + 4);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  // The scores of tile `next` beside the softmax of S (tile by tile, RB = 4), whose weights become P0, P1.
  __device__ __forceinline__ void ahead(const char* lds, unsigned next, const lt_floatx16& S, lt_floatx16& N, float c2, uint4& P0, uint4& P1) {
    constexpr int AHEAD = 4;
    Keys key = keys(lds, next);
    lt_bf16x8 f[AHEAD];
#pragma unroll
    for (int n = 0; n < AHEAD; ++n) f[n] = key(n);
    float top = S[0];
    unsigned w[8];
#pragma unroll
    for (int n = 0; n < LT_NK; ++n) {
      if (n + 1 < LT_NK) lt_step(N, f[n % AHEAD], q[step(n)], n);
      else lt_last(N, f[n % AHEAD], q[step(n)]);
      if (n + AHEAD < LT_NK) f[n % AHEAD] = key(n + AHEAD);
      if (n < 5) {
#pragma unroll
        for (int v = 3 * n + 1; v < 3 * n + 4; ++v) top = fmaxf(top, S[v]);
      }
      if (n == 5) refer(top);
      if (n >= 8 && n < 32 && (n - 8) % 3 == 0) w[(n - 8) / 3] = pair(S, c2, (n - 8) / 3);
      __builtin_amdgcn_sched_barrier(0);
    }
    P0 = make_uint4(w[0], w[1], w[2], w[3]);
    P1 = make_uint4(w[4], w[5], w[6], w[7]);
  }
};

}  // namespace hs
