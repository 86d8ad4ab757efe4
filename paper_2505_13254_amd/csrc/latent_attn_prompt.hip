// Expanded latent attention of prompt rows on the matrix cores: bfloat16, Dn = 128, Dr = 64, Dv = 128.
//
// A work item is up to 256 (or 128) rows of one (sequence, head) and one split of the keys that they see: eight waves of 32 rows each share tiles of 64 keys, which
// global_load_lds brings into a ring of three.  The products are those of the absorbed form (S^T = K Q^T, O^T += V^T P^T, a lane has a query) on keys of
// 192 and values of 128 elements; the scores of a 32-key block run beside the softmax of the block before it, and two waves to a SIMD fill each
// other's waits.  Tiles that some row sees only part of (its own last keys, causally: five tiles at most but for sequences with fewer keys than rows) are
// masked, and the elements of their values that are no numbers made zero by the wave that fetched them.
//
// LDS: a tile is 64 rows of keys (256 bytes), 64 of rotary parts (128) and 64 of values (256); 16-byte chunk c of row r stands at c ^ lt_key(r) (keys, values)
// or c ^ (r / 2 mod 8), so that fragments' reads fall into different banks.
// Bound by the matrix cores and the chip's power: 8192 rows of 32 heads, 1.02 to 1.08 PFLOP/s.  Short calls are bound by an item's start and end, 6 us.
// Heads are the fastest index of the items: with a multiple of eight of them, the groups of a head are on one XCD and find its keys in that L2.
#include <algorithm>

#include "latent_attn_tree.h"

namespace hs {

constexpr int LP_THREADS = 512, LP_WAVES = 8;
constexpr int LP_DN = 128, LP_DR = 64, LP_DV = 128;
constexpr int LP_GROUP = 256;                    // rows of an item at most
constexpr int LP_ROT = 64 * 2 * LP_DN, LP_VAL = LP_ROT + 64 * 2 * LP_DR, LP_TILE = LP_VAL + 64 * 2 * LP_DV;
constexpr int LP_RING = 3;
constexpr int LP_LOADS = LP_TILE / 1024 / LP_WAVES;  // to a wave, for a tile
static_assert(LP_LOADS == 5, "two of keys, one of rotary parts, two of values");
constexpr int LP_NK = (LP_DN + LP_DR) / 16, LP_NB = LP_DV / 32;
constexpr int LP_REC = LP_DV + ATTN_REC_PAD;
constexpr int LP_OUT_PITCH = 256 + 16;

struct LpArgs {
  LatPromptArgs a;
  float c2;
  int per;     // tiles of a split at most
  int sp_max;
  int group;   // rows of an item at most: 256, or 128 (four waves only move tiles)
  float* part;
  int records;  // that part holds
  int one_len;  // B == 1: the keys (its rows are N)
};

struct LpLds {
  char ring[LP_RING * LP_TILE];
  int64_t out_at[LP_WAVES][32];
  unsigned odd[4][2];  // of the masked tiles: which of their 64 values hold a NaN or an infinity
  int again, found[5];
  int64_t found_wide[2];
  int sums[LP_WAVES][2];
};
static_assert(sizeof(LpLds) <= 160 * 1024 && LP_WAVES * 32 * LP_OUT_PITCH <= LP_RING * LP_TILE, "LDS of a compute unit");

// Groups of n rows where they have `group` at most, their size (equal ones, whole blocks of 32), tiles of `keys` keys, splits of a sequence.
__host__ __device__ __forceinline__ int lp_groups(int n, int group) { return (n + group - 1) / group; }
__host__ __device__ __forceinline__ int lp_size(int n, int group) {
  const int all = 32 * lp_groups(n, group);
  return n <= 0 ? 32 : 32 * ((n + all - 1) / all);
}
__host__ __device__ __forceinline__ int lp_splits(int64_t keys, int per) {
  const int64_t tiles = (keys + 63) >> 6;
  return tiles <= per ? 1 : (int)((tiles + per - 1) / per);
}

struct LpItem {
  int s, n0, n, h, g, sp, n_sp;
  int rec0;  // the sequence's first record
  int64_t k0, T;
};

// What the device's arrays say of sequence s, within what the host's copies said.
__device__ __forceinline__ void lp_sequence(const LpArgs& gl, int s, int* n0, int* n, int64_t* k0, int64_t* T, int* n_sp) {
  const LatPromptArgs& a = gl.a;
  if (a.B == 1) {  // (no trip to memory)
    *n0 = 0, *k0 = 0;
    *n = a.N, *T = gl.one_len;
    *n_sp = lp_splits(*T, gl.per);
    return;
  }
  const int from = a.q_offsets[s], to = a.q_offsets[s + 1];
  *k0 = a.kv_offsets[s];
  const int64_t keys = a.kv_offsets[s + 1] - *k0;
  *T = keys < 0 ? 0 : std::min(keys, (int64_t)HS_MX_MAX_TOKENS);
  *n0 = from;
  const int rows = from < 0 ? 0 : std::min(to - from, a.N - from);
  *n = rows < 0 ? 0 : rows;
  *n_sp = std::min(lp_splits(*T, gl.per), gl.sp_max);
}
__device__ __forceinline__ int lp_records(int n, int H, int n_sp) { return n_sp > 1 ? n * H * n_sp : 0; }

__device__ __forceinline__ bool lp_find(const LpArgs& gl, LpItem& it, LpLds& mem) {
  const LatPromptArgs& a = gl.a;
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int item = blockIdx.x;  // (fewer than 2^22)
  auto place = [&](int at) {
    it.n_sp = std::min(lp_splits(it.T, gl.per), gl.sp_max);
    const int x = at / a.H;
    it.h = at - x * a.H;
    const int g = x / it.n_sp;
    it.sp = x - g * it.n_sp;
    it.g = lp_groups(it.n, gl.group) - 1 - g;  // (the longest first)
  };
  if (a.B == 1) {
    it.s = it.rec0 = 0;
    lp_sequence(gl, 0, &it.n0, &it.n, &it.k0, &it.T, &it.n_sp);
    place(item);
    return true;
  }
  if (tid == 0) mem.found[0] = -1;
  int items = 0, records = 0;
  for (int base = 0; base < a.B && items <= item; base += LP_THREADS) {
    const int s = base + tid;
    int n0 = 0, n = 0, n_sp = 1;
    int64_t k0 = 0, T = 0;
    if (s < a.B) lp_sequence(gl, s, &n0, &n, &k0, &T, &n_sp);
    const int mine = lp_groups(n, gl.group) * n_sp * a.H, recs = lp_records(n, a.H, n_sp);
    int to = wave_prefix_sum(mine), rec_to = wave_prefix_sum(recs);
    if (lane == 63) mem.sums[wave][0] = to, mem.sums[wave][1] = rec_to;
    __syncthreads();
    int all = 0, all_recs = 0;
    for (int w = 0; w < LP_WAVES; ++w) {
      if (w == wave) to += all, rec_to += all_recs;
      all += mem.sums[w][0];
      all_recs += mem.sums[w][1];
    }
    const int at = item - (items + to - mine);
    if (at >= 0 && at < mine) {
      mem.found[0] = s;
      mem.found[1] = n0;
      mem.found[2] = n;
      mem.found[3] = at;
      mem.found[4] = records + rec_to - recs;
      mem.found_wide[0] = k0;
      mem.found_wide[1] = T;
    }
    items += all;
    records += all_recs;
    __syncthreads();
  }
  auto get = [&](int v) { return __builtin_amdgcn_readfirstlane(v); };
  it.s = get(mem.found[0]);
  if (it.s < 0) return false;
  it.n0 = get(mem.found[1]);
  it.n = get(mem.found[2]);
  auto wide = [&](int64_t v) { return (int64_t)(uint32_t)get((int)v) | (int64_t)get((int)(v >> 32)) << 32; };
  it.k0 = wide(mem.found_wide[0]);
  it.T = wide(mem.found_wide[1]);
  place(get(mem.found[3]));
  it.rec0 = get(mem.found[4]);
  return it.n_sp == 1 || it.rec0 + lp_records(it.n, a.H, it.n_sp) <= gl.records;  // (always, where the arrays are as the host's copies)
}

struct LpState {
  lt_bf16x8 q[LP_NK];
  lt_floatx16 acc[LP_NB];
  float m, l, seen;
  unsigned k_at, r_at, v_at;

  __device__ __forceinline__ void start(int lane) {
    const unsigned half = lane >> 5, col = lane & 31;
    k_at = 256 * col + 16 * (half ^ lt_key(col));
    r_at = LP_ROT + 128 * col + 16 * (half ^ ((col >> 1) & 7));
    const unsigned a = lane & 3, j = (lane >> 2) & 3, dh = (lane >> 4) & 1, r0 = 4 * half + j;
    v_at = LP_VAL + 256 * r0 + 16 * ((2 * dh + (a >> 1)) ^ lt_key(r0)) + 8 * (a & 1);
  }
  __device__ __forceinline__ void clear(float reference) {
    m = seen = reference;
    l = 0.f;
#pragma unroll
    for (int t = 0; t < LP_NB; ++t)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[t][v] = 0.f;
  }
  // K fragment n of 32-key block b of the tile at `tile`.
  __device__ __forceinline__ lt_bf16x8 key(const char* lds, unsigned tile, int b, int n) const {
    const unsigned at = n < 8 ? (k_at ^ (32u * n)) + 8192u * b : (r_at ^ (32u * (n - 8))) + 4096u * b;
    return *reinterpret_cast<const lt_bf16x8*>(lds + tile + at);
  }
  // V^T fragment x of block b: block x / 2 of 32 columns, keys 16 (x % 2) .. .
  __device__ __forceinline__ lt_bf16x8 value(char* lds, unsigned tile, int b, int x) const {
    lt_bf16x8 f;
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      const lt_shortx4 got =
          __builtin_amdgcn_ds_read_tr16_b64_v4i16((lt_lds_s4)(lds + tile + (v_at ^ (64u * (x >> 1) | 32u * y)) + 8192 * b + 4096 * (x & 1) + 2048 * y));
      const lt_bf16x4 four = __builtin_bit_cast(lt_bf16x4, got);
#pragma unroll
      for (int e = 0; e < 4; ++e) f[4 * y + e] = four[e];
    }
    return f;
  }
  __device__ __forceinline__ void refer(float top) {  // (this and the next two as LtState's)
    seen = fmaxf(seen, lt_half_max(top));
    m = m == LT_FLOOR ? seen : m;
  }
  __device__ __forceinline__ bool rose(float c2) const { return (seen - m) * c2 > LT_RISE; }
  __device__ __forceinline__ unsigned pair(const lt_floatx16& S, float c2, int e) {
    const lt_floatx2 p = {exp2_fast((S[2 * e] - m) * c2), exp2_fast((S[2 * e + 1] - m) * c2)};
    l += p[0] + p[1];
    return __builtin_bit_cast(unsigned, __builtin_convertvector(p, lt_bf16x2));
  }
  __device__ __forceinline__ static lt_floatx16 zero() { return lt_floatx16{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}; }
  __device__ __forceinline__ lt_floatx16 scores(const char* lds, unsigned tile, int b) const {
    lt_floatx16 S;
    constexpr int AHEAD = 4;
    lt_bf16x8 f[AHEAD];
#pragma unroll
    for (int n = 0; n < AHEAD; ++n) f[n] = key(lds, tile, b, n);
#pragma unroll
    for (int n = 0; n < LP_NK; ++n) {
      S = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[n % AHEAD], q[n], n == 0 ? zero() : S, 0, 0, 0);
      if (n + AHEAD < LP_NK) f[n % AHEAD] = key(lds, tile, b, n + AHEAD);
      __builtin_amdgcn_sched_barrier(0);
    }
    return S;
  }
  __device__ __forceinline__ void product(char* lds, unsigned tile, int b, const uint4& P0, const uint4& P1) {
    const lt_bf16x8 b0 = __builtin_bit_cast(lt_bf16x8, P0), b1 = __builtin_bit_cast(lt_bf16x8, P1);
    lt_bf16x8 f[4];
#pragma unroll
    for (int x = 0; x < 4; ++x) f[x] = value(lds, tile, b, x);
#pragma unroll
    for (int x = 0; x < 2 * LP_NB; ++x) {
      acc[x >> 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[x & 3], x & 1 ? b1 : b0, acc[x >> 1], 0, 0, 0);
      if (x + 4 < 2 * LP_NB) f[x & 3] = value(lds, tile, b, x + 4);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  __device__ __forceinline__ void take(char* lds, unsigned tile, int b, const lt_floatx16& S, float c2) {
    float top = fmaxf(S[0], S[1]);
#pragma unroll
    for (int v = 2; v < 16; ++v) top = fmaxf(top, S[v]);
    refer(top);
    uint4 P0, P1;
    P0.x = pair(S, c2, 0), P0.y = pair(S, c2, 1), P0.z = pair(S, c2, 2), P0.w = pair(S, c2, 3);
    P1.x = pair(S, c2, 4), P1.y = pair(S, c2, 5), P1.z = pair(S, c2, 6), P1.w = pair(S, c2, 7);
    product(lds, tile, b, P0, P1);
  }
  // The scores N of block b of the tile at `next` beside the softmax of S, whose weights become P0, P1.
  __device__ __forceinline__ void ahead(const char* lds, unsigned next, int b, const lt_floatx16& S, lt_floatx16& N, float c2, uint4& P0, uint4& P1) {
    constexpr int AHEAD = 4;
    lt_bf16x8 f[AHEAD];
#pragma unroll
    for (int n = 0; n < AHEAD; ++n) f[n] = key(lds, next, b, n);
    float top = S[0];
    unsigned w[8];
#pragma unroll
    for (int n = 0; n < LP_NK; ++n) {
      N = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[n % AHEAD], q[n], n == 0 ? zero() : N, 0, 0, 0);
      if (n + AHEAD < LP_NK) f[n % AHEAD] = key(lds, next, b, n + AHEAD);
      if (n < 3) {
#pragma unroll
        for (int v = 5 * n + 1; v < 5 * n + 6; ++v) top = fmaxf(top, S[v]);
      }
      if (n == 2) refer(top);
      if (n >= 3 && n < 11) w[n - 3] = pair(S, c2, n - 3);
      __builtin_amdgcn_sched_barrier(0);
    }
    P0 = make_uint4(w[0], w[1], w[2], w[3]);
    P1 = make_uint4(w[4], w[5], w[6], w[7]);
  }
};

__global__ __launch_bounds__(LP_THREADS) void k_lat_prompt(LpArgs gl) {
  __shared__ LpLds mem;
  const LatPromptArgs& a = gl.a;
  LpItem it;
  if (threadIdx.x < 8) mem.odd[threadIdx.x >> 1][threadIdx.x & 1] = 0u;
  if (!lp_find(gl, it, mem)) return;
  char* const lds = mem.ring;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 31, half = lane >> 5;
  const int size = lp_size(it.n, gl.group), first = it.g * size, rows = std::min(size, it.n - first);  // rows first .. first + rows - 1 of the sequence
  const int mine_rows = std::min(32, rows - 32 * wave);                                      // <= 0: none, the wave only moves tiles
  const int row = first + std::min(32 * wave + col, rows - 1);                               // (rows behind the last repeat it)
  // row i of the sequence sees T - n + i + 1 keys
  const int64_t T = it.T, shift = T - it.n + 1;
  const int64_t most = std::max<int64_t>(0, shift + first + rows - 1), least = std::max<int64_t>(0, shift + first);
  const int tiles = (int)((most + 63) >> 6), whole = std::min(tiles, (int)(least >> 6));  // tiles that some row sees, tiles that every row sees whole
  const int t_lo = (int)((int64_t)it.sp * tiles / it.n_sp), t_hi = (int)((int64_t)(it.sp + 1) * tiles / it.n_sp);
  const int n_all = t_hi - t_lo, n_un = std::max(0, std::min(whole, t_hi) - t_lo);
  const int vis = (int)std::max<int64_t>(0, shift + row);  // keys that the lane's row sees

  // ---- a tile's five loads of a wave: 1 KB each of keys (rows 4 w ..), of keys (rows 32 + 4 w ..), rotary parts (rows 8 w ..), values like the keys
  const int64_t key0 = it.k0 + 64 * (int64_t)t_lo;
  const char* const k_base = static_cast<const char*>(a.k.p) + 2 * (key0 * a.k.row + it.h * a.k.head);
  const char* const v_base = static_cast<const char*>(a.v.p) + 2 * (key0 * a.v.row + it.h * a.v.head);
  const char* const r_base = static_cast<const char*>(a.k_rope) + 2 * key0 * a.k_rope_row;
  const unsigned k_pitch = 2 * (unsigned)a.k.row, v_pitch = 2 * (unsigned)a.v.row, r_pitch = 2 * (unsigned)a.k_rope_row;
  const unsigned lds0 = (unsigned)(uintptr_t)(__attribute__((address_space(3))) char*)lds;
  const int r4 = 4 * wave + (lane >> 4), r8 = 8 * wave + (lane >> 3);
  const unsigned in_kv = 16 * ((lane & 15) ^ lt_key(r4)), in_rot = 16 * ((lane & 7) ^ ((r8 >> 1) & 7));
  auto request = [&](int t) {
    if (t >= n_all) return;
    const int left = (int)std::min<int64_t>(64, T - 64 * (int64_t)(t_lo + t)) - 1;  // the last row that there is (rows behind it repeat it; they are masked)
    const unsigned to = lds0 + (unsigned)(t % LP_RING) * LP_TILE + 1024 * wave;
    const unsigned ra = std::min(r4, left), rb = std::min(r4 + 32, left), rc = std::min(r8, left);
    const char* const k = k_base + (int64_t)t * 64 * k_pitch;
    const char* const v = v_base + (int64_t)t * 64 * v_pitch;
    const char* const r = r_base + (int64_t)t * 64 * r_pitch;
    unsigned saved;
    asm volatile(
        "s_mov_b32 %0, m0\n\t"
        "s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %6, %11\n\t"
        "s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %7, %11\n\t"
        "s_mov_b32 m0, %3\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %8, %12\n\t"
        "s_mov_b32 m0, %4\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %9, %13\n\t"
        "s_mov_b32 m0, %5\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %10, %13\n\t"
        "s_mov_b32 m0, %0"
        : "=&s"(saved)
        : "s"(to), "s"(to + 8192), "s"(to + LP_ROT), "s"(to + LP_VAL), "s"(to + LP_VAL + 8192), "v"(ra * k_pitch + in_kv), "v"(rb * k_pitch + in_kv),
          "v"(rc * r_pitch + in_rot), "v"(ra * v_pitch + in_kv), "v"(rb * v_pitch + in_kv), "s"(k), "s"(r), "s"(v)
        : "memory");
  };
  LpState st;
  {
    const bf16_t* const q = static_cast<const bf16_t*>(a.q.p) + (int64_t)(it.n0 + row) * a.q.row + it.h * a.q.head + 8 * half;
    const bf16_t* const r = static_cast<const bf16_t*>(a.q_rope.p) + (int64_t)(it.n0 + row) * a.q_rope.row + it.h * a.q_rope.head + 8 * half;
#pragma unroll
    for (int x = 0; x < LP_NK; ++x) st.q[x] = *reinterpret_cast<const lt_bf16x8*>(x < LP_DN / 16 ? q + 16 * x : r + 16 * (x - LP_DN / 16));
  }
  st.start(lane);
  const float c2 = gl.c2;
  // What a wave fetched of a masked tile's values, once it is there: 0 x NaN must not reach rows that do not see them.  (Of keys it does not: masked scores are left
  // out, whatever they are.)
  auto mend = [&](int t, unsigned tile) {
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      uint4* const at = reinterpret_cast<uint4*>(lds + tile + LP_VAL + 8192 * x + 1024 * wave + 16 * lane);
      uint4 w = *at;
      lt_ushort2 high = {0, 0};
      unsigned* const e = &w.x;
#pragma unroll
      for (int y = 0; y < 4; ++y) high = __builtin_elementwise_max(high, __builtin_bit_cast(lt_ushort2, e[y] & 0x7fff7fffu));
      if (high[0] >= 0x7f80 || high[1] >= 0x7f80) {
#pragma unroll
        for (int y = 0; y < 4; ++y) {
          if ((e[y] & 0x7f80u) == 0x7f80u) e[y] &= 0xffff0000u;
          if ((e[y] & 0x7f800000u) == 0x7f800000u) e[y] &= 0xffffu;
        }
        *at = w;
        atomicOr(&mem.odd[t & 3][x], 1u << r4);
      }
    }
  };
  // Block b of tile t: scores that the lane's row does not see, and those of values that are no numbers.
  auto mask = [&](lt_floatx16& S, int t, int b) {
    if (t < n_un) return;
    const int sees = vis - 64 * (t_lo + t) - 32 * b - 4 * half;
    const unsigned odd = mem.odd[t & 3][b] >> (4 * half);
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      const int k = 8 * (v >> 2) + (v & 3);
      S[v] = k < sees ? S[v] : -HS_INF;
    }
    if (odd == 0u) return;
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      const int k = 8 * (v >> 2) + (v & 3);
      S[v] = k < sees && ((odd >> k) & 1u) ? __builtin_nanf("") : S[v];
    }
  };
  // Into tile t: it is there, whole and mended, and every wave is done with tile t - 2.  (The flags of tile t - 2 are free for t + 2.)
  auto enter = [&](int t, unsigned tile, bool younger) {
    if (younger) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LP_LOADS) : "memory");
    else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    if (t >= n_un) mend(t, tile);
    lt_meet();
    if (tid < 2) mem.odd[(t + 2) & 3][tid] = 0u;
  };
  float reference = LT_FLOOR;
#pragma unroll 1
  for (;;) {
    request(0);
    request(1);
    st.clear(reference);
    lt_meet();  // (the flags are cleared: of a lone sequence no barrier stood in front of this one, and tile 0 may be a masked one)
    unsigned here = 0;  // where the tile is in the ring
    auto after = [](unsigned tile) { return tile == (LP_RING - 1) * LP_TILE ? 0u : tile + LP_TILE; };
    if (n_all > 0) {
      enter(0, 0, n_all > 1);
      if (mine_rows > 0) {
        lt_floatx16 S = st.scores(lds, 0, 0), N;
        uint4 P0, P1;
        for (int t = 0; t + 1 < n_all; ++t) {
          mask(S, t, 0);
          st.ahead(lds, here, 1, S, N, c2, P0, P1);
          st.product(lds, here, 0, P0, P1);
          enter(t + 1, after(here), false);
          request(t + 2);
          mask(N, t, 1);
          st.ahead(lds, after(here), 0, N, S, c2, P0, P1);
          st.product(lds, here, 1, P0, P1);
          here = after(here);
        }
        mask(S, n_all - 1, 0);
        st.ahead(lds, here, 1, S, N, c2, P0, P1);
        st.product(lds, here, 0, P0, P1);
        mask(N, n_all - 1, 1);
        st.take(lds, here, 1, N, c2);
      } else {
        for (int t = 0; t + 1 < n_all; ++t) {
          enter(t + 1, after(here), false);
          request(t + 2);
          here = after(here);
        }
      }
    }
    // ---- a row whose scores rose too far above its reference?
    if (tid == 0) mem.again = 0;
    lt_meet();
    if (__ballot(st.rose(c2)) != 0ull && lane == 0) mem.again = 1;
    lt_meet();
    if (mem.again == 0) break;
    reference = st.seen;
    if (tid < 8) mem.odd[tid >> 1][tid & 1] = 0u;
  }
  if (mine_rows <= 0) return;
  const float total = lt_half_sum(st.l);
  const int64_t row0 = (int64_t)(it.n0 + first + 32 * wave) * a.H + it.h;  // of rows a.H apart
  char* const stage = lds + wave * 32 * LP_OUT_PITCH;
  if (it.n_sp == 1) {
    const float inv = vis == 0 ? 0.f : 1.f / total;  // (a row that sees keys of score -infinity alone is 0 / 0, its logarithm -infinity)
    if (half == 0 && col < mine_rows && a.lse != nullptr)
      a.lse[row0 + (int64_t)col * a.H] = st.m * a.scale + __log2f(total) * LT_LN2;
    if (half == 0) mem.out_at[wave][col] = (int64_t)(it.n0 + row) * a.o_row + it.h * a.o_head;
#pragma unroll
    for (int t = 0; t < LP_NB; ++t)
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        const lt_floatx2 x = {st.acc[t][4 * b] * inv, st.acc[t][4 * b + 1] * inv}, y = {st.acc[t][4 * b + 2] * inv, st.acc[t][4 * b + 3] * inv};
        *reinterpret_cast<uint2*>(stage + col * LP_OUT_PITCH + 64 * t + 16 * b + 8 * half) =
            make_uint2(__builtin_bit_cast(unsigned, __builtin_convertvector(x, lt_bf16x2)), __builtin_bit_cast(unsigned, __builtin_convertvector(y, lt_bf16x2)));
      }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll 4
    for (int x = lane; x < mine_rows * 16; x += 64)
      *reinterpret_cast<uint4*>(static_cast<bf16_t*>(a.o) + mem.out_at[wave][x >> 4] + 8 * (x & 15)) =
          *reinterpret_cast<const uint4*>(stage + (x >> 4) * LP_OUT_PITCH + 16 * (x & 15));
    return;
  }
  const int64_t rec0 = it.rec0 + ((int64_t)(first + 32 * wave) * a.H + it.h) * it.n_sp + it.sp;  // (records: row, head, split)
  if (half == 0 && col < mine_rows) {
    float* const rec = gl.part + (rec0 + (int64_t)col * a.H * it.n_sp) * LP_REC;
    rec[LP_DV] = st.m;
    rec[LP_DV + 1] = total;
  }
#pragma unroll
  for (int x0 = 0; x0 < LP_NB; x0 += 2) {  // 64 columns at a time
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int b = 0; b < 4; ++b)
        *reinterpret_cast<float4*>(stage + col * LP_OUT_PITCH + 128 * t + 32 * b + 16 * half) =
            make_float4(st.acc[x0 + t][4 * b], st.acc[x0 + t][4 * b + 1], st.acc[x0 + t][4 * b + 2], st.acc[x0 + t][4 * b + 3]);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll 4
    for (int x = lane; x < mine_rows * 16; x += 64)
      *reinterpret_cast<float4*>(gl.part + (rec0 + (int64_t)(x >> 4) * a.H * it.n_sp) * LP_REC + 32 * x0 + 4 * (x & 15)) =
          *reinterpret_cast<const float4*>(stage + (x >> 4) * LP_OUT_PITCH + 16 * (x & 15));
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }
}

// The merge of the splits: half a wave to a (row, head), four columns to a lane.
constexpr int LPM_THREADS = 256;
__global__ __launch_bounds__(LPM_THREADS) void k_lat_prompt_merge(LpArgs gl) {
  const LatPromptArgs& a = gl.a;
  const int lane = threadIdx.x & 31, wide = threadIdx.x & 63;
  const unsigned rows = (unsigned)a.N * (unsigned)a.H;  // (below 2^24)
  const unsigned at = (unsigned)blockIdx.x * (LPM_THREADS / 32) + (threadIdx.x >> 5), row = std::min(at, rows - 1);
  const int n = (int)(row / (unsigned)a.H), h = (int)(row - (unsigned)n * (unsigned)a.H);
  // the row's sequence, and its first record (whole waves: 64 sequences at a time)
  int own = 0, n_sp = 0, n0 = 0, rec0 = 0, keys = 0;
  bool found = a.B == 1;
  if (found) {
    int64_t k0, T;
    lp_sequence(gl, 0, &n0, &own, &k0, &T, &n_sp);
    keys = (int)T;
  }
  for (int base = 0, before = 0; base < a.B && a.B > 1; base += 64) {
    int s_n0 = 0, s_n = 0, s_sp = 0;
    int64_t k0, T = 0;
    if (base + wide < a.B) lp_sequence(gl, base + wide, &s_n0, &s_n, &k0, &T, &s_sp);
    const int recs = lp_records(s_n, a.H, s_sp), upto = wave_prefix_sum(recs);
#pragma unroll
    for (int x = 0; x < 2; ++x) {  // the wave's two rows
      const int want = __builtin_amdgcn_readlane(n, 32 * x);
      const unsigned long long hit = __ballot(s_n0 <= want && want < s_n0 + s_n);
      if (hit == 0ull) continue;
      const int who = __builtin_ctzll(hit);
      const int t_n = __builtin_amdgcn_readlane(s_n, who), t_sp = __builtin_amdgcn_readlane(s_sp, who), t_n0 = __builtin_amdgcn_readlane(s_n0, who),
                t_rec = before + __builtin_amdgcn_readlane(upto - recs, who), t_keys = __builtin_amdgcn_readlane((int)T, who);
      if (wide >> 5 == x) own = t_n, n_sp = t_sp, n0 = t_n0, rec0 = t_rec, keys = t_keys, found = true;
    }
    if (__ballot(!found) == 0ull) break;
    before += __builtin_amdgcn_readlane(upto, 63);
  }
  if (at >= rows || n_sp <= 1 || rec0 + lp_records(own, a.H, n_sp) > gl.records) return;
  const float* const rec = gl.part + (rec0 + ((int64_t)(n - n0) * a.H + h) * n_sp) * LP_REC;
  // (one pass, with the running maximum: the records of four splits at a time)
  float m = LT_FLOOR, total = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int x0 = 0; x0 < n_sp; x0 += 4) {
    float rm[4], rl[4];
    float4 v[4];
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const float* const r = rec + (int64_t)std::min(x0 + x, n_sp - 1) * LP_REC;
      rm[x] = r[LP_DV];
      rl[x] = r[LP_DV + 1];
      v[x] = *reinterpret_cast<const float4*>(r + 4 * lane);
    }
    const float up = fmaxf(fmaxf(m, fmaxf(rm[0], rm[1])), fmaxf(rm[2], rm[3])), old = exp2_fast((m - up) * gl.c2);
    total *= old, o.x *= old, o.y *= old, o.z *= old, o.w *= old;
    m = up;
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const float w = x0 + x < n_sp ? exp2_fast((rm[x] - m) * gl.c2) : 0.f;
      if (x0 + x >= n_sp) break;
      total = __builtin_fmaf(w, rl[x], total);
      o.x = __builtin_fmaf(w, v[x].x, o.x), o.y = __builtin_fmaf(w, v[x].y, o.y), o.z = __builtin_fmaf(w, v[x].z, o.z), o.w = __builtin_fmaf(w, v[x].w, o.w);
    }
  }
  const float inv = keys - own + (n - n0) < 0 ? 0.f : 1.f / total;  // (0: a row that sees no key)
  *reinterpret_cast<uint2*>(static_cast<bf16_t*>(a.o) + n * a.o_row + h * a.o_head + 4 * lane) =
      make_uint2(__builtin_bit_cast(unsigned, __builtin_convertvector((lt_floatx2{o.x * inv, o.y * inv}), lt_bf16x2)),
                 __builtin_bit_cast(unsigned, __builtin_convertvector((lt_floatx2{o.z * inv, o.w * inv}), lt_bf16x2)));
  if (lane == 0 && a.lse != nullptr) a.lse[row] = m * a.scale + __log2f(total) * LT_LN2;
}

// ------------------------------------------------------------------------------------------------ the host's part
bool lat_prompt_matrix(const LatPromptArgs& a, hs_dtype dt) {
  auto fits = [](const void* p, int64_t s, int64_t t) { return reinterpret_cast<uintptr_t>(p) % 16 == 0 && s % 8 == 0 && t % 8 == 0; };
  constexpr int64_t FAR = (int64_t)1 << 23;  // (64 rows of a tile within 32 bits)
  return dt == HS_BF16 && a.Dn == LP_DN && a.Dr == LP_DR && a.Dv == LP_DV && fits(a.q.p, a.q.row, a.q.head) && fits(a.q_rope.p, a.q_rope.row, a.q_rope.head) &&
         fits(a.k.p, a.k.row, a.k.head) && fits(a.v.p, a.v.row, a.v.head) && fits(a.k_rope, a.k_rope_row, 0) && fits(a.o, a.o_row, a.o_head) && a.k.row < FAR &&
         a.v.row < FAR && a.k_rope_row < FAR;
}

// Rows of a group and tiles of a split, by estimated times.  (Groups of 128 for calls of few items: 660 rows of 20 heads 29.6 -> 19.3 us, 3468 of 16 heads
// 106 -> 82; where the items fill the chip, groups of 256: 8192 rows of 32 heads 640 us, of 128 724.)
LatPlan lat_prompt_plan(const int32_t* qo, const int64_t* ko, int32_t B, int32_t H) {
  int64_t longest = 1;
  for (int s = 0; s < B; ++s)
    if (qo[s + 1] > qo[s]) longest = std::max(longest, (ko[s + 1] - ko[s] + 63) >> 6);
  constexpr double FIXED = 8.0, CU = 256.0, REC = 0.0002;  // us of an item without tiles, compute units, us a row's record
  LatPlan best = {};
  best.sp_max = 1;
  double best_us = 0.0;
  auto consider = [&](int64_t per, int group) {
    const double TILE = group == LP_GROUP ? 1.7 : 1.15;  // us: one wave to a SIMD has fewer products to do, and nobody who fills its waits
    double sum = 0.0, most = 0.0;
    int64_t items = 0, sp_max = 1, records = 0;
    for (int s = 0; s < B; ++s) {
      const int n = qo[s + 1] - qo[s];
      if (n == 0) continue;
      const int64_t T = ko[s + 1] - ko[s], n_sp = lp_splits(T, (int)per), groups = lp_groups(n, group);
      const double last = (double)((T + 63) >> 6), first = std::max(0.0, (double)(T - n) / 64.0);  // tiles of the last group, about those of the first
      sum += (double)groups * H * ((double)n_sp * FIXED + TILE * (last + first) / 2);
      most = std::max(most, FIXED + TILE * last / (double)n_sp);
      items += groups * n_sp * H;
      sp_max = std::max(sp_max, n_sp);
      if (n_sp > 1) records += (int64_t)n * H * n_sp;
    }
    double us = (double)items <= CU ? most : std::max(most, sum / CU + 0.3 * most);
    if (sp_max > 1) us += 4.0 + REC * (double)records;
    if (best.per == 0 || (us < best_us && records <= 4 * LAT_MAX_RECORDS))
      best_us = us, best.per = (int)per, best.sp_max = (int)sp_max, best.group = group, best.grid = items, best.records = records;
    return items;
  };
  for (int group : {LP_GROUP, LP_GROUP / 2}) {
    const int64_t whole = consider(longest, group);
    for (int64_t target : {(int64_t)64, (int64_t)128, (int64_t)192, (int64_t)256, (int64_t)384, (int64_t)512, (int64_t)1024, (int64_t)2048, whole + 256}) {
      if (target <= whole) continue;
      int64_t lo = 1, hi = longest;
      while (lo < hi) {
        const int64_t mid = (lo + hi) / 2;
        if (consider(mid, group) <= target) hi = mid;
        else lo = mid + 1;
      }
      if (lo == 1) break;
    }
  }
  return best;
}

size_t lat_prompt_bytes(const LatPlan& p) { return align_up((size_t)p.records * LP_REC * 4, 256); }

hs_status lat_prompt_launch(const LatPromptArgs& a, const LatPlan& p, int one_len, void* workspace, hipStream_t stream) {
  LpArgs g = {a, a.scale * LT_LOG2E, p.per, p.sp_max, p.group, static_cast<float*>(workspace), (int)p.records, one_len};
  hipLaunchKernelGGL(k_lat_prompt, dim3((unsigned)p.grid), dim3(LP_THREADS), 0, stream, g);
  const hs_status st = launch_status("latent prompt attention");
  if (st != HS_OK || p.sp_max == 1) return st;
  const int64_t rows = (int64_t)a.N * a.H;
  hipLaunchKernelGGL(k_lat_prompt_merge, dim3((unsigned)((rows + LPM_THREADS / 32 - 1) / (LPM_THREADS / 32))), dim3(LPM_THREADS), 0, stream, g);
  return launch_status("latent prompt attention, merge");
}

}  // namespace hs
