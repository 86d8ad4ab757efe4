// Shared pieces of the attention kernels on a quantised cache (internal).
#pragma once
#include "mx.h"

namespace hs {

hs_status mx_pool_check(const char* what, const MxPool& c, hs_mx_format fmt);
hs_status mx_pool_pointers(const char* what, const MxPool& c);

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef short shortx4 __attribute__((ext_vector_type(4)));
typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef float floatx2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) shortx4* lds_s4_ptr;

constexpr int MXA_THREADS = 512;
constexpr int MXA_WAVES = 8;
constexpr int MXA_MAX_M = 1024;       // tree rows of a sequence
constexpr float MX_LIMIT = 0x1p40f;   // a denominator (of a half-wave's keys) that reaches it moves the maximum
constexpr float MXA_FLOOR = -3.402823466e38f;
constexpr float MXA_LOG2E = 1.4426950408889634f, MXA_LN2 = 0.6931471805599453f;

struct MxAttnArgs {
  const void* q;
  const void* k_tree;
  const void* v_tree;
  int64_t q_stride, k_stride, v_stride;  // elements from row to row
  MxPool pool;
  const int32_t* parent;
  const int32_t* node_offsets;
  const int64_t* lens;
  int B, Hq, G;
  int blocks_most;       // row blocks of a work item at most: 1, 2, 4 or 8
  int target;            // what an item may cost (mx_cut)
  float c2;              // scale * log2(e)
  void* o;
  float* lse;
  float* part;           // records of D + 4 floats: o (not normalised), maximum (in octaves), denominator
};

// How a sequence is cut, on the host (the plan) and on the device (every workgroup finds its item).  Its rows of a KV head, in
// blocks of 32, are spread evenly over as few row groups of up to `blocks_most` blocks as hold them; the size of a group decides
// how the eight waves of its workgroup share the work:
//   one or two blocks    every wave by itself, on every eighth (fourth) 32 keys
//   three or four        tiles of 64 keys shared through LDS, two waves to a block, each with half of a tile
//   five to eight        the same, a wave to a block
// and with that what a page of 64 keys costs; the keys are cut into splits of as many pages as `target` pays for (64 splits at most).
enum MxForm { MX_PRIVATE_1 = 0, MX_PRIVATE_2 = 1, MX_SHARED_4 = 2, MX_SHARED_8 = 3 };
constexpr int MXA_SPLITS = 64;  // (a lane each where they meet)
// Costs of a page in the four forms, in sixteenths of a microsecond, by format: see mx_plan.
constexpr int MX_PAGE_COST[2][4] = {{8, 10, 16, 28}, {6, 9, 16, 28}};
struct MxCut {
  int n_blk, n_rg, form, pages, n_sp;  // pages: of a split
};
__host__ __device__ __forceinline__ MxCut mx_cut(int rows, int64_t L, int fmt, int blocks_most, int target) {
  MxCut c;
  c.n_blk = (rows + 31) >> 5;
  const int shift = blocks_most == 8 ? 3 : blocks_most == 4 ? 2 : blocks_most == 2 ? 1 : 0;
  c.n_rg = (c.n_blk + blocks_most - 1) >> shift;
  const bool over4 = c.n_blk > 4 * c.n_rg, over2 = c.n_blk > 2 * c.n_rg, over1 = c.n_blk > c.n_rg;
  c.form = over4 ? MX_SHARED_8 : over2 ? MX_SHARED_4 : over1 ? MX_PRIVATE_2 : MX_PRIVATE_1;
  const int cost = over4 ? MX_PAGE_COST[fmt][3] : over2 ? MX_PAGE_COST[fmt][2] : over1 ? MX_PAGE_COST[fmt][1] : MX_PAGE_COST[fmt][0];
  const int all = (int)((L + MX_PAGE - 1) / MX_PAGE), least = (all + MXA_SPLITS - 1) / MXA_SPLITS;
  c.pages = (int)((unsigned)target / (unsigned)cost);
  c.pages = c.pages < least ? least : c.pages;
  c.pages = c.pages < 1 ? 1 : c.pages;
  c.n_sp = (int)((unsigned)(all + c.pages - 1) / (unsigned)c.pages);
  c.n_sp = c.n_sp < 1 ? 1 : c.n_sp;
  c.pages = (int)((unsigned)(all + c.n_sp - 1) / (unsigned)c.n_sp);  // (splits of equal size)
  c.pages = c.pages < 1 ? 1 : c.pages;
  return c;
}

// The work item of this workgroup: items are numbered sequence by sequence, in a sequence
// (split * row groups + row group) * Hkv + KV head.  Every wave finds it by a prefix sum over the sequences.
struct MxItem {
  int s, n0, M, g, sp, n_sp, pages, form;
  int blk0, blk_n;  // row blocks
  int64_t L;
  int64_t rec0;     // records of the sequences before
};
template <int FMT>
__device__ __forceinline__ bool mx_item(const MxAttnArgs& a, int item, MxItem& w) {
  const int lane = (int)(threadIdx.x & 63);
  int done = 0;
  int64_t recs = 0;
  for (int base = 0; base < a.B; base += 64) {
    const int s = base + lane;
    int n0 = 0, M = 0, L = 0;
    if (s < a.B) {
      n0 = a.node_offsets[s];
      M = a.node_offsets[s + 1] - n0;
      L = (int)a.lens[s];
    }
    const MxCut c = mx_cut(a.G * M, L, FMT, a.blocks_most, a.target);
    const int items = M > 0 ? c.n_sp * c.n_rg * a.pool.Hkv : 0;
    const int rec = M > 0 && c.n_sp > 1 ? M * a.Hq * c.n_sp : 0;
    const int upto = done + wave_prefix_sum(items), rec_upto = wave_prefix_sum(rec);
    const unsigned long long behind = __ballot(upto > item);
    if (behind != 0ull) {
      const int e = __builtin_ctzll(behind);
      w.s = base + e;
      w.n0 = __builtin_amdgcn_readlane(n0, e);
      w.M = __builtin_amdgcn_readlane(M, e);
      w.L = __builtin_amdgcn_readlane(L, e);
      w.n_sp = __builtin_amdgcn_readlane(c.n_sp, e);
      w.pages = __builtin_amdgcn_readlane(c.pages, e);
      w.form = __builtin_amdgcn_readlane(c.form, e);
      const int n_blk = __builtin_amdgcn_readlane(c.n_blk, e), n_rg = __builtin_amdgcn_readlane(c.n_rg, e);
      w.rec0 = recs + __builtin_amdgcn_readlane(rec_upto, e) - __builtin_amdgcn_readlane(rec, e);
      unsigned local = (unsigned)(item - (__builtin_amdgcn_readlane(upto, e) - __builtin_amdgcn_readlane(items, e)));
      const unsigned hkv = (unsigned)a.pool.Hkv;
      w.g = (int)(local % hkv);
      local /= hkv;
      const int rg = (int)(local % (unsigned)n_rg);
      w.sp = (int)(local / (unsigned)n_rg);
      const int each = n_blk / n_rg, more = n_blk - each * n_rg;  // the first `more` groups hold one block more
      w.blk0 = rg * each + (rg < more ? rg : more);
      w.blk_n = each + (rg < more ? 1 : 0);
      return true;
    }
    done = __builtin_amdgcn_readlane(upto, 63);
    recs += __builtin_amdgcn_readlane(rec_upto, 63);
  }
  return false;
}

// (an element of a vector is copied before its bits are taken: a bit cast of the element itself reads the first one)
__device__ __forceinline__ float2 both_halves(float x) {  // this lane's value in the lower and in the upper half-wave
  const unsigned u = __builtin_bit_cast(unsigned, x);
  const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  const unsigned lo = r[0], hi = r[1];
  return make_float2(__builtin_bit_cast(float, lo), __builtin_bit_cast(float, hi));
}
__device__ __forceinline__ float half_max(float x) {
  const float2 h = both_halves(x);
  return fmaxf(h.x, h.y);
}
__device__ __forceinline__ float half_sum(float x) {
  const float2 h = both_halves(x);
  return h.x + h.y;
}

// 16-byte chunk `c` of row r of a V tile in LDS (rows of D bfloat16): the four rows that a transposing read touches in a
// half-wave lie in four different 64-byte bank ranges.
template <int D>
__device__ __forceinline__ int v_at(int r, int c) {
  const int x = D == 128 ? ((r & 3) << 2) | ((r >> 2) & 3) : (((r >> 1) & 1) << 2) | ((r >> 2) & 3);
  return r * (2 * D) + ((c ^ x) << 4);
}

// NaN and infinity among the values of tree rows: a row that does not see such a row must not take 0 x NaN from it.  The
// largest magnitude bits of the elements tell (a packed 16-bit maximum a pair); where there are any, they are left out of
// the product and added to the rows that see them.
typedef unsigned short ushort2v __attribute__((ext_vector_type(2)));
__device__ __forceinline__ void note_bits(ushort2v& most, const uint4& w) {
  const unsigned x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) most = __builtin_elementwise_max(most, __builtin_bit_cast(ushort2v, x[i] & 0x7fff7fffu));
}
__device__ __forceinline__ bool has_odd(ushort2v most) { return most[0] >= 0x7f80 || most[1] >= 0x7f80; }
__device__ __forceinline__ unsigned without_odd(unsigned w) {
  if ((w & 0x7f80u) == 0x7f80u) w &= 0xffff0000u;
  if ((w & 0x7f800000u) == 0x7f800000u) w &= 0xffffu;
  return w;
}
__device__ __forceinline__ uint4 without_odd(const uint4& w) {
  return make_uint4(without_odd(w.x), without_odd(w.y), without_odd(w.z), without_odd(w.w));
}

// One softmax state: 32 rows of a wave.
template <int D>
struct MxState {
  static constexpr int NT = D / 32;
  floatx16 acc[NT];  // O^T: element 32 tt + 8 (v / 4) + 4 half + v % 4 of row `col`
  float m, l;        // running maximum of the scaled scores (octaves), sum relative to it (this half-wave's keys)
  __device__ __forceinline__ void clear() {
    m = MXA_FLOOR;
    l = 0.f;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[t][v] = 0.f;
  }
  // The odd values of `rows` tree rows from v on, for the rows that see them (`word`).
  __device__ __forceinline__ void add_odd(const bf16_t* v, int64_t stride, int rows, unsigned word, int half) {
    for (int j = 0; j < rows; ++j)
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const float x = bf16_to_f32(v[j * stride + 32 * t + 8 * (e >> 2) + 4 * half + (e & 3)]);
          if (((word >> j) & 1u) != 0u && !(fabsf(x) < HS_INF)) acc[t][e] += x;
        }
  }
  // The maximum of the rows whose denominator reaches MX_LIMIT (or is a NaN) moves to the largest of a block's scores; the
  // other rows keep theirs, so that no row's rounding depends on its neighbours.
  __device__ __forceinline__ void move(const floatx16& S, float c2, float sum) {
    float top = fmaxf(S[0], S[1]);
#pragma unroll
    for (int v = 2; v < 16; ++v) top = fmaxf(top, S[v]);
    const bool moves = half_max(sum < MX_LIMIT ? 0.f : 1.f) > 0.f;
    const float up = moves ? fmaxf(m, half_max(top) * c2) : m, alpha = exp2_fast(m - up);
    m = up;
    l *= alpha;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[t][v] *= alpha;
  }
  // The first scores of a pass (accumulators and sum are zero): their maximum is the row's.
  __device__ __forceinline__ void start(const floatx16& S, float c2) {
    float top = fmaxf(S[0], S[1]);
#pragma unroll
    for (int v = 2; v < 16; ++v) top = fmaxf(top, S[v]);
    m = fmaxf(MXA_FLOOR, half_max(top) * c2);
  }
  __device__ __forceinline__ floatx2 exps(const floatx16& S, float c2, int j) const {  // scores 2j, 2j + 1
    return floatx2{exp2_fast(__builtin_fmaf(S[2 * j], c2, -m)), exp2_fast(__builtin_fmaf(S[2 * j + 1], c2, -m))};
  }
  // Four pairs of scores (half h of a block) to bfloat16 pairs; they are added to `sum` one after the other.
  __device__ __forceinline__ void exp_half(const floatx16& S, float c2, int h, uint4& P, float& sum) const {
    unsigned w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const floatx2 p = exps(S, c2, 4 * h + j);
      sum += p[0] + p[1];
      w[j] = __builtin_bit_cast(unsigned, __builtin_convertvector(p, bf16x2));
    }
    P = make_uint4(w[0], w[1], w[2], w[3]);
  }
  __device__ __forceinline__ static bool over(float s) { return __ballot(!(s < MX_LIMIT)) != 0ull; }
  // Scores (masked ones at -inf) to P: bfloat16 pairs of the first 16 and the second 16 keys.
  __device__ __forceinline__ void softmax(const floatx16& S, float c2, uint4& p0, uint4& p1) {
    float s = l;
    exp_half(S, c2, 0, p0, s);
    exp_half(S, c2, 1, p1, s);
    if (over(s)) {
      move(S, c2, s);
      s = l;
      exp_half(S, c2, 0, p0, s);
      exp_half(S, c2, 1, p1, s);
    }
    l = s;
  }
};

// The tree's parents and hops in LDS, by the whole workgroup (a barrier inside and behind).
__device__ __forceinline__ void mx_stage_tree(const MxAttnArgs& a, const MxItem& it, int* par, int2* hops) {
  for (int j = threadIdx.x; j < it.M; j += MXA_THREADS) par[j] = a.parent[it.n0 + j];
  __syncthreads();
  for (int j = threadIdx.x; j < it.M; j += MXA_THREADS) {
    unsigned bits = 1u << (j & 31);
    int x = j;
    for (;;) {
      const int up = par[x];
      x = up < x ? up : -1;  // (a malformed tree cannot keep the walk from ending)
      if (x < (j & ~31)) break;
      bits |= 1u << (x & 31);
    }
    hops[j] = make_int2((int)bits, x < 0 ? -1 : x);
  }
  __syncthreads();
}
// The part of a row's root path in tree rows 32 b .. 32 b + 31; b falls from call to call.
__device__ __forceinline__ unsigned mx_path_word(const int2* hops, int& cur, int b) {
  if (cur < 0 || (cur >> 5) != b) return 0u;
  const int2 hop = hops[cur];
  cur = hop.y;
  return (unsigned)hop.x;
}

// Columns d .. d + 3 of a row: a result (the sequence has one split), or a part of the split's record.
__device__ __forceinline__ void mx_write4(const MxAttnArgs& a, bool whole, int64_t out, float* rec, int d, float4 sum, float inv) {
  if (whole) {
    const floatx2 lo = {sum.x * inv, sum.y * inv}, hi = {sum.z * inv, sum.w * inv};
    uint2 w;
    w.x = __builtin_bit_cast(unsigned, __builtin_convertvector(lo, bf16x2));
    w.y = __builtin_bit_cast(unsigned, __builtin_convertvector(hi, bf16x2));
    *reinterpret_cast<uint2*>(static_cast<bf16_t*>(a.o) + out * a.pool.D + d) = w;
  } else {
    *reinterpret_cast<float4*>(rec + d) = sum;
  }
}

constexpr int MXS_BUF = 3;
// Rows of a tile in LDS, in bytes.  K: 16 bytes more than a row, so that the 16-byte pieces that 16 lanes read, of 16 rows, lie in
// different banks; V: 64 bytes more, so that the four rows that a transposing read touches in a half-wave do.  (Padding
// instead of an exchange of pieces: every fragment is one register plus an immediate.)
constexpr int mxs_k_row(int D) { return 2 * D + 16; }
constexpr int mxs_v_row(int D) { return 2 * D + 64; }

// A workgroup's LDS: the shared tiles (K buffers, then V buffers), or the private V tiles, and at the end the waves' sums.
template <int D>
struct MxLds {
  static constexpr int SHARED = MXS_BUF * MX_PAGE * (mxs_k_row(D) + mxs_v_row(D));
  static constexpr int SUMS = MXA_WAVES * (D / 32) * 16 * 64 * 4;
  alignas(16) char tiles[SHARED > SUMS ? SHARED : SUMS];
  float den[MXA_WAVES][2][32];  // maxima and sums of the waves
  int par[MXA_MAX_M];
  int2 hops[MXA_MAX_M];         // of a tree row: its root path inside its own 32 rows as bits, the next row of it outside
  int odd, redo;
};

}  // namespace hs
