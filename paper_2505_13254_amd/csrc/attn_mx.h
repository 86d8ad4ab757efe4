// Shared pieces of the attention kernels on a quantised cache (internal).
#pragma once
#include <type_traits>

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
constexpr float MX_LIMIT = 0x1p80f;   // a denominator (of a half-wave's keys) that reaches it moves the maximum, or sends its row to attn_mx_follow
constexpr float MXA_FLOOR = -3.402823466e38f;
constexpr float MXA_LOG2E = 1.4426950408889634f, MXA_LN2 = 0.6931471805599453f;

// How the sequences of a call are cut, on the host (the plan) and on the device (every workgroup finds its item).  A
// sequence's rows of a KV head, in blocks of 32, are spread evenly over as few row groups of up to `blocks_most` blocks as hold
// them; the size of a group decides how the eight waves of its workgroup share the work:
//   one or two blocks    every wave by itself, on every eighth (fourth) 32 keys
//   three or four        tiles of 64 keys shared through LDS, two waves to a block, each with half of a tile
//   five to eight        the same, a wave to a block
// Its keys are cut into splits of equal numbers of 64-token pages, at most pages[form] each; the tree's own rows go with the last
// split, or are a split of their own where they would not fit it.
enum MxForm { MX_PRIVATE_1 = 0, MX_PRIVATE_2 = 1, MX_SHARED_4 = 2, MX_SHARED_8 = 3 };
constexpr int MXA_SPLITS = 64;  // of a sequence at most (a lane each where they meet)
struct MxCuts {
  int blocks_most;  // 1, 2, 4 or 8
  int pages[4];
};
// x / d, exact, for 0 <= x < 2^23 and 1 <= d: a float product and one correction.
__host__ __device__ __forceinline__ int mx_div(int x, int d) {
#ifdef __HIP_DEVICE_COMPILE__
  int q = (int)((float)x * __builtin_amdgcn_rcpf((float)d));
  const int r = x - q * d;
  q += r < 0 ? -1 : r >= d ? 1 : 0;
  return q;
#else
  return x / d;
#endif
}
struct MxCut {
  int n_blk, n_rg, form, pages, n_sp;  // pages: of a split
};
__host__ __device__ __forceinline__ MxCut mx_groups(int M, int G, int blocks_most) {
  MxCut c;
  c.n_blk = (G * M + 31) >> 5;
  const int shift = blocks_most == 8 ? 3 : blocks_most == 4 ? 2 : blocks_most == 2 ? 1 : 0;
  c.n_rg = (c.n_blk + blocks_most - 1) >> shift;
  const bool over4 = c.n_blk > 4 * c.n_rg, over2 = c.n_blk > 2 * c.n_rg, over1 = c.n_blk > c.n_rg;
  c.form = over4 ? MX_SHARED_8 : over2 ? MX_SHARED_4 : over1 ? MX_PRIVATE_2 : MX_PRIVATE_1;
  return c;
}
__host__ __device__ __forceinline__ void mx_splits(int M, int L, int per, MxCut& c) {
  const int pages = (L + MX_PAGE - 1) >> 6, tiles = (M + MX_PAGE - 1) >> 6, all = pages + tiles;
  const int least = mx_div(all + MXA_SPLITS - 2, MXA_SPLITS - 1);
  per = per < least ? least : per < 1 ? 1 : per;
  const int even = mx_div(all + per - 1, per);
  c.pages = mx_div(all + even - 1, even < 1 ? 1 : even);
  c.pages = c.pages < 1 ? 1 : c.pages;
  c.n_sp = mx_div(pages + c.pages - 1, c.pages);
  if (c.n_sp > 0 && tiles > c.n_sp * c.pages - pages) ++c.n_sp;
  c.n_sp = c.n_sp < 1 ? 1 : c.n_sp;
}
__host__ __device__ __forceinline__ MxCut mx_cut(int M, int G, int L, const MxCuts& cuts) {
  MxCut c = mx_groups(M, G, cuts.blocks_most);
  mx_splits(M, L, c.form == 3 ? cuts.pages[3] : c.form == 2 ? cuts.pages[2] : c.form == 1 ? cuts.pages[1] : cuts.pages[0], c);
  return c;
}

// What a launch attends to travels in its arguments, taken from the host arrays: a captured launch keeps it, whatever becomes of the device's.
// A sequence with rows as the host cut it.  The entries of up to MXA_ENTRIES sequences, in the order of their items: a workgroup
// knows its item after one trip to memory.  Of longer batches the rows and lengths of up to MXA_SEQS sequences to a launch, which the device cuts.
struct MxEntry {
  int first;       // its first item
  int n0, M, L;
  int pages;       // of a split
  int n_sp_form;   // splits | form << 8 | sequence << 16
  int groups;      // row blocks | row groups << 16
  int rec0;        // records of the sequences before
};
static_assert(sizeof(MxEntry) == 32, "two 16-byte loads");
constexpr int MXA_ENTRIES = 64;
struct MxSeq {
  int n0, L;  // first row (behind the last sequence: where its rows end), prefix tokens
};
constexpr int MXA_SEQS = MXA_ENTRIES * (int)(sizeof(MxEntry) / sizeof(MxSeq)) - 1;  // (in the entries' place)

struct MxAttnArgs {
  const void* q;
  const void* k_tree;
  const void* v_tree;
  int64_t q_stride, k_stride, v_stride;  // elements from row to row
  MxPool pool;
  const int32_t* parent;
  int Hq, G;
  MxCuts cuts;
  float inv_G;           // 1 / G
  float c2;              // scale * log2(e)
  void* o;
  float* lse;
  float* part;           // records of D + 4 floats: o of the split's keys, maximum (in octaves), denominator
  int n_entries;         // 0: more sequences than entries
  int n_seqs, seq0;      // then: sequences of the launch, and the first one's number
  union {
    alignas(16) MxEntry entries[MXA_ENTRIES];
    alignas(16) MxSeq seqs[MXA_SEQS + 1];
  };
};
static_assert(sizeof(MxAttnArgs) <= 4096 && sizeof(MxSeq) * (MXA_SEQS + 1) == sizeof(MxEntry) * MXA_ENTRIES, "kernel arguments");

// The work item of this workgroup: items are numbered sequence by sequence, in a sequence
// (split * row groups + row group) * Hkv + KV head.  Every wave finds it by a prefix sum over the sequences.
struct MxItem {
  int s, n0, M, L, g, form;
  int blk0, blk_n;      // row blocks
  int sp, n_sp, pages;  // its split, of how many, of how many pages
  int64_t rec0;         // records of the sequences before
};
// Fields that several ways of finding an item share; `local` is the item's number in its sequence.
__device__ __forceinline__ void mx_place(const MxAttnArgs& a, int local, int n_blk, int n_rg, MxItem& w) {
  const int x = __builtin_amdgcn_readfirstlane(mx_div(local, a.pool.Hkv));
  w.g = local - x * a.pool.Hkv;
  w.sp = n_rg == 1 ? x : __builtin_amdgcn_readfirstlane(mx_div(x, n_rg));
  const int rg = x - w.sp * n_rg;
  const int each = n_rg == 1 ? n_blk : __builtin_amdgcn_readfirstlane(mx_div(n_blk, n_rg)), more = n_blk - each * n_rg;
  w.blk0 = rg * each + (rg < more ? rg : more);  // (the first `more` groups hold one block more)
  w.blk_n = each + (rg < more ? 1 : 0);
}
__device__ __forceinline__ bool mx_item(const MxAttnArgs& a, int item, MxItem& w) {
  const int lane = (int)(threadIdx.x & 63);
  if (a.n_entries == 1) {  // (its entry comes with the other arguments)
    const MxEntry& e = a.entries[0];
    w.s = e.n_sp_form >> 16, w.n0 = e.n0, w.M = e.M, w.L = e.L, w.pages = e.pages, w.rec0 = 0;
    w.n_sp = e.n_sp_form & 255, w.form = (e.n_sp_form >> 8) & 255;
    mx_place(a, item, e.groups & 0xffff, (int)((unsigned)e.groups >> 16), w);
    return true;
  }
  if (a.n_entries > 0) {
    const int4 lo = *reinterpret_cast<const int4*>(&a.entries[lane]), hi = *(reinterpret_cast<const int4*>(&a.entries[lane]) + 1);
    const int e = __builtin_popcountll(__ballot(lane < a.n_entries && lo.x <= item)) - 1;
    w.n0 = __builtin_amdgcn_readlane(lo.y, e);
    w.M = __builtin_amdgcn_readlane(lo.z, e);
    w.L = __builtin_amdgcn_readlane(lo.w, e);
    w.pages = __builtin_amdgcn_readlane(hi.x, e);
    const int nf = __builtin_amdgcn_readlane(hi.y, e), groups = __builtin_amdgcn_readlane(hi.z, e);
    w.n_sp = nf & 255;
    w.form = (nf >> 8) & 255;
    w.s = nf >> 16;
    w.rec0 = __builtin_amdgcn_readlane(hi.w, e);
    mx_place(a, item - __builtin_amdgcn_readlane(lo.x, e), groups & 0xffff, (int)((unsigned)groups >> 16), w);
    return true;
  }
  int done = 0;
  int64_t recs = 0;
  for (int base = 0; base < a.n_seqs; base += 64) {
    const int s = base + lane;
    int n0 = 0, M = 0, L = 0;
    if (s < a.n_seqs) {
      n0 = a.seqs[s].n0;
      M = a.seqs[s + 1].n0 - n0;
      L = a.seqs[s].L;
    }
    const MxCut c = mx_cut(M, a.G, L, a.cuts);
    const int items = M > 0 ? c.n_sp * c.n_rg * a.pool.Hkv : 0;
    const int rec = M > 0 && c.n_sp > 1 ? M * a.Hq * c.n_sp : 0;
    const int upto = done + wave_prefix_sum(items), rec_upto = wave_prefix_sum(rec);
    const unsigned long long behind = __ballot(upto > item);
    if (behind != 0ull) {
      const int e = __builtin_ctzll(behind);
      w.s = a.seq0 + base + e;
      w.n0 = __builtin_amdgcn_readlane(n0, e);
      w.M = __builtin_amdgcn_readlane(M, e);
      w.L = __builtin_amdgcn_readlane(L, e);
      w.n_sp = __builtin_amdgcn_readlane(c.n_sp, e);
      w.pages = __builtin_amdgcn_readlane(c.pages, e);
      w.form = __builtin_amdgcn_readlane(c.form, e);
      w.rec0 = recs + __builtin_amdgcn_readlane(rec_upto, e) - __builtin_amdgcn_readlane(rec, e);
      mx_place(a, item - (__builtin_amdgcn_readlane(upto, e) - __builtin_amdgcn_readlane(items, e)), __builtin_amdgcn_readlane(c.n_blk, e),
               __builtin_amdgcn_readlane(c.n_rg, e), w);
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

// 16 bytes of each lane's own address straight into LDS, lane l's at `to` (the wave's) + 16 l.  The caller waits for them with vmcnt(0).
// (As a builtin the compiler waits for every load in flight ahead of each loop's first read of LDS.)
__device__ __forceinline__ void mx_to_lds(const void* from, char* to) {
  const unsigned at = __builtin_amdgcn_readfirstlane((unsigned)(uintptr_t)(__attribute__((address_space(3))) char*)to);
  unsigned saved;
  asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, off\n\ts_mov_b32 m0, %0" : "=&s"(saved) : "s"(at), "v"(from) : "memory");
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
  // The first scores of an item (accumulators and sum are zero): their maximum is the row's.
  __device__ __forceinline__ void start(const floatx16& S, float c2) {
    float top = fmaxf(S[0], S[1]);
#pragma unroll
    for (int v = 2; v < 16; ++v) top = fmaxf(top, S[v]);
    m = fmaxf(MXA_FLOOR, half_max(top) * c2);
  }
  // The maximum of the rows whose denominator reaches MX_LIMIT moves to the largest of a block's scores; the
  // other rows keep theirs, so that no row's rounding depends on its neighbours.
  __device__ __forceinline__ void move(const floatx16& S, float c2, float sum) {
    float top = fmaxf(S[0], S[1]);
#pragma unroll
    for (int v = 2; v < 16; ++v) top = fmaxf(top, S[v]);
    const bool moves = half_max(sum >= MX_LIMIT ? 1.f : 0.f) > 0.f;
    const float up = moves ? fmaxf(m, half_max(top) * c2) : m, alpha = exp2_fast(m - up);
    m = up;
    l *= alpha;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[t][v] *= alpha;
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
  __device__ __forceinline__ static bool over(float s) { return __ballot(s >= MX_LIMIT) != 0ull; }  // (a NaN stays one)
  // Rows (bits) of `wave`'s 32 whose sums left their range, for attn_mx_follow: [0] those of a denominator beyond MX_LIMIT (`over`: it
  // was), [1] those of an accumulator that is not finite although no score was a NaN (the denominator would be one).  `sum`: of both halves.
  __device__ __forceinline__ void note_lost(bool over, float sum, int wave, int lane, unsigned (*lost)[2]) const {
    float x = 0.f, y = 0.f;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int v = 0; v < 16; v += 2) x = __builtin_fmaf(acc[t][v], 0.f, x), y = __builtin_fmaf(acc[t][v + 1], 0.f, y);
    x += y;
    const unsigned long long beyond = __ballot(over || l >= MX_LIMIT), odd = __ballot(x != x && sum == sum);
    if (lane == 0) lost[wave][0] = (unsigned)beyond | (unsigned)(beyond >> 32), lost[wave][1] = (unsigned)odd | (unsigned)(odd >> 32);
  }
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

// Barrier of the workgroup for LDS; loads in flight stay in flight.
__device__ __forceinline__ void mx_meet() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// Tree row i and query head h of row r of a KV head (r / G < 1024 and G <= 1024: by a float product it is exact).
struct MxOwn {
  int i, h;
};
__device__ __forceinline__ MxOwn mx_own(const MxAttnArgs& a, const MxItem& it, int r) {
  const int i = (int)(((float)r + 0.5f) * a.inv_G);
  return MxOwn{i, it.g * a.G + (r - i * a.G)};
}
// Q: 32 rows from memory in whole rows into LDS (rows of 2 D + 16 bytes: 16 lanes that read a piece each, of 16 rows, meet 16
// banks).  (Every lane its own row's pieces from memory: 32 lines to a load, 3000 cycles where eight waves read the same rows.)
template <int D>
constexpr int MX_Q_ROW = 2 * D + 16;
template <int D>
__device__ __forceinline__ void mx_stage_q(const MxAttnArgs& a, const MxItem& it, int row_base, char* to, int first, int step) {
  const int Rh = a.G * it.M;
  for (int id = first; id < 32 * (D / 8); id += step) {
    const int r = id / (D / 8), c = id % (D / 8);
    const MxOwn o = mx_own(a, it, row_base + r < Rh ? row_base + r : Rh - 1);  // (rows behind the last repeat it)
    *reinterpret_cast<uint4*>(to + r * MX_Q_ROW<D> + c * 16) =
        *reinterpret_cast<const uint4*>(static_cast<const bf16_t*>(a.q) + (int64_t)(it.n0 + o.i) * a.q_stride + (int64_t)o.h * D + c * 8);
  }
}

// Root paths.  Trees of up to 64 rows: a wave finds all of them in registers, every row's mask of ancestors and pointer doubled
// until the pointers have left the tree, and keeps its rows' masks: no LDS, no barrier, as many rounds as the depth has
// binary digits (a walk through LDS took 3000 cycles for 8 rows and 6000 for 64).  Larger trees: hops in LDS (see mx_stage_tree),
// which a lane follows from its row up, a word of 32 tree rows at a time, as the tree's key blocks fall from call to call.
struct MxPath {
  unsigned lo, hi;  // small trees: the lane's row's path
  int cur;          // large ones: where it has got to
};
__device__ __forceinline__ void mx_small_paths(int parent, int M, int row, MxPath& path) {  // parent: of tree row `lane`
  const int lane = (int)(threadIdx.x & 63);
  unsigned lo = lane < 32 ? 1u << lane : 0u, hi = lane >= 32 ? 1u << (lane - 32) : 0u;
  int up = lane < M && parent >= 0 && parent < lane ? parent : -1;
  while (__ballot(up >= 0) != 0ull) {
    const int from = up >= 0 ? up : lane;
    lo |= (unsigned)__shfl((int)lo, from);
    hi |= (unsigned)__shfl((int)hi, from);
    const int next = __shfl(up, from);
    up = up >= 0 ? next : -1;
  }
  path.lo = (unsigned)__shfl((int)lo, row);
  path.hi = (unsigned)__shfl((int)hi, row);
}
// The tree's parents, requested early, and its hops in LDS, by the whole workgroup (a barrier inside and behind).
struct MxParents {
  int a, b;
};
__device__ __forceinline__ MxParents mx_request_parents(const MxAttnArgs& a, const MxItem& it) {
  const int32_t* const from = a.parent + it.n0;
  const int i = it.M <= 64 ? (int)(threadIdx.x & 63) : (int)threadIdx.x, j = i + MXA_THREADS;
  return MxParents{from[i < it.M ? i : 0], from[j < it.M ? j : 0]};
}
__device__ __forceinline__ void mx_stage_tree(const MxItem& it, const MxParents& mine, int* par, int2* hops) {
  if ((int)threadIdx.x < it.M) par[threadIdx.x] = mine.a;
  if ((int)threadIdx.x + MXA_THREADS < it.M) par[threadIdx.x + MXA_THREADS] = mine.b;
  mx_meet();
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
  mx_meet();
}
// The part of the path in tree rows 32 b .. 32 b + 31; b falls from call to call.
__device__ __forceinline__ unsigned mx_path_word(bool small, const int2* hops, MxPath& path, int b) {
  if (small) return b == 0 ? path.lo : path.hi;
  if (path.cur < 0 || (path.cur >> 5) != b) return 0u;
  const int2 hop = hops[path.cur];
  path.cur = hop.y;
  return (unsigned)hop.x;
}

// What a row's accumulators are multiplied by, ahead of any sum over waves or splits: their mean is in range where a sum need not be.
// (A split without weight, all its scores at -infinity, leaves a record of zeros.)
__device__ __forceinline__ float mx_inverse(float total, bool whole) { return whole || total > 0.f ? 1.f / total : 0.f; }

// Columns d .. d + 3 of a row: a result (the sequence has one split), or a part of the split's record.
__device__ __forceinline__ void mx_write4(const MxAttnArgs& a, bool whole, int64_t out, float* rec, int d, float4 sum) {
  if (whole) {
    const floatx2 lo = {sum.x, sum.y}, hi = {sum.z, sum.w};
    uint2 w;
    w.x = __builtin_bit_cast(unsigned, __builtin_convertvector(lo, bf16x2));
    w.y = __builtin_bit_cast(unsigned, __builtin_convertvector(hi, bf16x2));
    *reinterpret_cast<uint2*>(static_cast<bf16_t*>(a.o) + out * a.pool.D + d) = w;
  } else {
    *reinterpret_cast<float4*>(rec + d) = sum;
  }
}

// Columns D / 2 x .. D / 2 x + D / 2 - 1 of a wave's 32 rows, by way of its part of the tile buffers (rows as Q's): whole lines leave, 16 bytes to
// a lane.  (Every lane its own row's columns, 32 bytes to a line: 7000 cycles for 256 rows, this 3500.)
template <int D>
__device__ __forceinline__ void mx_write_half(const MxAttnArgs& a, const MxItem& it, int row_base, int x, const floatx16* acc, float inv, char* to, int lane) {
  constexpr int NT = D / 64;  // of 32 columns
  const int Rh = a.G * it.M, col = lane & 31, half = lane >> 5;
  char* const mine = to + col * MX_Q_ROW<D>;
  auto rows = [&](auto pieces, auto store) {
    constexpr int PIECES = decltype(pieces)::value;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    for (int id = lane; id < 32 * PIECES; id += 64) {
      const int r = id / PIECES, c = id % PIECES;
      if (row_base + r < Rh) store(mx_own(a, it, row_base + r), c, *reinterpret_cast<const uint4*>(to + r * MX_Q_ROW<D> + c * 16));
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  };
  if (it.n_sp == 1) {
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        const floatx2 lo = {acc[t][4 * b] * inv, acc[t][4 * b + 1] * inv}, hi = {acc[t][4 * b + 2] * inv, acc[t][4 * b + 3] * inv};
        uint2 w;
        w.x = __builtin_bit_cast(unsigned, __builtin_convertvector(lo, bf16x2));
        w.y = __builtin_bit_cast(unsigned, __builtin_convertvector(hi, bf16x2));
        *reinterpret_cast<uint2*>(mine + 64 * t + 16 * b + 8 * half) = w;
      }
    rows(std::integral_constant<int, D / 16>{}, [&](const MxOwn& o, int c, const uint4& w) {
      *reinterpret_cast<uint4*>(static_cast<bf16_t*>(a.o) + ((int64_t)(it.n0 + o.i) * a.Hq + o.h) * D + x * (D / 2) + 8 * c) = w;
    });
  } else {
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int b = 0; b < 4; ++b)
        *reinterpret_cast<float4*>(mine + 128 * t + 32 * b + 16 * half) =
            make_float4(acc[t][4 * b] * inv, acc[t][4 * b + 1] * inv, acc[t][4 * b + 2] * inv, acc[t][4 * b + 3] * inv);
    rows(std::integral_constant<int, D / 8>{}, [&](const MxOwn& o, int c, const uint4& w) {
      *reinterpret_cast<uint4*>(a.part + (it.rec0 + ((int64_t)o.i * a.Hq + o.h) * it.n_sp + it.sp) * (D + ATTN_REC_PAD) + x * (D / 2) + 4 * c) = w;
    });
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
  int odd;
  unsigned lost[MXA_WAVES][2];  // see MxState::note_lost
  unsigned nan_columns;
};
// Whether no wave noted a row.  (behind a barrier; the same for all waves)
template <int D>
__device__ __forceinline__ bool mx_none_lost(const MxLds<D>& mem) {
  return __ballot((&mem.lost[0][0])[threadIdx.x & (2 * MXA_WAVES - 1)] != 0u) == 0ull;
}

}  // namespace hs
