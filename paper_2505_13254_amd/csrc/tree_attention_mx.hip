// hs_tree_attention_mx: tree attention over a quantised cache (mx.h) and the tree's own bfloat16 rows.
//
// Per KV head the rows are r = i * G + gi (tree row i, member gi of its G query heads), in blocks of 32.  One workgroup of
// eight waves takes R row blocks of one (sequence, KV head, key split): wave w works for row block w % R on every
// (8 / R)-th 32 keys, alone: its keys go from memory into its registers, its softmax state is its own, and the waves of a
// row block meet once, at the end.
//
// Both products are computed transposed on the matrix cores (v_mfma_f32_32x32x16_bf16):
//     S^T[key, row] = K[key, :] . Q[row, :]         A = K, B = Q
//     O^T[d, row]  += V^T[d, key] P^T[key, row]     A = V, B = P
// so that a lane holds 16 scores of one row: the row's maximum and sum are in-lane plus one exchange of half-waves, and P is
// already laid out as the second product's operand.  A code times its scale is a bfloat16 without rounding, Q is used as
// it is, and the scale of the scores is applied to the float32 accumulator: the only roundings are P's to bfloat16 and the output's.
//
// K needs no LDS: which 8 elements of a row a lane's operand register holds is free as long as Q's agree, so a lane
// loads 16 bytes of codes of its own key and converts them in place.  V is converted in the order it is
// loaded, written to the wave's 8 KB of LDS and fetched from there with the transposing read.
//
// The running maximum moves only when a score exceeds it by more than 2^8 (P and the sums are floating point, so a late move
// costs no precision), which spares the rescaling of the accumulators in almost every step.
//
// Ancestor masks: every lane walks its row's root path from the row up, a word of 32 tree rows at a time, with the
// tree's key blocks taken from the last to the first.
#include <algorithm>

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
constexpr float MXA_LAZY = 8.f;       // octaves that a score may lie above the running maximum
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
  int pages_per_split, sp_max;
  float c2;              // scale * log2(e)
  void* o;
  float* lse;
  float* part;           // records of D + 4 floats: o (not normalised), maximum (in octaves), denominator
};

// The work item of this workgroup: items are numbered sequence by sequence, in a sequence
// (split * row groups + row group) * Hkv + KV head.  Every wave finds it by a prefix sum over the sequences.
struct MxItem {
  int s, n0, M, g, rg, sp, n_sp;
  int64_t L;
  int64_t rec0;  // records of the sequences before
};
template <int ROWS>
__device__ __forceinline__ bool mx_item(const MxAttnArgs& a, int item, MxItem& w) {
  const int lane = (int)(threadIdx.x & 63);
  int done = 0;
  int64_t recs = 0;
  for (int base = 0; base < a.B; base += 64) {
    const int s = base + lane;
    int n0 = 0, M = 0, n_sp = 0, items = 0, L = 0;
    if (s < a.B) {
      n0 = a.node_offsets[s];
      M = a.node_offsets[s + 1] - n0;
      L = (int)a.lens[s];
    }
    if (M > 0) {
      const int pages = (L + MX_PAGE - 1) / MX_PAGE;
      n_sp = (pages + a.pages_per_split - 1) / a.pages_per_split;
      n_sp = n_sp < 1 ? 1 : n_sp > a.sp_max ? a.sp_max : n_sp;
      items = n_sp * ((a.G * M + ROWS - 1) / ROWS) * a.pool.Hkv;
    }
    const int upto = done + wave_prefix_sum(items);
    const int rec = n_sp > 1 ? M * a.Hq * n_sp : 0;
    const int rec_upto = wave_prefix_sum(rec);
    const unsigned long long behind = __ballot(upto > item);
    if (behind != 0ull) {
      const int e = __builtin_ctzll(behind);
      w.s = base + e;
      w.n0 = __builtin_amdgcn_readlane(n0, e);
      w.M = __builtin_amdgcn_readlane(M, e);
      w.L = __builtin_amdgcn_readlane(L, e);
      w.n_sp = __builtin_amdgcn_readlane(n_sp, e);
      w.rec0 = recs + __builtin_amdgcn_readlane(rec_upto, e) - __builtin_amdgcn_readlane(rec, e);
      int local = item - (__builtin_amdgcn_readlane(upto, e) - __builtin_amdgcn_readlane(items, e));
      const int n_rg = (a.G * w.M + ROWS - 1) / ROWS;
      w.g = local % a.pool.Hkv;
      local /= a.pool.Hkv;
      w.rg = local % n_rg;
      w.sp = local / n_rg;
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
  // Scores (masked ones at -inf) to P: bfloat16 pairs of the first 16 and the second 16 keys.
  __device__ __forceinline__ void softmax(const floatx16& S, float c2, uint4& p0, uint4& p1) {
    float top = fmaxf(S[0], S[1]);
#pragma unroll
    for (int v = 2; v < 16; ++v) top = fmaxf(top, S[v]);
    top = half_max(top) * c2;
    if (__ballot(top > m + MXA_LAZY) != 0ull) {
      const float up = fmaxf(m, top), alpha = exp2_fast(m - up);
      m = up;
      l *= alpha;
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int v = 0; v < 16; ++v) acc[t][v] *= alpha;
    }
    unsigned w[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const floatx2 p = {exp2_fast(__builtin_fmaf(S[2 * j], c2, -m)), exp2_fast(__builtin_fmaf(S[2 * j + 1], c2, -m))};
      l += p[0] + p[1];
      w[j] = __builtin_bit_cast(unsigned, __builtin_convertvector(p, bf16x2));
    }
    p0 = make_uint4(w[0], w[1], w[2], w[3]);
    p1 = make_uint4(w[4], w[5], w[6], w[7]);
  }
};

template <int FMT, int D, int R>
__global__ __launch_bounds__(MXA_THREADS) void k_attn_mx(MxAttnArgs a) {
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
  constexpr int MERGE = MXA_WAVES * NT * 16 * 64 * 4;
  static_assert(MERGE >= MXA_WAVES * TILE, "the tiles lie in the memory of the merge");
  __shared__ __attribute__((aligned(16))) char lds[MERGE];
  __shared__ float den[MXA_WAVES][2][32];  // maxima and sums of the waves
  __shared__ int par[MXA_MAX_M];
  __shared__ int2 hops[MXA_MAX_M];  // of a tree row: its root path inside its own 32 rows as bits, the next row of it outside

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 31, half = lane >> 5;
  const int rb = wave % R, way = wave / R;
  MxItem it;
  if (!mx_item<32 * R>(a, blockIdx.x, it)) return;
  const int Rh = a.G * it.M;
  const int row_base = (it.rg * R + rb) * 32;
  const bool active = row_base < Rh;
  const int r_own = row_base + col < Rh ? row_base + col : Rh - 1;
  const int i_own = r_own / a.G, h_own = it.g * a.G + (r_own - i_own * a.G);
  const int64_t L = it.L;
  const bool last_split = it.sp == it.n_sp - 1;
  const int64_t k_lo = (int64_t)it.sp * a.pages_per_split * MX_PAGE;
  const int64_t k_hi = last_split ? L : k_lo + (int64_t)a.pages_per_split * MX_PAGE;
  const int n_blocks = (int)((k_hi - k_lo + 31) >> 5);  // 32-key blocks of the prefix part

  // ---- the tree's parents, for the split that has the tree
  if (last_split) {
    for (int j = tid; j < it.M; j += MXA_THREADS) par[j] = a.parent[it.n0 + j];
    __syncthreads();
    for (int j = tid; j < it.M; j += MXA_THREADS) {
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
    if (mine > 0) request(0);
    for (int j = 0; j < mine; ++j) {
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
      const int left = (int)(k_hi - k_lo - (int64_t)(way + j * W) * 32);  // keys of this block
      if (j + 1 < mine) request(j + 1);
      if (left < 32) {
#pragma unroll
        for (int v = 0; v < 16; ++v) S[v] = 8 * (v >> 2) + 4 * half + (v & 3) < left ? S[v] : -HS_INF;
      }
      uint4 p0, p1;
      st.softmax(S, a.c2, p0, p1);
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // the tile is read by other lanes than wrote it
      second(p0, p1);
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }

    // ---- the tree's own rows, block by block from the last that a row of this wave can see to the first
    if (last_split) {
      const int r_top = row_base + 31 < Rh ? row_base + 31 : Rh - 1;
      int cur = i_own;
      for (int b = (r_top / a.G) >> 5; b >= 0; --b) {
        unsigned word = 0;
        if (cur >= 0 && (cur >> 5) == b) {
          const int2 hop = hops[cur];
          word = (unsigned)hop.x;
          cur = hop.y;
        }
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
    const int d = 8 * x + 4 * half;  // 32 (x / 4) + 8 (x % 4) + 4 half
    if (it.n_sp == 1) {
      const floatx2 lo = {sum.x * inv, sum.y * inv}, hi = {sum.z * inv, sum.w * inv};
      uint2 w;
      w.x = __builtin_bit_cast(unsigned, __builtin_convertvector(lo, bf16x2));
      w.y = __builtin_bit_cast(unsigned, __builtin_convertvector(hi, bf16x2));
      *reinterpret_cast<uint2*>(static_cast<bf16_t*>(a.o) + out_row * D + d) = w;
    } else {
      *reinterpret_cast<float4*>(rec + d) = sum;
    }
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

// The splits of a (row, head) meet: D / 4 lanes each, four columns to a lane.
constexpr int MXM_THREADS = 256;
template <int D>
__global__ __launch_bounds__(MXM_THREADS) void k_attn_mx_merge(MxAttnArgs a, int64_t rows) {
  constexpr int LANES = D / 4, PER = MXM_THREADS / LANES;
  const int64_t x = (int64_t)blockIdx.x * PER + threadIdx.x / LANES;  // n * Hq + h
  const int d = 4 * (threadIdx.x % LANES);
  // the sequence, by the same prefix sums as the attention's
  const int n_first = (int)((int64_t)blockIdx.x * PER / a.Hq);
  const int lane = (int)(threadIdx.x & 63);
  int64_t recs = 0;
  for (int base = 0; base < a.B; base += 64) {
    const int s = base + lane;
    int n0 = 0x7fffffff, M = 0, n_sp = 0;
    if (s < a.B) {
      n0 = a.node_offsets[s];
      M = a.node_offsets[s + 1] - n0;
      const int pages = (int)((a.lens[s] + MX_PAGE - 1) / MX_PAGE);
      n_sp = (pages + a.pages_per_split - 1) / a.pages_per_split;
      n_sp = n_sp < 1 ? 1 : n_sp > a.sp_max ? a.sp_max : n_sp;
    }
    const int rec = n_sp > 1 ? M * a.Hq * n_sp : 0;
    const int upto = wave_prefix_sum(rec);
    // (a workgroup's rows may be of several sequences: each lane looks among those that the wave holds)
    for (int e = 0; e < 64 && base + e < a.B; ++e) {
      const int f0 = __builtin_amdgcn_readlane(n0, e), fm = __builtin_amdgcn_readlane(M, e), fs = __builtin_amdgcn_readlane(n_sp, e);
      if (f0 + fm <= n_first) continue;
      if ((int64_t)f0 * a.Hq >= (int64_t)(blockIdx.x + 1) * PER) return;
      const int64_t local = x - (int64_t)f0 * a.Hq;
      if (fs <= 1 || local < 0 || local >= (int64_t)fm * a.Hq || x >= rows) continue;
      const float* const from = a.part + (recs + __builtin_amdgcn_readlane(upto, e) - __builtin_amdgcn_readlane(rec, e) + local * fs) * (D + ATTN_REC_PAD);
      float top = MXA_FLOOR;
      for (int k = 0; k < fs; ++k) top = fmaxf(top, from[k * (D + ATTN_REC_PAD) + D]);
      float total = 0.f;
      float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int k = 0; k < fs; ++k) {
        const float* const r = from + k * (D + ATTN_REC_PAD);
        const float c = exp2_fast(r[D] - top);
        const float4 f = *reinterpret_cast<const float4*>(r + d);
        total += c * r[D + 1];
        sum.x += c * f.x, sum.y += c * f.y, sum.z += c * f.z, sum.w += c * f.w;
      }
      const float inv = 1.f / total;
      const floatx2 lo = {sum.x * inv, sum.y * inv}, hi = {sum.z * inv, sum.w * inv};
      uint2 w;
      w.x = __builtin_bit_cast(unsigned, __builtin_convertvector(lo, bf16x2));
      w.y = __builtin_bit_cast(unsigned, __builtin_convertvector(hi, bf16x2));
      *reinterpret_cast<uint2*>(static_cast<bf16_t*>(a.o) + x * D + d) = w;
      if (a.lse != nullptr && d == 0) a.lse[x] = (top + __log2f(total)) * MXA_LN2;
    }
    recs += __builtin_amdgcn_readlane(upto, 63);
  }
}

// ---- the plan: how many pages a split takes, from the host's row counts and lengths alone
constexpr int64_t MXA_RECORDS = 1 << 18;  // records that a call uses at most
struct MxPlan {
  int pages_per_split, sp_max;
  int64_t items, records;
};
static inline int mx_splits(int64_t L, int pages) {
  const int64_t n = ((L + MX_PAGE - 1) / MX_PAGE + pages - 1) / pages;
  return n < 1 ? 1 : (int)n;
}
static MxPlan mx_plan(const int32_t* hno, const int64_t* hlens, int B, int Hq, int Hkv, int rows_per_wg, int64_t max_records) {
  const int G = Hq / Hkv;
  int64_t max_L = 0;
  for (int s = 0; s < B; ++s)
    if (hno[s + 1] > hno[s]) max_L = std::max(max_L, hlens[s]);
  const int max_pages = (int)std::max<int64_t>(1, (max_L + MX_PAGE - 1) / MX_PAGE);
  MxPlan best = {max_pages, 1, 0, 0};
  for (int want = 1; want <= 64; ++want) {  // splits of the longest sequence
    const int pages = (max_pages + want - 1) / want;
    MxPlan p = {pages, mx_splits(max_L, pages), 0, 0};
    for (int s = 0; s < B; ++s) {
      const int64_t M = hno[s + 1] - hno[s];
      if (M <= 0) continue;
      const int n = mx_splits(hlens[s], pages);
      p.items += (int64_t)n * ((G * M + rows_per_wg - 1) / rows_per_wg) * Hkv;
      if (n > 1) p.records += M * Hq * n;
    }
    if (want > 1 && p.records > max_records) break;
    best = p;
    if (p.items >= 256) break;  // a workgroup to each compute unit
  }
  return best;
}

}  // namespace hs

using namespace hs;

static hs_status mx_attn_host_check(const int32_t* hno, const int64_t* hlens, int32_t B, int32_t Hq, int32_t Hkv, int32_t D) {
  HS_REQUIRE(B >= 0 && Hq >= 1 && Hkv >= 1, HS_ERR_SHAPE, "hs_tree_attention_mx: B=%d Hq=%d Hkv=%d", B, Hq, Hkv);
  HS_REQUIRE(Hq % Hkv == 0, HS_ERR_SHAPE, "hs_tree_attention_mx: Hq=%d is not a multiple of Hkv=%d", Hq, Hkv);
  HS_REQUIRE(D == 64 || D == 128, HS_ERR_UNSUPPORTED, "hs_tree_attention_mx: D=%d (64 and 128 are built)", D);
  if (B == 0) return HS_OK;
  HS_REQUIRE(hno && hlens, HS_ERR_NULL, "hs_tree_attention_mx: NULL host array");
  HS_REQUIRE(hno[0] == 0, HS_ERR_SHAPE, "hs_tree_attention_mx: node_offsets[0] = %d", hno[0]);
  for (int s = 0; s < B; ++s) {
    HS_REQUIRE(hno[s + 1] >= hno[s], HS_ERR_SHAPE, "hs_tree_attention_mx: node_offsets fall at sequence %d", s);
    HS_REQUIRE(hno[s + 1] - hno[s] <= MXA_MAX_M, HS_ERR_UNSUPPORTED, "hs_tree_attention_mx: sequence %d has %d tree rows (at most %d)", s,
               hno[s + 1] - hno[s], MXA_MAX_M);
    HS_REQUIRE(hlens[s] >= 0, HS_ERR_SHAPE, "hs_tree_attention_mx: prefix length %lld of sequence %d", (long long)hlens[s], s);
    HS_REQUIRE(hlens[s] <= HS_MX_MAX_TOKENS, HS_ERR_UNSUPPORTED, "hs_tree_attention_mx: sequence %d has %lld tokens", s, (long long)hlens[s]);
  }
  HS_REQUIRE((int64_t)hno[B] * Hq < ((int64_t)1 << 31), HS_ERR_UNSUPPORTED, "hs_tree_attention_mx: %d rows of %d heads", hno[B], Hq);
  return HS_OK;
}

static size_t mx_bytes(const MxPlan& p, int D) { return (size_t)p.records * (D + ATTN_REC_PAD) * sizeof(float); }

extern "C" size_t hs_tree_attention_mx_workspace(const int32_t* host_node_offsets, const int64_t* host_prefix_lens, int32_t B,
                                                 int32_t Hq, int32_t Hkv, int32_t D) {
  clear_error();
  if (mx_attn_host_check(host_node_offsets, host_prefix_lens, B, Hq, Hkv, D) != HS_OK || B == 0) return 0;
  return mx_bytes(mx_plan(host_node_offsets, host_prefix_lens, B, Hq, Hkv, 32, MXA_RECORDS), D);
}

extern "C" hs_status hs_tree_attention_mx(const void* q, int64_t q_stride, const void* k_codes, const void* k_scales,
                                          const void* v_codes, const void* v_scales, hs_mx_format fmt, const void* k_tree,
                                          int64_t k_stride, const void* v_tree, int64_t v_stride, const int32_t* parent,
                                          const int32_t* node_offsets, const int32_t* host_node_offsets,
                                          const int32_t* block_table, int32_t max_blocks, int32_t n_pages,
                                          const int64_t* prefix_lens, const int64_t* host_prefix_lens, int32_t B, int32_t Hq,
                                          int32_t Hkv, int32_t D, hs_dtype dt, float scale, void* o, float* lse, void* workspace,
                                          size_t workspace_bytes, hs_stream stream) {
  clear_error();
  const char* const what = "hs_tree_attention_mx";
  hs_status st = mx_attn_host_check(host_node_offsets, host_prefix_lens, B, Hq, Hkv, D);
  if (st != HS_OK) return st;
  HS_REQUIRE(dt == HS_F32 || dt == HS_BF16, HS_ERR_SHAPE, "%s: unknown dtype %d", what, (int)dt);
  HS_REQUIRE(dt == HS_BF16, HS_ERR_UNSUPPORTED, "%s: bfloat16 rows only", what);
  HS_REQUIRE(scale > 0.f && scale < 1e30f, HS_ERR_UNSUPPORTED, "%s: scale %g (positive scales are built)", what, (double)scale);
  MxAttnArgs a = {};
  auto bytes = [](const void* p) { return static_cast<unsigned char*>(const_cast<void*>(p)); };
  a.pool = MxPool{bytes(k_codes), bytes(k_scales), bytes(v_codes), bytes(v_scales), block_table, max_blocks, n_pages, Hkv, D};
  st = mx_pool_check(what, a.pool, fmt);
  if (st != HS_OK) return st;
  const int32_t NN = B > 0 ? host_node_offsets[B] : 0;
  if (NN == 0) return HS_OK;
  int64_t tokens = 0;
  for (int s = 0; s < B; ++s) {
    if (host_node_offsets[s + 1] == host_node_offsets[s]) continue;
    tokens += host_prefix_lens[s];
    HS_REQUIRE(host_prefix_lens[s] <= (int64_t)max_blocks * MX_PAGE, HS_ERR_SHAPE, "%s: %lld tokens of sequence %d do not fit %d blocks", what,
               (long long)host_prefix_lens[s], s, max_blocks);
  }
  HS_REQUIRE(q && k_tree && v_tree && parent && node_offsets && prefix_lens && o, HS_ERR_NULL, "%s: NULL argument", what);
  if (tokens > 0) {
    st = mx_pool_pointers(what, a.pool);
    if (st != HS_OK) return st;
    HS_REQUIRE(n_pages >= 1, HS_ERR_SHAPE, "%s: prefix tokens, but no pages", what);
  }
  HS_REQUIRE(q_stride >= (int64_t)Hq * D && k_stride >= (int64_t)Hkv * D && v_stride >= (int64_t)Hkv * D, HS_ERR_SHAPE,
             "%s: a row stride is less than heads * D", what);
  HS_REQUIRE(((reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(k_tree) | reinterpret_cast<uintptr_t>(v_tree) | reinterpret_cast<uintptr_t>(o)) & 15) == 0 &&
                 (q_stride | k_stride | v_stride) % 8 == 0,
             HS_ERR_UNSUPPORTED, "%s: rows must begin at multiples of 16 bytes", what);
  a.q = q, a.k_tree = k_tree, a.v_tree = v_tree, a.q_stride = q_stride, a.k_stride = k_stride, a.v_stride = v_stride;
  a.parent = parent, a.node_offsets = node_offsets, a.lens = prefix_lens;
  a.B = B, a.Hq = Hq, a.G = Hq / Hkv;
  a.c2 = scale * MXA_LOG2E;
  a.o = o, a.lse = lse, a.part = static_cast<float*>(workspace);
  const MxPlan p = mx_plan(host_node_offsets, host_prefix_lens, B, Hq, Hkv, 32, MXA_RECORDS);
  HS_REQUIRE(p.items < ((int64_t)1 << 31), HS_ERR_UNSUPPORTED, "%s: too many rows for one call", what);
  const size_t need = mx_bytes(p, D);
  if (need > 0) {
    HS_REQUIRE(workspace && reinterpret_cast<uintptr_t>(workspace) % 256 == 0 && workspace_bytes >= need, HS_ERR_WORKSPACE,
               "%s: workspace of %zu bytes, %zu are needed (256-byte aligned)", what, workspace_bytes, need);
  }
  a.pages_per_split = p.pages_per_split, a.sp_max = p.sp_max;
  const dim3 grid((unsigned)p.items), block(MXA_THREADS);
#define MXA_LAUNCH(F, DD) hipLaunchKernelGGL((k_attn_mx<F, DD, 1>), grid, block, 0, static_cast<hipStream_t>(stream), a)
  if (fmt == HS_MX_E4M3) {
    if (D == 128) MXA_LAUNCH(HS_MX_E4M3, 128);
    else MXA_LAUNCH(HS_MX_E4M3, 64);
  } else {
    if (D == 128) MXA_LAUNCH(HS_MX_E2M1, 128);
    else MXA_LAUNCH(HS_MX_E2M1, 64);
  }
#undef MXA_LAUNCH
  st = launch_status(what);
  if (st != HS_OK || p.records == 0) return st;
  const int64_t rows = (int64_t)NN * Hq;
  if (D == 128)
    hipLaunchKernelGGL((k_attn_mx_merge<128>), dim3((unsigned)((rows + 7) / 8)), dim3(MXM_THREADS), 0, static_cast<hipStream_t>(stream), a, rows);
  else
    hipLaunchKernelGGL((k_attn_mx_merge<64>), dim3((unsigned)((rows + 15) / 16)), dim3(MXM_THREADS), 0, static_cast<hipStream_t>(stream), a, rows);
  return launch_status(what);
}
