// hs_tree_attention_mx: tree attention over a quantised cache (mx.h) and the tree's own bfloat16 rows.
//
// Per KV head the rows are r = i * G + gi (tree row i, member gi of its G query heads), in blocks of 32.  A workgroup of
// eight waves takes a group of one to eight row blocks of one (sequence, KV head, key split); how its waves share the work
// depends on the size of the group (attn_mx.h: the cut; attn_mx_private.h, attn_mx_shared.h: the two kinds).
//
// Both products are computed transposed on the matrix cores (v_mfma_f32_32x32x16_bf16):
//     S^T[key, row] = K[key, :] . Q[row, :]         A = K, B = Q
//     O^T[d, row]  += V^T[d, key] P^T[key, row]     A = V, B = P
// so that a lane holds 16 scores of one row: the row's maximum and sum are in-lane plus one exchange of half-waves, and P is
// already laid out as the second product's operand.  A code times its scale is a bfloat16 without rounding, Q is used as
// it is, and the scale of the scores is applied to the float32 accumulator: the only roundings are P's to bfloat16 and the output's.  P's is
// a choice: a second product in more bits would be two of them (P as a sum of two bfloat16), for an error against 64 bits of 0.0016 of the
// outputs' norm, the output's own rounding, instead of 0.0022 to 0.0024 (trees and batches above).
//
// Ancestor masks: of trees of up to 64 rows every wave finds all root paths in registers; of larger ones a lane walks its row's
// path from the row up, a word of 32 tree rows at a time, with the tree's key blocks taken from the last to the first.
//
// What bounds it (D = 128, 8 KV heads, us of this kernel): one row to a sequence is a stream of the cache, 64 sequences of 512 to 16384
// tokens in e4m3 (601 MB) 117, 5.1 TB/s: three rounds of items, of whose time a sixth is their start and end, and 6.9 TB/s between (with
// codes requested a whole step ahead, into LDS, it is no faster); 776 rows to a KV head are matrix
// work, 4 x 8192 tokens in e2m1 122 (0.85 PFLOP/s; a full group of eight blocks runs at 1.35); one tree of 61 rows on 2048 tokens is a
// chain of latencies, 13.7: 1 to know its item, 2 for Q and the pages, 1.5 for the tree, 0.3 a page, 2 to add up the waves, and 4 for the merge.
#include <algorithm>
#include <cmath>

#include "attn_mx.h"

namespace hs {

void attn_mx_launch_e4m3(const MxAttnArgs& a, unsigned items, hipStream_t stream);
void attn_mx_launch_e2m1(const MxAttnArgs& a, unsigned items, hipStream_t stream);

// The splits of a (row, head) meet: a wave each, whose lanes first find the splits' weights, a split to a lane, and then add up
// the records, D / 4 lanes and four columns to a lane to each of 64 / (D / 4) records at a time.  Rows first .. first + rows - 1 of n * Hq + h.
constexpr int MXM_THREADS = 256;
template <int D>
__global__ __launch_bounds__(MXM_THREADS) void k_attn_mx_merge(MxAttnArgs a, int row0, int rows) {
  constexpr int LANES = D / 4, AT_ONCE = 64 / LANES;
  const int lane = (int)(threadIdx.x & 63);
  const int at = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * (MXM_THREADS / 64) + (threadIdx.x >> 6)));
  if (at >= rows) return;
  const int64_t x = row0 + at;  // n * Hq + h  (less than 2^26 of them)
  const int n = (int)(x / a.Hq);
  // its sequence and the records before
  int64_t recs = 0, first = -1;
  int n_sp = 0;
  if (a.n_entries > 0) {
    const int4 lo = *reinterpret_cast<const int4*>(&a.entries[lane]), hi = *(reinterpret_cast<const int4*>(&a.entries[lane]) + 1);
    const unsigned long long mine = __ballot(lane < a.n_entries && lo.y <= n && n < lo.y + lo.z);
    if (mine == 0ull) return;
    const int e = __builtin_ctzll(mine);
    n_sp = __builtin_amdgcn_readlane(hi.y, e) & 255;
    first = __builtin_amdgcn_readlane(hi.w, e) + (x - (int64_t)__builtin_amdgcn_readlane(lo.y, e) * a.Hq) * n_sp;
  }
  for (int base = 0; a.n_entries == 0 && base < a.n_seqs; base += 64) {
    const int s = base + lane;
    int n0 = 0, M = 0, sp = 0;
    if (s < a.n_seqs) {
      n0 = a.seqs[s].n0;
      M = a.seqs[s + 1].n0 - n0;
      sp = mx_cut(M, a.G, a.seqs[s].L, a.cuts).n_sp;
    }
    const int rec = M > 0 && sp > 1 ? M * a.Hq * sp : 0;
    const int upto = wave_prefix_sum(rec);
    const unsigned long long mine = __ballot(M > 0 && n0 <= n && n < n0 + M);
    if (mine != 0ull) {
      const int e = __builtin_ctzll(mine);
      n_sp = __builtin_amdgcn_readlane(sp, e);
      first = recs + __builtin_amdgcn_readlane(upto, e) - __builtin_amdgcn_readlane(rec, e) + (x - (int64_t)__builtin_amdgcn_readlane(n0, e) * a.Hq) * n_sp;
      break;
    }
    recs += __builtin_amdgcn_readlane(upto, 63);
  }
  if (n_sp <= 1) return;
  const float* const from = a.part + first * (D + ATTN_REC_PAD);
  const int d = 4 * (lane % LANES), k0 = lane / LANES;
  float4 f[4];
  auto fetch = [&](int k) {  // (behind the last record: the last one again, at weight 0)
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int at = k + u * AT_ONCE + k0;
      f[u] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (k + u * AT_ONCE < n_sp) f[u] = *reinterpret_cast<const float4*>(from + (at < n_sp ? at : n_sp - 1) * (D + ATTN_REC_PAD) + d);
    }
  };
  const int sp = lane < n_sp ? lane : 0;  // (at most 64 splits)
  const float2 ml = *reinterpret_cast<const float2*>(from + sp * (D + ATTN_REC_PAD) + D);
  fetch(0);  // (the first records with their maxima: one trip to memory)
  const float m = lane < n_sp ? ml.x : MXA_FLOOR, l = lane < n_sp ? ml.y : 0.f;
  const float top = wave_max(m), part = exp2_fast(m - top) * l, total = wave_sum(part), weight = part * (1.f / total);
  float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int k = 0;;) {
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int at = k + u * AT_ONCE + k0;
      const float c = __shfl(weight, at & 63);
      if (at < n_sp) sum.x += c * f[u].x, sum.y += c * f[u].y, sum.z += c * f[u].z, sum.w += c * f[u].w;
    }
    k += 4 * AT_ONCE;
    if (k >= n_sp) break;
    fetch(k);
  }
#pragma unroll
  for (int o = LANES; o < 64; o *= 2) {
    sum.x += __shfl_xor(sum.x, o), sum.y += __shfl_xor(sum.y, o), sum.z += __shfl_xor(sum.z, o), sum.w += __shfl_xor(sum.w, o);
  }
  if (k0 == 0) {
    const floatx2 lo = {sum.x, sum.y}, hi = {sum.z, sum.w};
    uint2 w;
    w.x = __builtin_bit_cast(unsigned, __builtin_convertvector(lo, bf16x2));
    w.y = __builtin_bit_cast(unsigned, __builtin_convertvector(hi, bf16x2));
    *reinterpret_cast<uint2*>(static_cast<bf16_t*>(a.o) + x * D + d) = w;
  }
  if (a.lse != nullptr && lane == 0) a.lse[x] = (top + __log2f(total)) * MXA_LN2;
}

// ---- the plan
// A call's work is cut for the shortest estimated time.  What an item takes is a fixed part and one in proportion to its
// pages, measured (D = 128) on 256 workgroups at once, where the memory and the clock give less to each, and on up to half as many.
// Of a list of times that an item may take (a page less or more in it moves whole rounds of items) every sequence cuts itself
// for the least total, or, where the call does not fill the chip, for the shortest items, and the best estimate of the call is taken: the
// total over the compute units, the longest item, and for every k the k + 1 rounds that 256 k + 1 items of some size need at least;
// items run longest first.
constexpr int64_t MXA_RECORDS = 1 << 18;  // records that a call uses at most
constexpr double MX_ITEM_US[4] = {5.5, 6.5, 9.0, 11.0};         // an item, by form
constexpr double MX_PAGE_FREE_US[4] = {0.30, 0.60, 0.92, 1.27};  // a page of it, by form: up to 128 items
constexpr double MX_PAGE_FULL_US[2][9] = {{0.0, 0.63, 0.89, 1.17, 1.34, 1.66, 1.79, 1.88, 1.99},   // 256 items, by row blocks, e4m3
                                          {0.0, 0.37, 0.73, 0.94, 1.05, 1.29, 1.40, 1.52, 1.59}};  // e2m1
struct MxSeqPlan {
  MxCut cut;
  int s;
  int64_t items;
  double free_us, full_us;  // its longest item
};
struct MxPlan {
  MxCuts cuts;                  // B > MXA_ENTRIES: of all
  MxSeqPlan seq[MXA_ENTRIES];   // otherwise: each, longest items first
  int n_seq;
  int64_t items, records;
};
static void mx_seq_plan(int M, int G, int L, int Hkv, int D, int fmt, int most, double us, MxSeqPlan& p, double& total) {
  MxCut c = mx_groups(M, G, most);
  const double per = D == 128 ? 1.0 : 0.5, fixed = MX_ITEM_US[c.form];
  // (the row groups of a sequence share what its keys cost the memory, which is what e4m3 takes longer than e2m1)
  const int size = c.n_rg == 1 ? c.n_blk : (c.n_blk + c.n_rg - 1) / c.n_rg;
  const double full = (MX_PAGE_FULL_US[1][size] + (MX_PAGE_FULL_US[fmt][size] - MX_PAGE_FULL_US[1][size]) / c.n_rg) * per;
  mx_splits(M, L, us > 1e8 ? 1 << 20 : std::max(1, (int)((us - fixed) / full)), c);
  const int all = (L + MX_PAGE - 1) / MX_PAGE + (M + MX_PAGE - 1) / MX_PAGE, longest = std::min(all, c.pages + (c.n_sp == 1 ? all : 0));
  p.cut = c;
  p.items = (int64_t)c.n_sp * c.n_rg * Hkv;
  p.free_us = fixed + longest * MX_PAGE_FREE_US[c.form] * per;
  p.full_us = fixed + longest * full;
  total = (double)c.n_rg * Hkv * (c.n_sp * fixed + all * full);
}
static void mx_plan(const int32_t* hno, const int64_t* hlens, int B, int Hq, int Hkv, int D, int fmt, MxPlan& best) {
  const int G = Hq / Hkv;
  const bool each = B <= MXA_ENTRIES;
  MxPlan p;
  double best_us = 1e30, most_work = 0.0;
  best.items = best.records = 0, best.n_seq = 0;
  // the sequences looked at: all, or of those that are cut on the device an even choice of 64, for the others too, and the one with the most work
  int look[MXA_ENTRIES + 1], n_look = 0, most_blk = 0;
  double others = 1.0;
  if (each) {
    for (int s = 0; s < B; ++s)
      if (hno[s + 1] > hno[s]) look[n_look++] = s;
  } else {
    int n = 0, largest = 0;
    double work = -1.0;
    for (int s = 0; s < B; ++s) {
      const int n_blk = (int)(((int64_t)G * (hno[s + 1] - hno[s]) + 31) >> 5);
      if (n_blk == 0) continue;
      ++n;
      most_blk = std::max(most_blk, n_blk);
      if ((double)n_blk * (double)(hlens[s] + MX_PAGE) > work) work = (double)n_blk * (double)(hlens[s] + MX_PAGE), largest = s;
    }
    const int step = (n + MXA_ENTRIES - 1) / MXA_ENTRIES;
    for (int s = 0, at = 0; s < B; ++s)
      if (hno[s + 1] > hno[s] && at++ % step == 0) look[n_look++] = s;
    if (n_look > 0) {
      others = (double)n / n_look;
      look[n_look++] = largest;
    }
  }
  const int tries = each ? std::max(11, std::min(15, 256 / std::max(1, B))) : 7;
  const double ratio = tries == 15 ? 1.154 : std::pow(5.6, 1.0 / (tries - 3));
  double us = 1e9, longest_item = 0.0;
  for (int t = 0; t < tries; ++t) {  // uncut (twice: then the work is known), then from 1.4 times an equal share (or 11 us) down to a quarter
    for (int most = each ? 8 : 1; most <= 8; most *= 2) {  // (sequences that are cut on the device share the size of their groups)
      p.items = p.records = 0, p.n_seq = 0;
      p.cuts.blocks_most = most;
      for (int f = 0; f < 4; ++f) p.cuts.pages[f] = us > 1e8 ? 1 << 20 : std::max(1, (int)((us - MX_ITEM_US[f]) / (MX_PAGE_FULL_US[fmt][1 << f] * (D == 128 ? 1.0 : 0.5))));
      double total = 0.0, longest = 0.0;
      for (int i = 0; i < n_look; ++i) {
        const int s = look[i], M = hno[s + 1] - hno[s];
        const double share = each || i + 1 == n_look ? 1.0 : others;
        MxSeqPlan now = {}, q;
        double least = 1e30, least_score = 1e30, one;
        if (each) {
          const int n_blk = (G * M + 31) >> 5;
          for (int m = 1;; m *= 2) {
            mx_seq_plan(M, G, (int)hlens[s], Hkv, D, fmt, m, us, q, one);
            const double score = std::max(most_work, t == 0 ? 0.0 : q.free_us) + one / 256.0;
            if (score < least_score) least_score = score, least = one, now = q;
            if (m >= n_blk || m == 8) break;
          }
          now.s = s;
          p.seq[p.n_seq++] = now;
        } else {
          mx_seq_plan(M, G, (int)hlens[s], Hkv, D, fmt, most, us, now, least);
          const MxCut c = mx_cut(M, G, (int)hlens[s], p.cuts);
          now.items = (int64_t)c.n_sp * c.n_rg * Hkv;
          now.cut = c;
        }
        p.items += now.items;
        if (now.cut.n_sp > 1) p.records += (int64_t)(share * (double)((int64_t)M * Hq * now.cut.n_sp));
        total += share * least;
        longest = std::max(longest, now.full_us);
      }
      if (t == 0) most_work = total / 256.0;
      if (us < 1e8 && p.records > MXA_RECORDS) {
        if (!each && most >= most_blk) break;
        continue;
      }
      double took = std::max(total / 256.0, 0.0);
      if (each) {
        if (p.n_seq > 1) std::sort(p.seq, p.seq + p.n_seq, [](const MxSeqPlan& a, const MxSeqPlan& b) { return a.full_us > b.full_us || (a.full_us == b.full_us && a.s < b.s); });
        const double load = std::min(1.0, std::max(0.0, (double)(p.items - 128) / 128.0));
        int64_t at = 0, k = 0;
        for (int i = 0; i < p.n_seq; ++i) {
          const MxSeqPlan& q = p.seq[i];
          if (i == 0) took = std::max(took, q.free_us + (q.full_us - q.free_us) * load);
          at += q.items;
          if (k == 0) k = 1;
          while (at > 256 * k && k < 64) took = std::max(took, (double)(++k) * q.full_us);
        }
      } else {
        took += longest * 0.5;
      }
      longest_item = longest;
      took += p.records > 0 ? 4.0 + p.records * 2.2e-4 : 0.0;
      if (took < best_us) {
        best_us = took;
        best.cuts = p.cuts, best.n_seq = p.n_seq, best.items = p.items, best.records = p.records;
        std::copy(p.seq, p.seq + p.n_seq, best.seq);
      }
      if (!each && most >= most_blk) break;
    }
    // (where no item is longer than half of a share, or than a cut one and the merge, cuts gain little: not worth the host's time for many
    // sequences; 64 short ones 33 -> 16 us a call)
    if (t == 1 && n_look > 8 && longest_item <= std::max(0.5 * most_work, 10.0)) break;
    us = t == 0 ? us : t == 1 ? std::max(8.0, most_work) * 1.4 : us / ratio;
  }
  for (bool again = !each && n_look > 0; again;) {  // what that cut comes to, of all
    again = false;
    best.items = best.records = 0;
    for (int s = 0; s < B; ++s) {
      const int M = hno[s + 1] - hno[s];
      if (M <= 0) continue;
      const MxCut c = mx_cut(M, G, (int)hlens[s], best.cuts);
      best.items += (int64_t)c.n_sp * c.n_rg * Hkv;
      if (c.n_sp > 1) best.records += (int64_t)M * Hq * c.n_sp;
    }
    if (best.records > MXA_RECORDS) {  // (the choice said fewer: uncut there are none)
      for (int f = 0; f < 4; ++f) best.cuts.pages[f] = 1 << 20;
      again = true;
    }
  }
}

}  // namespace hs

using namespace hs;

static hs_status mx_attn_host_check(const int32_t* hno, const int64_t* hlens, int32_t B, int32_t Hq, int32_t Hkv, int32_t D) {
  HS_REQUIRE(B >= 0 && Hq >= 1 && Hkv >= 1, HS_ERR_SHAPE, "hs_tree_attention_mx: B=%d Hq=%d Hkv=%d", B, Hq, Hkv);
  HS_REQUIRE(Hq % Hkv == 0, HS_ERR_SHAPE, "hs_tree_attention_mx: Hq=%d is not a multiple of Hkv=%d", Hq, Hkv);
  HS_REQUIRE(D == 64 || D == 128, HS_ERR_UNSUPPORTED, "hs_tree_attention_mx: D=%d (64 and 128 are built)", D);
  HS_REQUIRE(Hq / Hkv <= 1024 && Hkv <= 4096, HS_ERR_UNSUPPORTED, "hs_tree_attention_mx: Hq=%d Hkv=%d", Hq, Hkv);
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
  HS_REQUIRE((int64_t)hno[B] * Hq < ((int64_t)1 << 26), HS_ERR_UNSUPPORTED, "hs_tree_attention_mx: %d rows of %d heads", hno[B], Hq);
  return HS_OK;
}

static size_t mx_bytes(const MxPlan& p, int D) { return (size_t)p.records * (D + ATTN_REC_PAD) * sizeof(float); }

extern "C" size_t hs_tree_attention_mx_workspace(const int32_t* host_node_offsets, const int64_t* host_prefix_lens, int32_t B,
                                                 int32_t Hq, int32_t Hkv, int32_t D) {
  clear_error();
  if (mx_attn_host_check(host_node_offsets, host_prefix_lens, B, Hq, Hkv, D) != HS_OK || B == 0) return 0;
  size_t need = 0;  // of either format
  MxPlan p;
  for (int fmt = 0; fmt < 2; ++fmt) {
    mx_plan(host_node_offsets, host_prefix_lens, B, Hq, Hkv, D, fmt, p);
    need = std::max(need, mx_bytes(p, D));
  }
  return need;
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
  a.parent = parent;
  a.Hq = Hq, a.G = Hq / Hkv, a.inv_G = 1.f / (float)(Hq / Hkv);
  a.c2 = scale * MXA_LOG2E;
  a.o = o, a.lse = lse;
  MxPlan p;
  mx_plan(host_node_offsets, host_prefix_lens, B, Hq, Hkv, D, (int)fmt, p);
  HS_REQUIRE(p.items < ((int64_t)1 << 23), HS_ERR_UNSUPPORTED, "%s: too many rows for one call", what);  // (2^32 threads)
  const size_t need = mx_bytes(p, D);
  if (need > 0) {
    HS_REQUIRE(workspace && reinterpret_cast<uintptr_t>(workspace) % 256 == 0 && workspace_bytes >= need, HS_ERR_WORKSPACE,
               "%s: workspace of %zu bytes, %zu are needed (256-byte aligned)", what, workspace_bytes, need);
  }
  a.cuts = p.cuts;
  a.part = static_cast<float*>(workspace);
  // One launch of all items, and one more where splits meet.  (rows: of the launch's sequences)
  auto launch = [&](int64_t items, int64_t records, int n_first, int n_end) {
    if (items == 0) return HS_OK;
    (fmt == HS_MX_E4M3 ? attn_mx_launch_e4m3 : attn_mx_launch_e2m1)(a, (unsigned)items, static_cast<hipStream_t>(stream));
    const hs_status failed = launch_status(what);
    if (failed != HS_OK || records == 0) return failed;
    const int row0 = n_first * Hq, rows = (n_end - n_first) * Hq;
    const dim3 grid((unsigned)((rows + MXM_THREADS / 64 - 1) / (MXM_THREADS / 64)));
    if (D == 128) hipLaunchKernelGGL((k_attn_mx_merge<128>), grid, dim3(MXM_THREADS), 0, static_cast<hipStream_t>(stream), a, row0, rows);
    else hipLaunchKernelGGL((k_attn_mx_merge<64>), grid, dim3(MXM_THREADS), 0, static_cast<hipStream_t>(stream), a, row0, rows);
    return launch_status(what);
  };
  if (B <= MXA_ENTRIES) {
    a.n_entries = p.n_seq;
    for (int e = 0, first = 0, rec0 = 0; e < a.n_entries; ++e) {
      const MxCut& c = p.seq[e].cut;
      const int s = p.seq[e].s, n0 = host_node_offsets[s], M = host_node_offsets[s + 1] - n0;
      a.entries[e] = MxEntry{first, n0, M, (int)host_prefix_lens[s], c.pages, c.n_sp | c.form << 8 | s << 16, (int)((unsigned)c.n_blk | (unsigned)c.n_rg << 16), rec0};
      first += c.n_sp * c.n_rg * Hkv, rec0 += c.n_sp > 1 ? M * Hq * c.n_sp : 0;
    }
    return launch(p.items, p.records, 0, NN);
  }
  // (the launches share a cut, and the workspace one after the other)
  const int parts = (B + MXA_SEQS - 1) / MXA_SEQS, each = (B + parts - 1) / parts;
  for (int s0 = 0; s0 < B; s0 += each) {
    a.seq0 = s0, a.n_seqs = std::min(each, B - s0);
    int64_t items = 0, records = 0;
    for (int i = 0; i <= a.n_seqs; ++i) {
      const int s = s0 + i;
      a.seqs[i] = MxSeq{host_node_offsets[s], i < a.n_seqs ? (int)host_prefix_lens[s] : 0};
      const int M = i < a.n_seqs ? host_node_offsets[s + 1] - host_node_offsets[s] : 0;
      if (M == 0) continue;
      const MxCut c = mx_cut(M, a.G, (int)host_prefix_lens[s], a.cuts);
      items += (int64_t)c.n_sp * c.n_rg * Hkv, records += c.n_sp > 1 ? (int64_t)M * Hq * c.n_sp : 0;
    }
    st = launch(items, records, host_node_offsets[s0], host_node_offsets[s0 + a.n_seqs]);
    if (st != HS_OK) return st;
  }
  return HS_OK;
}
