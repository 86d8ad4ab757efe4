// Attention over latents (internal): what the two calls hand to their kernels.
//
// Absorbed form: every query head of a tree row scores the same keys, a token's latent c [R] and rotary part r [Dr], and the values
// are the latents themselves.  Expanded form: every head has keys [Dn] and values [Dv] of its own, the rotary part is shared.
#pragma once
#include <string.h>

#include "attn_common.h"

namespace hs {

struct LatRows {  // [rows, heads, n] with strides of its own, in elements
  const void* p;
  int64_t row, head;
};

struct LatTreeArgs {
  LatRows q, q_rope;
  const void* pool;  // [n_pages, 64, R + Dr]
  const void* c_tree;
  const void* r_tree;
  int64_t c_stride, r_stride;
  const int32_t* parent;
  const int32_t* node_offsets;
  const int32_t* table;
  int max_blocks, n_pages;
  const int64_t* prefix_lens;
  int B, NN, Hq, R, Dr;
  float scale;
  void* o;
  int64_t o_row, o_head;
  float* lse;
};

struct LatPromptArgs {
  LatRows q, q_rope, k, v;
  const void* k_rope;
  int64_t k_rope_row;
  const int32_t* q_offsets;
  const int64_t* kv_offsets;
  int B, N, H, Dn, Dr, Dv;
  float scale;
  void* o;
  int64_t o_row, o_head;
  float* lse;
};

// latent_attn_tree.hip: bfloat16, R = 512, Dr = 64, everything aligned to 16 bytes, on the matrix cores.
constexpr int64_t LAT_MAX_RECORDS = (int64_t)1 << 22;  // (8.7 GB of 512 columns)
struct LatPlan {
  int per;       // pages of a split at most
  int sp_max;    // splits of a sequence at most
  int group;     // rows of an item at most
  int64_t first[9];  // the first item of each XCD, and the number of items
  int64_t grid;      // workgroups
  int64_t records;   // of the rows of sequences with several splits, one to a split
};
// The last plan of a thread (the layers of a step ask for the same one, and so does a call after its workspace query): of calls of up to 4096 sequences.
template <LatPlan (*PLAN)(const int32_t*, const int64_t*, int32_t, int32_t), int LENS>
LatPlan lat_remember(const int32_t* rows, const int64_t* lens, int32_t B, int32_t heads) {
  constexpr int MOST = 4096;
  static thread_local struct {
    int32_t B = -1, heads;
    int32_t rows[MOST + 1];
    int64_t lens[MOST + 1];
    LatPlan plan;
  } last;
  if (B > MOST) return PLAN(rows, lens, B, heads);
  const size_t n = sizeof(int32_t) * (size_t)(B + 1), m = sizeof(int64_t) * (size_t)(B + LENS);
  if (last.B != B || last.heads != heads || memcmp(last.rows, rows, n) != 0 || memcmp(last.lens, lens, m) != 0) {
    last.plan = PLAN(rows, lens, B, heads);
    last.B = B;
    last.heads = heads;
    memcpy(last.rows, rows, n);
    memcpy(last.lens, lens, m);
  }
  return last.plan;
}
bool lat_tree_matrix(const LatTreeArgs& a, hs_dtype dt);
LatPlan lat_tree_plan(const int32_t* host_node_offsets, const int64_t* host_prefix_lens, int32_t B, int32_t Hq);
size_t lat_tree_bytes(const LatPlan& p);
hs_status lat_tree_launch(const LatTreeArgs& a, const LatPlan& p, int one_len, void* workspace, hipStream_t stream);  // one_len: B == 1, the stored tokens

// latent_attn_prompt.hip: bfloat16, Dn = 128, Dr = 64, Dv = 128, everything aligned to 16 bytes, on the matrix cores.  (A plan's `per` are tiles of 64 keys, `grid`
// the items.)
bool lat_prompt_matrix(const LatPromptArgs& a, hs_dtype dt);
LatPlan lat_prompt_plan(const int32_t* host_q_offsets, const int64_t* host_kv_offsets, int32_t B, int32_t H);
size_t lat_prompt_bytes(const LatPlan& p);
hs_status lat_prompt_launch(const LatPromptArgs& a, const LatPlan& p, int one_len, void* workspace, hipStream_t stream);  // one_len: B == 1, the keys

// What a launch may have of workgroups (a grid's threads are counted in 32 bits); a call of more, of very many short sequences, takes the other kernel.
constexpr int64_t LAT_MAX_GRID = (int64_t)1 << 22;

// latent_attn_any.hip: any shape and type, float32 arithmetic throughout.
hs_status lat_tree_any(const LatTreeArgs& a, hs_dtype dt, hipStream_t stream);
hs_status lat_prompt_any(const LatPromptArgs& a, hs_dtype dt, hipStream_t stream);

}  // namespace hs
