// hs_tree_attention_latent, hs_prompt_attention_latent: checks of the arguments, and which kernel a call takes.
#include "latent_attn.h"

namespace hs {

constexpr int LAT_MAX_TREE = 1024;
constexpr int64_t LAT_MAX_TOKENS = HS_MX_MAX_TOKENS;
constexpr int64_t LAT_MAX_ROWS = (int64_t)1 << 24;  // (row, head) pairs of a call
constexpr int64_t LAT_MAX_STRIDE = (int64_t)1 << 38;

static bool lat_strides(int64_t row, int64_t head) { return row >= 0 && head >= 0 && row < LAT_MAX_STRIDE && head < LAT_MAX_STRIDE; }

// Rows of an output [N, H, n] that do not overlap: heads inside a row, or rows inside a head.
static bool lat_apart(int64_t N, int64_t H, int64_t n, int64_t row, int64_t head) {
  if (!lat_strides(row, head)) return false;
  if (N <= 1) return H <= 1 || head >= n;
  if (H <= 1) return row >= n;
  return (head >= n && row >= (H - 1) * head + n) || (row >= n && head >= (N - 1) * row + n);
}

// What a call's host arrays say of its trees and lengths.
static hs_status lat_tree_hosts(const int32_t* no, const int64_t* pl, int32_t B, int32_t max_blocks) {
  HS_REQUIRE(no[0] == 0, HS_ERR_SHAPE, "hs_tree_attention_latent: host_node_offsets[0] must be 0");
  for (int s = 0; s < B; ++s) {
    HS_REQUIRE(no[s + 1] >= no[s], HS_ERR_SHAPE, "hs_tree_attention_latent: host_node_offsets decrease at %d", s);
    HS_REQUIRE(no[s + 1] - no[s] <= LAT_MAX_TREE, HS_ERR_UNSUPPORTED, "hs_tree_attention_latent: sequence %d has %d tree rows, at most %d", s, no[s + 1] - no[s],
               LAT_MAX_TREE);
    HS_REQUIRE(pl[s] >= 0 && pl[s] <= (int64_t)max_blocks * 64, HS_ERR_SHAPE, "hs_tree_attention_latent: sequence %d has %lld tokens in %d pages", s,
               (long long)pl[s], max_blocks);
    HS_REQUIRE(pl[s] <= LAT_MAX_TOKENS, HS_ERR_UNSUPPORTED, "hs_tree_attention_latent: sequence %d has %lld tokens", s, (long long)pl[s]);
  }
  return HS_OK;
}

// The same of a call on prompts.
static hs_status lat_prompt_hosts(const int32_t* qo, const int64_t* ko, int32_t B) {
  HS_REQUIRE(qo[0] == 0 && ko[0] == 0, HS_ERR_SHAPE, "hs_prompt_attention_latent: offsets must begin with 0");
  for (int s = 0; s < B; ++s) {
    HS_REQUIRE(qo[s + 1] >= qo[s] && ko[s + 1] >= ko[s], HS_ERR_SHAPE, "hs_prompt_attention_latent: offsets decrease at %d", s);
    HS_REQUIRE(ko[s + 1] - ko[s] <= LAT_MAX_TOKENS, HS_ERR_UNSUPPORTED, "hs_prompt_attention_latent: sequence %d has %lld keys", s, (long long)(ko[s + 1] - ko[s]));
  }
  return HS_OK;
}

}  // namespace hs

using namespace hs;

extern "C" size_t hs_tree_attention_latent_workspace(const int32_t* host_node_offsets, const int64_t* host_prefix_lens, int32_t B, int32_t Hq, int32_t R,
                                                     int32_t Dr) {
  clear_error();
  if (B < 1 || Hq < 1 || host_node_offsets == nullptr || host_prefix_lens == nullptr || R != 512 || Dr != 64) return 0;
  if (lat_tree_hosts(host_node_offsets, host_prefix_lens, B, 0x7fffffff) != HS_OK || (int64_t)host_node_offsets[B] * Hq >= LAT_MAX_ROWS) return 0;
  return lat_tree_bytes(lat_remember<lat_tree_plan, 0>(host_node_offsets, host_prefix_lens, B, Hq));
}

extern "C" hs_status hs_tree_attention_latent(const void* q, int64_t q_stride, int64_t q_head_stride, const void* q_rope, int64_t q_rope_stride,
                                              int64_t q_rope_head_stride, const void* pool, const void* c_tree, int64_t c_stride, const void* r_tree,
                                              int64_t r_stride, const int32_t* parent, const int32_t* node_offsets, const int32_t* host_node_offsets,
                                              const int32_t* block_table, int32_t max_blocks, int32_t n_pages, const int64_t* prefix_lens,
                                              const int64_t* host_prefix_lens, int32_t B, int32_t Hq, int32_t R, int32_t Dr, hs_dtype dt, float scale, void* o,
                                              int64_t o_stride, int64_t o_head_stride, float* lse, void* workspace, size_t workspace_bytes, hs_stream stream) {
  clear_error();
  HS_REQUIRE(B >= 0 && Hq >= 1 && R >= 1 && Dr >= 0 && max_blocks >= 0 && n_pages >= 0, HS_ERR_SHAPE,
             "hs_tree_attention_latent: B=%d Hq=%d R=%d Dr=%d max_blocks=%d n_pages=%d", B, Hq, R, Dr, max_blocks, n_pages);
  HS_REQUIRE(dt == HS_F32 || dt == HS_BF16, HS_ERR_SHAPE, "hs_tree_attention_latent: unknown dtype %d", (int)dt);
  HS_REQUIRE(scale > 0.f && scale < HS_INF, HS_ERR_SHAPE, "hs_tree_attention_latent: scale must be positive");
  HS_REQUIRE(R <= 1024 && Dr <= 1024, HS_ERR_UNSUPPORTED, "hs_tree_attention_latent: R and Dr must be at most 1024");
  if (B == 0) return HS_OK;
  HS_REQUIRE(host_node_offsets && host_prefix_lens, HS_ERR_NULL, "hs_tree_attention_latent: NULL host array");
  const hs_status st = lat_tree_hosts(host_node_offsets, host_prefix_lens, B, max_blocks);
  if (st != HS_OK) return st;
  const int NN = host_node_offsets[B];
  if (NN == 0) return HS_OK;
  HS_REQUIRE((int64_t)NN * Hq < LAT_MAX_ROWS, HS_ERR_UNSUPPORTED, "hs_tree_attention_latent: rows times heads must be below 2^24");
  bool stored = false;
  for (int s = 0; s < B; ++s) stored = stored || (host_prefix_lens[s] > 0 && host_node_offsets[s + 1] > host_node_offsets[s]);
  HS_REQUIRE(!stored || n_pages > 0, HS_ERR_SHAPE, "hs_tree_attention_latent: stored tokens without pages");
  HS_REQUIRE(q && (q_rope || Dr == 0) && c_tree && (r_tree || Dr == 0) && parent && node_offsets && prefix_lens && o && (!stored || (pool && block_table)),
             HS_ERR_NULL, "hs_tree_attention_latent: NULL argument");
  HS_REQUIRE(lat_strides(q_stride, q_head_stride) && lat_strides(q_rope_stride, q_rope_head_stride) && lat_strides(c_stride, r_stride), HS_ERR_SHAPE,
             "hs_tree_attention_latent: strides must be within 0 .. 2^38");
  HS_REQUIRE(lat_apart(NN, Hq, R, o_stride, o_head_stride), HS_ERR_SHAPE, "hs_tree_attention_latent: rows of the output overlap (strides %lld, %lld)",
             (long long)o_stride, (long long)o_head_stride);
  LatTreeArgs a = {{q, q_stride, q_head_stride}, {q_rope, q_rope_stride, q_rope_head_stride}, pool, c_tree, r_tree, c_stride, r_stride, parent, node_offsets,
                   block_table, max_blocks, n_pages, prefix_lens, B, NN, Hq, R, Dr, scale, o, o_stride, o_head_stride, lse};
  if (!lat_tree_matrix(a, dt)) return lat_tree_any(a, dt, static_cast<hipStream_t>(stream));
  const LatPlan p = lat_remember<lat_tree_plan, 0>(host_node_offsets, host_prefix_lens, B, Hq);
  if (p.grid >= LAT_MAX_GRID) return lat_tree_any(a, dt, static_cast<hipStream_t>(stream));
  const size_t need = lat_tree_bytes(p);
  HS_REQUIRE(need == 0 || (workspace != nullptr && workspace_bytes >= need && reinterpret_cast<uintptr_t>(workspace) % 256 == 0), HS_ERR_WORKSPACE,
             "hs_tree_attention_latent: needs %zu bytes of workspace, got %zu", need, workspace_bytes);
  return lat_tree_launch(a, p, (int)host_prefix_lens[0], workspace, static_cast<hipStream_t>(stream));
}

extern "C" size_t hs_prompt_attention_latent_workspace(const int32_t* host_q_offsets, const int64_t* host_kv_offsets, int32_t B, int32_t H, int32_t Dv) {
  clear_error();
  if (B < 1 || H < 1 || Dv != 128 || host_q_offsets == nullptr || host_kv_offsets == nullptr) return 0;
  if (lat_prompt_hosts(host_q_offsets, host_kv_offsets, B) != HS_OK || (int64_t)host_q_offsets[B] * H >= LAT_MAX_ROWS) return 0;
  return lat_prompt_bytes(lat_remember<lat_prompt_plan, 1>(host_q_offsets, host_kv_offsets, B, H));
}

extern "C" hs_status hs_prompt_attention_latent(const void* q, int64_t q_stride, int64_t q_head_stride, const void* q_rope, int64_t q_rope_stride,
                                                int64_t q_rope_head_stride, const void* k, int64_t k_stride, int64_t k_head_stride, const void* k_rope,
                                                int64_t k_rope_stride, const void* v, int64_t v_stride, int64_t v_head_stride, const int32_t* q_offsets,
                                                const int64_t* kv_offsets, const int32_t* host_q_offsets, const int64_t* host_kv_offsets, int32_t B, int32_t H,
                                                int32_t Dn, int32_t Dr, int32_t Dv, hs_dtype dt, float scale, void* o, int64_t o_stride, int64_t o_head_stride,
                                                float* lse, void* workspace, size_t workspace_bytes, hs_stream stream) {
  clear_error();
  HS_REQUIRE(B >= 0 && H >= 1 && Dn >= 1 && Dr >= 0 && Dv >= 1, HS_ERR_SHAPE, "hs_prompt_attention_latent: B=%d H=%d Dn=%d Dr=%d Dv=%d", B, H, Dn, Dr, Dv);
  HS_REQUIRE(dt == HS_F32 || dt == HS_BF16, HS_ERR_SHAPE, "hs_prompt_attention_latent: unknown dtype %d", (int)dt);
  HS_REQUIRE(scale > 0.f && scale < HS_INF, HS_ERR_SHAPE, "hs_prompt_attention_latent: scale must be positive");
  HS_REQUIRE(Dn <= 1024 && Dr <= 1024 && Dv <= 1024, HS_ERR_UNSUPPORTED, "hs_prompt_attention_latent: Dn, Dr and Dv must be at most 1024");
  if (B == 0) return HS_OK;
  HS_REQUIRE(host_q_offsets && host_kv_offsets, HS_ERR_NULL, "hs_prompt_attention_latent: NULL host array");
  const hs_status st = lat_prompt_hosts(host_q_offsets, host_kv_offsets, B);
  if (st != HS_OK) return st;
  bool any = false;
  for (int s = 0; s < B; ++s) any = any || (host_q_offsets[s + 1] > host_q_offsets[s] && host_kv_offsets[s + 1] > host_kv_offsets[s]);
  const int N = host_q_offsets[B];
  if (N == 0) return HS_OK;
  HS_REQUIRE((int64_t)N * H < LAT_MAX_ROWS, HS_ERR_UNSUPPORTED, "hs_prompt_attention_latent: rows times heads must be below 2^24");
  HS_REQUIRE(q && (q_rope || Dr == 0) && q_offsets && kv_offsets && o && (!any || (k && v && (k_rope || Dr == 0))), HS_ERR_NULL,
             "hs_prompt_attention_latent: NULL argument");
  HS_REQUIRE(lat_strides(q_stride, q_head_stride) && lat_strides(q_rope_stride, q_rope_head_stride) && lat_strides(k_stride, k_head_stride) &&
                 lat_strides(v_stride, v_head_stride) && lat_strides(k_rope_stride, 0),
             HS_ERR_SHAPE, "hs_prompt_attention_latent: strides must be within 0 .. 2^38");
  HS_REQUIRE(lat_apart(N, H, Dv, o_stride, o_head_stride), HS_ERR_SHAPE, "hs_prompt_attention_latent: rows of the output overlap (strides %lld, %lld)",
             (long long)o_stride, (long long)o_head_stride);
  LatPromptArgs a = {{q, q_stride, q_head_stride}, {q_rope, q_rope_stride, q_rope_head_stride}, {k, k_stride, k_head_stride}, {v, v_stride, v_head_stride}, k_rope,
                     k_rope_stride, q_offsets, kv_offsets, B, N, H, Dn, Dr, Dv, scale, o, o_stride, o_head_stride, lse};
  if (!lat_prompt_matrix(a, dt)) return lat_prompt_any(a, dt, static_cast<hipStream_t>(stream));
  const LatPlan p = lat_remember<lat_prompt_plan, 1>(host_q_offsets, host_kv_offsets, B, H);
  if (p.grid >= LAT_MAX_GRID) return lat_prompt_any(a, dt, static_cast<hipStream_t>(stream));
  const size_t need = lat_prompt_bytes(p);
  HS_REQUIRE(need == 0 || (workspace != nullptr && workspace_bytes >= need && reinterpret_cast<uintptr_t>(workspace) % 256 == 0), HS_ERR_WORKSPACE,
             "hs_prompt_attention_latent: needs %zu bytes of workspace, got %zu", need, workspace_bytes);
  return lat_prompt_launch(a, p, (int)host_kv_offsets[1], workspace, static_cast<hipStream_t>(stream));
}
