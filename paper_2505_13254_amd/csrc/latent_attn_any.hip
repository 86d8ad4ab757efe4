// Attention over latents, any shape and type.
//
// o = softmax_j(scale (q . k_j + q_rope . r_j)) . v_j in float32, one pass over the keys with the running maximum and sum of a
// softmax.  A workgroup of four waves has one (row, query head); each wave takes every fourth 64 keys.  A lane has a key for the
// scores (the query stands in LDS, one broadcast read to 64 products) and every 64th column for the values.  Keys that a row does not
// see are skipped, not multiplied by zero, so that nothing in them reaches it; a score of -infinity is a weight of zero that is multiplied, so that an infinity
// in its value does.  The waves' sums meet in LDS.
//
// Bound by the vector pipe and by reads of a key a lane: what float32, and shapes without matrix-core kernels, take.
// (bfloat16, one row of 16 heads on 2048 tokens of 512 + 64: 642 us, where the matrix cores take 15.)
#include "latent_attn.h"

namespace hs {

constexpr int LA_THREADS = 256, LA_WAVES = 4;
constexpr int LA_MOST = 1024;  // columns of a value
constexpr float LA_FLOOR = -__FLT_MAX__;

template <typename T>
__device__ __forceinline__ float la_at(const T* p, int64_t i);
template <>
__device__ __forceinline__ float la_at<float>(const float* p, int64_t i) { return p[i]; }
template <>
__device__ __forceinline__ float la_at<bf16_t>(const bf16_t* p, int64_t i) { return bf16_to_f32(p[i]); }

// `tiles` 64-key tiles; seen(t) -> the bits of the keys of tile t that the row sees (the same for all lanes); key(t, j, &k, &r, &v): the
// addresses of key j of tile t.
template <typename T, typename Seen, typename Key>
__device__ __forceinline__ void la_row(const T* q, int a_n, const T* qr, int b_n, int v_n, int64_t tiles, float scale, T* o, float* lse, Seen seen, Key key) {
  __shared__ float q_lds[2 * LA_MOST], p_lds[LA_WAVES][64], out[LA_WAVES][LA_MOST], stat[LA_WAVES][2];
  __shared__ int some[LA_WAVES];
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  for (int x = tid; x < a_n + b_n; x += LA_THREADS) q_lds[x] = x < a_n ? la_at(q, x) : la_at(qr, x - a_n);
  __syncthreads();
  float acc[LA_MOST / 64], m = LA_FLOOR, l = 0.f;
  bool any = false;  // the wave's keys that the row sees: is there one?
#pragma unroll
  for (int x = 0; x < LA_MOST / 64; ++x) acc[x] = 0.f;
  for (int64_t t = wave; t < tiles; t += LA_WAVES) {
    const unsigned long long bits = seen(t);
    if (bits == 0ull) continue;
    any = true;
    const bool on = (bits >> lane) & 1ull;
    float s = -HS_INF;
    if (on) {
      const T *k, *r, *v;
      key(t, lane, &k, &r, &v);
      float sum = 0.f;
      for (int x = 0; x < a_n; ++x) sum = __builtin_fmaf(q_lds[x], la_at(k, x), sum);
      for (int x = 0; x < b_n; ++x) sum = __builtin_fmaf(q_lds[a_n + x], la_at(r, x), sum);
      s = sum * scale;
    }
    const float up = fmaxf(m, wave_max(s)), old = __expf(m - up);  // (a NaN among the scores is not the largest, and makes the sum one)
    const float p = on ? __expf(s - up) : 0.f;
    m = up;
    l = l * old + wave_sum(p);
    p_lds[wave][lane] = p;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
    for (int x = 0; x < LA_MOST / 64; ++x) acc[x] *= old;
    for (unsigned long long left = bits; left != 0ull; left &= left - 1) {
      const int j = __builtin_ctzll(left);
      const T *k, *r, *v;
      key(t, j, &k, &r, &v);
      const float w = p_lds[wave][j];
#pragma unroll
      for (int x = 0; x < LA_MOST / 64; ++x)
        if (64 * x + lane < v_n) acc[x] = __builtin_fmaf(w, la_at(v, 64 * x + lane), acc[x]);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }
  if (lane == 0) stat[wave][0] = m, stat[wave][1] = l, some[wave] = any;
#pragma unroll
  for (int x = 0; x < LA_MOST / 64; ++x)
    if (64 * x + lane < v_n) out[wave][64 * x + lane] = acc[x];
  __syncthreads();
  float top = stat[0][0], total = 0.f, f[LA_WAVES];
#pragma unroll
  for (int w = 1; w < LA_WAVES; ++w) top = fmaxf(top, stat[w][0]);
#pragma unroll
  for (int w = 0; w < LA_WAVES; ++w) f[w] = __expf(stat[w][0] - top), total += f[w] * stat[w][1];
  bool none = true;  // no key at all.  (Keys whose scores are all -infinity have no weight either: they give 0 / 0.)
#pragma unroll
  for (int w = 0; w < LA_WAVES; ++w) none = none && !some[w];
  for (int x = tid; x < v_n; x += LA_THREADS) {
    float y = 0.f;
#pragma unroll
    for (int w = 0; w < LA_WAVES; ++w) y = __builtin_fmaf(f[w], out[w][x], y);  // (of a wave without keys 0; of scores of -infinity 0 too, or the NaN of 0 x infinity)
    store_elem(o + x, none ? 0.f : y / total);
  }
  if (tid == 0 && lse != nullptr) *lse = none ? -HS_INF : top + __logf(total);
}

template <typename T>
__global__ __launch_bounds__(LA_THREADS) void k_lat_tree_any(LatTreeArgs a) {
  const int64_t id = blockIdx.x;
  const int n = (int)(id / a.Hq), h = (int)(id - (int64_t)n * a.Hq);
  int lo = 0, hi = a.B;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (a.node_offsets[mid] <= n) lo = mid;
    else hi = mid;
  }
  const int s = lo, n0 = a.node_offsets[s], i = n - n0;
  const int64_t most = (int64_t)a.max_blocks * 64, len = a.prefix_lens[s], L = len < 0 ? 0 : (len > most ? most : len), pages = (L + 63) >> 6;
  const int W = a.R + a.Dr;
  const int32_t* const parent = a.parent + n0;
  auto seen = [&](int64_t t) -> unsigned long long {
    if (t < pages) return L - 64 * t >= 64 ? ~0ull : ~0ull >> (64 - (L - 64 * t));
    unsigned long long bits = 0ull;
    const int base = (int)(t - pages) * 64;
    for (int j = i; j >= base;) {
      if (j < base + 64) bits |= 1ull << (j - base);
      const int up = parent[j];
      j = up < j ? up : -1;  // (a malformed tree cannot keep the walk from ending)
    }
    return bits;
  };
  auto key = [&](int64_t t, int j, const T** k, const T** r, const T** v) {
    if (t < pages) {
      const int p = a.table[(int64_t)s * a.max_blocks + t];
      *k = static_cast<const T*>(a.pool) + ((int64_t)(p < 0 || p >= a.n_pages ? 0 : p) * 64 + j) * W;  // (an entry that is no page would be a caller's error)
      *r = *k + a.R;
    } else {
      const int64_t row = n0 + (t - pages) * 64 + j;
      *k = static_cast<const T*>(a.c_tree) + row * a.c_stride;
      *r = static_cast<const T*>(a.r_tree) + row * a.r_stride;
    }
    *v = *k;
  };
  la_row<T>(static_cast<const T*>(a.q.p) + n * a.q.row + h * a.q.head, a.R, static_cast<const T*>(a.q_rope.p) + n * a.q_rope.row + h * a.q_rope.head, a.Dr, a.R,
            pages + i / 64 + 1, a.scale, static_cast<T*>(a.o) + n * a.o_row + h * a.o_head, a.lse == nullptr ? nullptr : a.lse + id, seen, key);
}

template <typename T>
__global__ __launch_bounds__(LA_THREADS) void k_lat_prompt_any(LatPromptArgs a) {
  const int64_t id = blockIdx.x;
  const int n = (int)(id / a.H), h = (int)(id - (int64_t)n * a.H);
  int lo = 0, hi = a.B;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (a.q_offsets[mid] <= n) lo = mid;
    else hi = mid;
  }
  const int s = lo;
  const int64_t k0 = a.kv_offsets[s], keys = a.kv_offsets[s + 1] - k0;
  const int64_t most = keys - (a.q_offsets[s + 1] - 1 - n);  // keys that the row sees
  const int64_t L = most < 0 ? 0 : most;
  auto seen = [&](int64_t t) { return L - 64 * t >= 64 ? ~0ull : ~0ull >> (64 - (L - 64 * t)); };
  auto key = [&](int64_t t, int j, const T** k, const T** r, const T** v) {
    const int64_t row = k0 + 64 * t + j;
    *k = static_cast<const T*>(a.k.p) + row * a.k.row + h * a.k.head;
    *r = static_cast<const T*>(a.k_rope) + row * a.k_rope_row;
    *v = static_cast<const T*>(a.v.p) + row * a.v.row + h * a.v.head;
  };
  la_row<T>(static_cast<const T*>(a.q.p) + n * a.q.row + h * a.q.head, a.Dn, static_cast<const T*>(a.q_rope.p) + n * a.q_rope.row + h * a.q_rope.head, a.Dr, a.Dv,
            (L + 63) >> 6, a.scale, static_cast<T*>(a.o) + n * a.o_row + h * a.o_head, a.lse == nullptr ? nullptr : a.lse + id, seen, key);
}

hs_status lat_tree_any(const LatTreeArgs& a, hs_dtype dt, hipStream_t stream) {
  const unsigned grid = (unsigned)a.NN * (unsigned)a.Hq;
  if (dt == HS_F32) hipLaunchKernelGGL(k_lat_tree_any<float>, dim3(grid), dim3(LA_THREADS), 0, stream, a);
  else hipLaunchKernelGGL(k_lat_tree_any<bf16_t>, dim3(grid), dim3(LA_THREADS), 0, stream, a);
  return launch_status("latent attention");
}

hs_status lat_prompt_any(const LatPromptArgs& a, hs_dtype dt, hipStream_t stream) {
  const unsigned grid = (unsigned)a.N * (unsigned)a.H;
  if (dt == HS_F32) hipLaunchKernelGGL(k_lat_prompt_any<float>, dim3(grid), dim3(LA_THREADS), 0, stream, a);
  else hipLaunchKernelGGL(k_lat_prompt_any<bf16_t>, dim3(grid), dim3(LA_THREADS), 0, stream, a);
  return launch_status("latent prompt attention");
}

}  // namespace hs
