// hs_rotary, hs_tree_rotary: rotary positions of query and key rows.
//
// Pair j of a head's first `rot` elements is turned by the angle p * inv_freq[j], p the row's position:
//   (a, b) -> mscale * (a cos - b sin, b cos + a sin)
// with (a, b) = elements (j, j + rot / 2), or (2j, 2j + 1).  All heads of a row share its angles.
//
// The angle is formed in double precision as a number of turns, of which the whole ones are dropped before the rest
// becomes a float (2^-26 of a turn; float32 results are 4.7e-8 of their norm off, 3.6e-8 with 64 bits to the end): of position 10^6 a
// float product would be off by up to 0.06 radians.  Sine and cosine are computed
// once per row and pair and shared through LDS, so that the rest is a copy with four multiply-adds to a pair: bound by memory.
#include "mx.h"

namespace hs {

constexpr int ROT_THREADS = 256;
constexpr int ROT_MANY = 2048;    // rows from which on a workgroup takes as many as it has threads for (9 heads of 64, bfloat16: 5.9 us
                                  // instead of 11.2 for 8192 rows, 36 instead of 80 for 65536; at 2048 either way 5)
constexpr int ROT_STAGE = 1024;   // tree rows whose parents are staged in LDS

struct RotaryArgs {
  const void* in[2];   // q, k
  void* out[2];
  int64_t in_stride[2], out_stride[2];  // elements from row to row
  int heads[2];
  int N, D, rot, tokens;
  const int64_t* positions;     // [N], or
  const int32_t* parent;        // trees: position = prefix_lens[s] + depth
  const int32_t* node_offsets;
  const int64_t* prefix_lens;
  int B;
  const double* inv_freq;
  float mscale;
};

// 16 bytes: four float32 or eight bfloat16
template <typename T>
constexpr int ROT_WIDE = 16 / (int)sizeof(T);
template <typename T>
__device__ __forceinline__ void values(const uint4& a, float* f) {
  const unsigned w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 4) {
      f[i] = __builtin_bit_cast(float, w[i]);
    } else {
      f[2 * i] = __builtin_bit_cast(float, w[i] << 16);
      f[2 * i + 1] = __builtin_bit_cast(float, w[i] & 0xffff0000u);
    }
  }
}
__device__ __forceinline__ void store16(float* p, const float* f) { *reinterpret_cast<float4*>(p) = make_float4(f[0], f[1], f[2], f[3]); }
__device__ __forceinline__ void store16(bf16_t* p, const float* f) {
  unsigned w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = (unsigned)f32_to_bf16(f[2 * i]) | ((unsigned)f32_to_bf16(f[2 * i + 1]) << 16);
  *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ float elem(const float* p) { return *p; }
__device__ __forceinline__ float elem(const bf16_t* p) { return bf16_to_f32(*p); }

// Depth of tree row i, counted by the whole workgroup: every row's distance to the row it points to and that
// pointer are doubled until the pointers have left the tree (a chain of 1024 rows takes ten rounds).
__device__ int tree_depth(const int32_t* parent, int i, int2* hop) {
  __shared__ int found[2];
  const int n = i < ROT_STAGE ? i + 1 : ROT_STAGE;  // (parents are earlier rows: the first i + 1 rows hold the path)
  if (threadIdx.x == 0) {
    int far = 0, j = i;  // rows beyond the stage are walked one by one
    while (j >= ROT_STAGE) {
      const int up = parent[j];
      const bool edge = up >= 0 && up < j;
      far += edge ? 1 : 0;
      j = edge ? up : -1;
    }
    found[0] = far;
    found[1] = j;
  }
  for (int r = threadIdx.x; r < n; r += ROT_THREADS) {
    const int up = parent[r];
    hop[r] = up >= 0 && up < r ? make_int2(1, up) : make_int2(0, -1);
  }
  __syncthreads();
  constexpr int PER = ROT_STAGE / ROT_THREADS;
  for (int span = 1; span < n; span *= 2) {
    int2 next[PER];
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      const int r = threadIdx.x + k * ROT_THREADS;
      if (r < n) {
        next[k] = hop[r];
        if (next[k].y >= 0) {
          const int2 up = hop[next[k].y];
          next[k] = make_int2(next[k].x + up.x, up.y);
        }
      }
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      const int r = threadIdx.x + k * ROT_THREADS;
      if (r < n) hop[r] = next[k];
    }
    __syncthreads();
  }
  return found[0] + (found[1] >= 0 ? hop[found[1]].x : 0);
}

// PAIRS: 0 = halves, 1 = neighbours.  VEC: 16 bytes at a time (aligned rows, pairs in whole eights).
template <typename T, int PAIRS, bool TREE, bool VEC>
__global__ __launch_bounds__(ROT_THREADS) void k_rotary(RotaryArgs a) {
  extern __shared__ __attribute__((aligned(16))) char lds_raw[];
  const int h = a.rot >> 1;
  float* const c_lds = reinterpret_cast<float*>(lds_raw);  // [tokens][h]
  float* const s_lds = c_lds + a.tokens * h;
  const int tid = threadIdx.x;
  const int n0 = blockIdx.x * a.tokens;
  const int n_here = a.N - n0 < a.tokens ? a.N - n0 : a.tokens;
  const int heads = a.heads[0] + a.heads[1];
  // what a head is made of: `turned` units that hold pairs, then units behind the turned part
  constexpr int WIDE = ROT_WIDE<T>, width = VEC ? WIDE : 1;
  const int turned = VEC && PAIRS == 1 ? a.rot / WIDE : h / width;
  const int units = turned + (a.D - a.rot) / width;
  // (row t, head, unit x) of this thread, and the step to its next one: the divisions are done once
  const int per_row = heads * units;
  int t = tid / per_row, head_t = (tid - t * per_row) / units, x = tid - t * per_row - head_t * units;
  const int step_t = ROT_THREADS / per_row, step_h = (ROT_THREADS - step_t * per_row) / units, step_x = ROT_THREADS - step_t * per_row - step_h * units;
  auto next = [&]() {
    x += step_x, head_t += step_h, t += step_t;
    if (x >= units) x -= units, ++head_t;
    if (head_t >= heads) head_t -= heads, ++t;
  };
  auto angles = [&]() {  // false: the row lies behind the last sequence
    int64_t tree_pos = 0;
    if constexpr (TREE) {  // (one row to a workgroup)
      const int end = a.node_offsets[a.B];
      const int s = seq_of_row(a.node_offsets, a.B, n0);
      const int first = a.node_offsets[s];
      if (n0 >= end) return false;
      tree_pos = a.prefix_lens[s] + tree_depth(a.parent + first, n0 - first, reinterpret_cast<int2*>(lds_raw + 8 * h));
    }
    for (int u = tid; u < n_here * h; u += ROT_THREADS) {
      const int t = u / h, j = u - t * h;
      const int64_t p = TREE ? tree_pos : a.positions[n0 + t];
      const double turns = (double)p * (a.inv_freq[j] * 0.15915494309189533577);  // 1 / (2 pi)
      const float rest = (float)(turns - rint(turns));
      float sn, cs;
      sincospif(2.f * rest, &sn, &cs);
      c_lds[u] = cs * a.mscale;
      s_lds[u] = sn * a.mscale;
    }
    __syncthreads();
    return true;
  };
  if constexpr (VEC) {
    // A thread's first unit is read while the angles are computed, every later one ahead of the write of the one before, which a wait for it
    // then need not cover.  (Behind that write: 52 us instead of 36 for 8192 rows of 40 heads.)
    struct Unit {
      uint4 p, q;
      T* to;   // NULL: nothing
      int at;  // of the angles; -1: behind the turned part, as it is
    };
    auto read = [&]() {
      Unit r = {make_uint4(0u, 0u, 0u, 0u), make_uint4(0u, 0u, 0u, 0u), nullptr, -1};
      if (t >= n_here) return r;
      const int which = head_t < a.heads[0] ? 0 : 1, head = which ? head_t - a.heads[0] : head_t;
      const bool turns = x < turned;
      const int d = turns ? WIDE * x : a.rot + (x - turned) * WIDE;
      const T* const src = static_cast<const T*>(a.in[which]) + (n0 + t) * a.in_stride[which] + (int64_t)head * a.D + d;
      r.to = static_cast<T*>(a.out[which]) + (n0 + t) * a.out_stride[which] + (int64_t)head * a.D + d;
      r.at = turns ? t * h + (PAIRS == 0 ? WIDE : WIDE / 2) * x : -1;
      r.p = *reinterpret_cast<const uint4*>(src);
      if (PAIRS == 0 && turns) r.q = *reinterpret_cast<const uint4*>(src + h);
      next();
      return r;
    };
    Unit ahead = read();
    if (!angles()) return;
    while (ahead.to != nullptr) {
      const Unit now = ahead;
      ahead = read();
      if (now.at < 0) {
        *reinterpret_cast<uint4*>(now.to) = now.p;
        continue;
      }
      const float* const cs = c_lds + now.at;
      const float* const sn = s_lds + now.at;
      float f[WIDE], g[WIDE], r[WIDE];
      values<T>(now.p, f);
      if constexpr (PAIRS == 0) {
        values<T>(now.q, g);
#pragma unroll
        for (int e = 0; e < WIDE; ++e) r[e] = f[e] * cs[e] - g[e] * sn[e];
        store16(now.to, r);
#pragma unroll
        for (int e = 0; e < WIDE; ++e) r[e] = g[e] * cs[e] + f[e] * sn[e];
        store16(now.to + h, r);
      } else {
#pragma unroll
        for (int e = 0; e < WIDE / 2; ++e) {
          r[2 * e] = f[2 * e] * cs[e] - f[2 * e + 1] * sn[e];
          r[2 * e + 1] = f[2 * e + 1] * cs[e] + f[2 * e] * sn[e];
        }
        store16(now.to, r);
      }
    }
  } else {
    if (!angles()) return;
    while (t < n_here) {
      const int which = head_t < a.heads[0] ? 0 : 1, head = which ? head_t - a.heads[0] : head_t;
      const T* const src = static_cast<const T*>(a.in[which]) + (n0 + t) * a.in_stride[which] + (int64_t)head * a.D;
      T* const dst = static_cast<T*>(a.out[which]) + (n0 + t) * a.out_stride[which] + (int64_t)head * a.D;
      if (x >= turned) {
        const int d = a.rot + (x - turned);
        dst[d] = src[d];
      } else {
        const float cs = c_lds[t * h + x], sn = s_lds[t * h + x];
        const int d0 = PAIRS ? 2 * x : x, d1 = PAIRS ? 2 * x + 1 : x + h;
        const float p = elem(src + d0), q = elem(src + d1);
        store_elem(dst + d0, p * cs - q * sn);
        store_elem(dst + d1, q * cs + p * sn);
      }
      next();
    }
  }
}

}  // namespace hs

using namespace hs;

static hs_status rotary_impl(RotaryArgs a, hs_dtype dt, hs_rotary_pairs pairs, bool tree, hs_stream stream) {
  HS_REQUIRE(dt == HS_F32 || dt == HS_BF16, HS_ERR_SHAPE, "hs_rotary: unknown dtype %d", (int)dt);
  HS_REQUIRE(pairs == HS_ROTARY_HALF || pairs == HS_ROTARY_NEIGHBOURS, HS_ERR_SHAPE, "hs_rotary: unknown pairing %d", (int)pairs);
  HS_REQUIRE(a.N >= 0 && a.heads[0] >= 1 && a.heads[1] >= 0 && a.D >= 2, HS_ERR_SHAPE, "hs_rotary: N=%d Hq=%d Hkv=%d D=%d", a.N,
             a.heads[0], a.heads[1], a.D);
  HS_REQUIRE(a.rot >= 2 && a.rot % 2 == 0 && a.rot <= a.D, HS_ERR_SHAPE, "hs_rotary: rot_dim=%d must be even and at most D=%d", a.rot, a.D);
  HS_REQUIRE(a.D <= 1024 && (int64_t)(a.heads[0] + (int64_t)a.heads[1]) * a.D <= (1 << 24), HS_ERR_UNSUPPORTED,
             "hs_rotary: D=%d with %d + %d heads", a.D, a.heads[0], a.heads[1]);
  if (a.N == 0) return HS_OK;
  const int tensors = a.heads[1] > 0 ? 2 : 1;
  const int size = dt == HS_F32 ? 4 : 2;
  bool vec = a.D % 8 == 0 && a.rot % (pairs == HS_ROTARY_HALF ? 16 : 8) == 0;
  for (int i = 0; i < tensors; ++i) {
    HS_REQUIRE(a.in[i] && a.out[i], HS_ERR_NULL, "hs_rotary: NULL tensor");
    const int64_t least = (int64_t)a.heads[i] * a.D;
    HS_REQUIRE(a.in_stride[i] >= least && a.out_stride[i] >= least, HS_ERR_SHAPE, "hs_rotary: a row stride is less than heads * D = %lld",
               (long long)least);
    HS_REQUIRE(a.in[i] != a.out[i] || a.in_stride[i] == a.out_stride[i], HS_ERR_SHAPE, "hs_rotary: in place, but with two row strides");
    const uintptr_t p = reinterpret_cast<uintptr_t>(a.in[i]), q = reinterpret_cast<uintptr_t>(a.out[i]);
    HS_REQUIRE(p % size == 0 && q % size == 0, HS_ERR_UNSUPPORTED, "hs_rotary: tensors must be aligned to their elements");
    vec = vec && p % 16 == 0 && q % 16 == 0 && a.in_stride[i] % 8 == 0 && a.out_stride[i] % 8 == 0;
  }
  HS_REQUIRE(a.inv_freq, HS_ERR_NULL, "hs_rotary: NULL inv_freq");
  if (tree) HS_REQUIRE(a.parent && a.node_offsets && a.prefix_lens && a.B >= 1, HS_ERR_NULL, "hs_tree_rotary: NULL tree arrays, or rows of no sequence");
  else HS_REQUIRE(a.positions, HS_ERR_NULL, "hs_rotary: NULL positions");
  const int wide = vec ? 16 / size : 1, units = (a.heads[0] + a.heads[1]) * ((pairs == HS_ROTARY_HALF || !vec ? a.rot / 2 : a.rot) + a.D - a.rot) / wide;
  a.tokens = !tree && a.N >= ROT_MANY && units < ROT_THREADS ? ROT_THREADS / units : 1;
  while (!tree && (a.N - 1) / a.tokens >= 1 << 23) a.tokens *= 2;  // (a launch has fewer than 2^32 threads)
  HS_REQUIRE((a.N - 1) / a.tokens < 1 << 23, HS_ERR_UNSUPPORTED, "hs_tree_rotary: %d rows are too many for one call", a.N);
  const int h = a.rot / 2;
  const size_t lds = (size_t)a.tokens * h * 8 + (tree ? ROT_STAGE * 8 : 0);
  const dim3 grid((unsigned)((a.N - 1) / a.tokens + 1)), block(ROT_THREADS);
#define ROT_LAUNCH(T, P, TR, V) hipLaunchKernelGGL((k_rotary<T, P, TR, V>), grid, block, lds, static_cast<hipStream_t>(stream), a)
#define ROT_VEC(T, P, TR) \
  do {                    \
    if (vec) ROT_LAUNCH(T, P, TR, true); \
    else ROT_LAUNCH(T, P, TR, false);    \
  } while (0)
#define ROT_TREE(T, P)           \
  do {                           \
    if (tree) ROT_VEC(T, P, true); \
    else ROT_VEC(T, P, false);     \
  } while (0)
  if (dt == HS_F32) {
    if (pairs == HS_ROTARY_HALF) ROT_TREE(float, 0);
    else ROT_TREE(float, 1);
  } else {
    if (pairs == HS_ROTARY_HALF) ROT_TREE(bf16_t, 0);
    else ROT_TREE(bf16_t, 1);
  }
#undef ROT_TREE
#undef ROT_VEC
#undef ROT_LAUNCH
  return launch_status("rotary");
}

static RotaryArgs rotary_args(const void* q, int64_t qs, const void* k, int64_t ks, int32_t N, int32_t Hq, int32_t Hkv, int32_t D,
                              int32_t rot, const double* f, float m, void* qo, int64_t qos, void* ko, int64_t kos) {
  RotaryArgs a = {};
  a.in[0] = q, a.in[1] = k, a.out[0] = qo, a.out[1] = ko;
  a.in_stride[0] = qs, a.in_stride[1] = ks, a.out_stride[0] = qos, a.out_stride[1] = kos;
  a.heads[0] = Hq, a.heads[1] = Hkv;
  a.N = N, a.D = D, a.rot = rot;
  a.inv_freq = f, a.mscale = m;
  return a;
}

extern "C" hs_status hs_rotary(const void* q, int64_t q_stride, const void* k, int64_t k_stride, const int64_t* positions, int32_t N,
                               int32_t Hq, int32_t Hkv, int32_t D, hs_dtype dt, const double* inv_freq, int32_t rot_dim,
                               hs_rotary_pairs pairs, float mscale, void* q_out, int64_t q_out_stride, void* k_out,
                               int64_t k_out_stride, hs_stream stream) {
  clear_error();
  RotaryArgs a = rotary_args(q, q_stride, k, k_stride, N, Hq, Hkv, D, rot_dim, inv_freq, mscale, q_out, q_out_stride, k_out, k_out_stride);
  a.positions = positions;
  return rotary_impl(a, dt, pairs, false, stream);
}

extern "C" hs_status hs_tree_rotary(const void* q, int64_t q_stride, const void* k, int64_t k_stride, const int32_t* parent,
                                    const int32_t* node_offsets, const int64_t* prefix_lens, int32_t B, int32_t N, int32_t Hq,
                                    int32_t Hkv, int32_t D, hs_dtype dt, const double* inv_freq, int32_t rot_dim,
                                    hs_rotary_pairs pairs, float mscale, void* q_out, int64_t q_out_stride, void* k_out,
                                    int64_t k_out_stride, hs_stream stream) {
  clear_error();
  HS_REQUIRE(B >= 0, HS_ERR_SHAPE, "hs_tree_rotary: B=%d", B);
  RotaryArgs a = rotary_args(q, q_stride, k, k_stride, N, Hq, Hkv, D, rot_dim, inv_freq, mscale, q_out, q_out_stride, k_out, k_out_stride);
  a.parent = parent, a.node_offsets = node_offsets, a.prefix_lens = prefix_lens, a.B = B;
  return rotary_impl(a, dt, pairs, true, stream);
}

// ---- the table of a scaled rotation, on the host in double precision
#include <math.h>

extern "C" hs_status hs_rotary_frequencies(int32_t rot_dim, double base, hs_rotary_scaling scaling, double factor, double context,
                                           double low, double high, double* host_inv_freq, float* host_mscale) {
  clear_error();
  HS_REQUIRE(host_inv_freq && host_mscale, HS_ERR_NULL, "hs_rotary_frequencies: NULL output");
  HS_REQUIRE(rot_dim >= 2 && rot_dim % 2 == 0, HS_ERR_SHAPE, "hs_rotary_frequencies: rot_dim=%d must be even", rot_dim);
  HS_REQUIRE(base > 1.0 && isfinite(base), HS_ERR_SHAPE, "hs_rotary_frequencies: base=%g", base);
  HS_REQUIRE(scaling >= HS_ROTARY_PLAIN && scaling <= HS_ROTARY_YARN, HS_ERR_SHAPE, "hs_rotary_frequencies: unknown scaling %d", (int)scaling);
  if (scaling != HS_ROTARY_PLAIN)
    HS_REQUIRE(factor >= 1.0 && isfinite(factor), HS_ERR_SHAPE, "hs_rotary_frequencies: factor=%g", factor);
  if (scaling == HS_ROTARY_BASE) HS_REQUIRE(rot_dim > 2, HS_ERR_SHAPE, "hs_rotary_frequencies: a stretched base needs rot_dim > 2");
  if (scaling == HS_ROTARY_WAVELENGTH || scaling == HS_ROTARY_YARN)
    HS_REQUIRE(context > 0.0 && isfinite(context) && low > 0.0 && high > low && isfinite(high), HS_ERR_SHAPE,
               "hs_rotary_frequencies: context=%g, low=%g, high=%g", context, low, high);
  const double two_pi = 6.28318530717958647693, n = (double)rot_dim;
  if (scaling == HS_ROTARY_BASE) base *= pow(factor, n / (n - 2.0));
  // YaRN: the pairs whose wave turns `high` and `low` times within the context; between them a ramp
  double first = 0.0, last = 0.0;
  if (scaling == HS_ROTARY_YARN) {
    auto pair_of = [&](double turns) { return n * log(context / (turns * two_pi)) / (2.0 * log(base)); };
    first = fmax(floor(pair_of(high)), 0.0);
    last = fmin(ceil(pair_of(low)), n - 1.0);
  }
  for (int j = 0; j < rot_dim / 2; ++j) {
    const double f = pow(base, -2.0 * j / n);
    double keep = 1.0;  // share of the unstretched frequency
    if (scaling == HS_ROTARY_LINEAR) keep = 0.0;
    if (scaling == HS_ROTARY_WAVELENGTH) keep = fmin(fmax((context * f / two_pi - low) / (high - low), 0.0), 1.0);
    if (scaling == HS_ROTARY_YARN) keep = 1.0 - fmin(fmax((j - first) / fmax(last - first, 1e-3), 0.0), 1.0);
    host_inv_freq[j] = scaling == HS_ROTARY_PLAIN || scaling == HS_ROTARY_BASE ? f : (1.0 - keep) * f / factor + keep * f;
  }
  *host_mscale = scaling == HS_ROTARY_YARN ? (float)(0.1 * log(factor) + 1.0) : 1.0f;
  return HS_OK;
}
