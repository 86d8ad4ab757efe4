// hs_kv_append_mx, hs_kv_commit_mx, hs_kv_read_mx: rows join a quantised cache, and are read back.
//
// A workgroup takes a few rows and, of K's and V's columns side by side, as many eighths (units) as it has threads.  Its first
// lanes look the rows up (sequence, token, page) into LDS, and a thread keeps its unit - which of K and V, head and columns - through
// the rows, four of them at a time: what is left of a unit is an address of the row's and one of the thread's, a load, four
// conversions and a store.  (Every lane by itself, a 64-bit division and a look-up each: 83 us instead of 52 for 36000 rows of
// 8 heads out of e4m3, 16 instead of 12 for 8192 into it.)
//
// Storing, four lanes hold a block of 32: its largest magnitude meets in two lane exchanges (as an integer maximum of
// the bits, which puts NaN and infinity on top), its scale is a shift of that maximum's exponent, and conversion instructions
// round the elements.  Bound by memory: a bfloat16 row is read once, 0.52 (e4m3) or 0.27 (e2m1) of it is written.
#include "mx.h"

namespace hs {

constexpr int MXC_THREADS = 256;
constexpr int MXC_ROWS = 32;   // of a workgroup at most
constexpr int MXC_AT_ONCE = 4;

// Rows of a workgroup: four to a thread, whose loads then are in flight together, or fewer where that leaves less than 1024
// workgroups.  (Rows of 256 units, us at 1 | 2 | 4 | 8 | 16 | 32 rows: 36000 read 71 | 55 | 52 | 55 | 62 | 61, 8192 stored 19 | 14 | 12 |
// 12 | 14 | 23, 2000 read 5.8 | 6.2 | 6.2 | 6.3 | 8.5 | 15.)
static int mxc_rows(int64_t rows, const MxPool& c) {
  const int64_t units = 2ll * c.Hkv * (c.D >> 3), side = (units + MXC_THREADS - 1) / MXC_THREADS;
  int64_t per = MXC_AT_ONCE * (units < MXC_THREADS ? MXC_THREADS / units : 1);
  per = per < MXC_ROWS ? per : MXC_ROWS;
  while (per > 1 && rows * side < 1024 * per) per /= 2;
  return (int)per;
}
// The thread's unit of a row of `units` (gridDim.y workgroups side by side, or several rows to a workgroup): whether it has one,
// its first row of the workgroup's and the step to the next.
struct MxUnit {
  bool any, is_v;
  int row, step;
  int g, d;
};
__device__ __forceinline__ MxUnit mx_unit(const MxPool& c) {
  const int eights = c.D >> 3, half = c.Hkv * eights, units = 2 * half;
  MxUnit t;
  int u;
  if (units >= MXC_THREADS) {
    t.row = 0, t.step = 1;
    u = blockIdx.y * MXC_THREADS + threadIdx.x;
    t.any = u < units;
  } else {
    t.step = MXC_THREADS / units;
    t.row = (int)threadIdx.x / units;
    u = (int)threadIdx.x - t.row * units;
    t.any = t.row < t.step;
  }
  t.is_v = u >= half;
  if (t.is_v) u -= half;
  t.g = u / eights;
  t.d = 8 * (u - t.g * eights);
  return t;
}

template <typename T>
__device__ __forceinline__ void load8_bits(const T* p, unsigned* b);  // eight elements as float32 bits
template <>
__device__ __forceinline__ void load8_bits<float>(const float* p, unsigned* b) {
  const uint4 lo = *reinterpret_cast<const uint4*>(p), hi = *reinterpret_cast<const uint4*>(p + 4);
  b[0] = lo.x, b[1] = lo.y, b[2] = lo.z, b[3] = lo.w, b[4] = hi.x, b[5] = hi.y, b[6] = hi.z, b[7] = hi.w;
}
template <>
__device__ __forceinline__ void load8_bits<bf16_t>(const bf16_t* p, unsigned* b) {
  const uint4 w = *reinterpret_cast<const uint4*>(p);
  b[0] = w.x << 16, b[1] = w.x & 0xffff0000u, b[2] = w.y << 16, b[3] = w.y & 0xffff0000u;
  b[4] = w.z << 16, b[5] = w.z & 0xffff0000u, b[6] = w.w << 16, b[7] = w.w & 0xffff0000u;
}

// The lane's eight elements to `codes`, the block's scale (first lane of four) to `scale`.
template <int FMT>
__device__ __forceinline__ void mx_store8(const unsigned* b, unsigned char* codes, unsigned char* scale, bool first) {
  unsigned amax = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const unsigned m = b[i] & 0x7fffffffu;
    amax = m > amax ? m : amax;
  }
#pragma unroll
  for (int x = 1; x <= 2; x *= 2) {
    const unsigned m = (unsigned)__shfl_xor((int)amax, x);
    amax = m > amax ? m : amax;
  }
  const unsigned byte = mx_scale_byte<FMT>(amax);
  const float s = mx_scale(byte == 255u ? 127u : byte);
  float f[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] = byte == 255u ? 0.f : __builtin_bit_cast(float, b[i]);
  if constexpr (FMT == HS_MX_E4M3) {
    mx_s16x2 lo = {0, 0}, hi = {0, 0};
    lo = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(lo, f[0], f[1], s, false);
    lo = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(lo, f[2], f[3], s, true);
    hi = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(hi, f[4], f[5], s, false);
    hi = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(hi, f[6], f[7], s, true);
    *reinterpret_cast<uint2*>(codes) = make_uint2(__builtin_bit_cast(unsigned, lo), __builtin_bit_cast(unsigned, hi));
  } else {
    unsigned w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[0], f[1], s, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[2], f[3], s, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[4], f[5], s, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[6], f[7], s, 3);
    *reinterpret_cast<unsigned*>(codes) = w;
  }
  if (first) *scale = (unsigned char)byte;
}

struct MxStoreArgs {
  const void* k;
  const void* v;
  int64_t k_stride, v_stride;    // elements from row to row
  const int32_t* node_offsets;
  const int32_t* path;           // commit: accepted rows [B, max_depth] and their numbers [B]
  const int32_t* path_len;
  int max_depth;
  const int64_t* lens;
  int64_t* new_lens;             // may be NULL
  int B;
  int64_t places;                // rows (append), or B * (1 + max_depth) (commit)
  int per;                       // of a workgroup
  MxPool pool;
};

// Rows that sequence s has for its cache.
template <bool PATH>
__device__ __forceinline__ int64_t mx_rows(const MxStoreArgs& a, int s) {
  const int M = a.node_offsets[s + 1] - a.node_offsets[s];
  if (!PATH || M <= 0) return M > 0 ? M : 0;
  const int n = a.path_len[s];
  return 1 + (n < 0 ? 0 : n > a.max_depth ? a.max_depth : n);
}

template <typename T, int FMT, bool PATH>
__global__ __launch_bounds__(MXC_THREADS) void k_mx_store(MxStoreArgs a) {
  __shared__ int64_t from[MXC_ROWS], to[MXC_ROWS];  // row of k and v; row of head 0 in the pool (-1: none)
  const MxPool& c = a.pool;
  const int64_t cap = (int64_t)c.max_blocks * MX_PAGE;
  if (a.new_lens != nullptr && blockIdx.y == 0)
    for (int64_t s = (int64_t)blockIdx.x * MXC_THREADS + threadIdx.x; s < a.B; s += (int64_t)gridDim.x * MXC_THREADS) {
      const int64_t used = a.lens[s], rows = mx_rows<PATH>(a, (int)s), room = used >= cap ? 0 : cap - used;
      a.new_lens[s] = used + (rows < room ? rows : room);
    }
  const int64_t first = (int64_t)blockIdx.x * a.per;
  if (threadIdx.x < 64) {
    const int64_t place = first + threadIdx.x;
    int64_t row = 0, at = -1;
    int s = 0, t = -1;
    if constexpr (PATH) {
      if ((int)threadIdx.x < a.per && place < a.places) {
        s = (int)place / (1 + a.max_depth);
        t = (int)place - s * (1 + a.max_depth);
        const int n0 = a.node_offsets[s], M = a.node_offsets[s + 1] - n0;
        int r = t == 0 ? 0 : a.path[(int64_t)s * a.max_depth + t - 1];
        r = r < 0 ? 0 : r >= M ? M - 1 : r;  // (an entry outside the tree would be a caller's error)
        row = n0 + r;
        if (t >= mx_rows<true>(a, s)) t = -1;
      }
    } else {
      s = seq_of_row(a.node_offsets, a.B, first);
      if ((int)threadIdx.x < a.per && place < a.places) {
        while (s + 1 < a.B && place >= a.node_offsets[s + 1]) ++s;
        row = place;
        if (place < a.node_offsets[s + 1]) t = (int)(place - a.node_offsets[s]);
      }
    }
    if (t >= 0) {
      const int64_t tok = a.lens[s] + t;
      if (tok >= 0 && tok < cap) {
        const int page = c.table[(int64_t)s * c.max_blocks + tok / MX_PAGE];
        if (page >= 0 && page < c.n_pages) at = (int64_t)page * c.Hkv * MX_PAGE + (tok & (MX_PAGE - 1));
      }
    }
    if ((int)threadIdx.x < a.per) from[threadIdx.x] = row, to[threadIdx.x] = at;
  }
  __syncthreads();
  const MxUnit t = mx_unit(c);
  if (!t.any) return;  // (units are whole blocks of four lanes)
  const T* const src = static_cast<const T*>(t.is_v ? a.v : a.k) + (int64_t)t.g * c.D + t.d;
  const int64_t stride = t.is_v ? a.v_stride : a.k_stride;
  unsigned char* const codes = (t.is_v ? c.v_codes : c.k_codes) + ((int64_t)t.g * MX_PAGE * c.D + t.d) * Mx<FMT>::BITS / 8;
  unsigned char* const scales = (t.is_v ? c.v_scales : c.k_scales) + (int64_t)t.g * MX_PAGE * (c.D / MX_BLOCK) + t.d / MX_BLOCK;
  for (int i = t.row; i < a.per; i += MXC_AT_ONCE * t.step) {
    unsigned b[MXC_AT_ONCE][8];
    int64_t at[MXC_AT_ONCE];
#pragma unroll
    for (int x = 0; x < MXC_AT_ONCE; ++x) {
      const int r = i + x * t.step;
      at[x] = r < a.per ? to[r] : -1;
      if (at[x] >= 0) load8_bits(src + from[r] * stride, b[x]);
    }
#pragma unroll
    for (int x = 0; x < MXC_AT_ONCE; ++x)
      if (at[x] >= 0) mx_store8<FMT>(b[x], codes + at[x] * mx_row_bytes(FMT, c.D), scales + at[x] * (c.D / MX_BLOCK), (t.d & (MX_BLOCK - 1)) == 0);
  }
}

struct MxReadArgs {
  const int64_t* out_offsets;
  const int64_t* first;  // first token of each sequence; NULL: 0
  int B;
  int per;  // rows of a workgroup
  int64_t total;
  void* k_out;
  void* v_out;
  MxPool pool;
};

template <typename T, int FMT>
__global__ __launch_bounds__(MXC_THREADS) void k_mx_read(MxReadArgs a) {
  __shared__ int64_t from[MXC_ROWS];  // row of head 0 in the pool (-1: none)
  const MxPool& c = a.pool;
  const int64_t first = (int64_t)blockIdx.x * a.per;
  if (threadIdx.x < 64) {
    const int64_t row = first + threadIdx.x;
    int s = seq_of_row(a.out_offsets, a.B, first);
    if ((int)threadIdx.x < a.per) {
      int64_t at = -1;
      if (row < a.total) {
        while (s + 1 < a.B && row >= a.out_offsets[s + 1]) ++s;
        if (row < a.out_offsets[s + 1]) {
          const int64_t tok = row - a.out_offsets[s] + (a.first != nullptr ? a.first[s] : 0);
          if (tok >= 0 && tok < (int64_t)c.max_blocks * MX_PAGE) {
            const int page = c.table[(int64_t)s * c.max_blocks + tok / MX_PAGE];
            if (page >= 0 && page < c.n_pages) at = (int64_t)page * c.Hkv * MX_PAGE + (tok & (MX_PAGE - 1));
          }
        }
      }
      from[threadIdx.x] = at;
    }
  }
  __syncthreads();
  const MxUnit t = mx_unit(c);
  if (!t.any) return;
  const unsigned char* const codes = (t.is_v ? c.v_codes : c.k_codes) + ((int64_t)t.g * MX_PAGE * c.D + t.d) * Mx<FMT>::BITS / 8;
  const unsigned char* const scales = (t.is_v ? c.v_scales : c.k_scales) + (int64_t)t.g * MX_PAGE * (c.D / MX_BLOCK) + t.d / MX_BLOCK;
  T* const dst = static_cast<T*>(t.is_v ? a.v_out : a.k_out) + (first * c.Hkv + t.g) * c.D + t.d;
  for (int i = t.row; i < a.per; i += MXC_AT_ONCE * t.step) {
    uint2 w[MXC_AT_ONCE];
    unsigned byte[MXC_AT_ONCE];
    int64_t at[MXC_AT_ONCE];
#pragma unroll
    for (int x = 0; x < MXC_AT_ONCE; ++x) {
      const int r = i + x * t.step;
      at[x] = r < a.per ? from[r] : -1;
      if (at[x] >= 0) {
        const unsigned char* const p = codes + at[x] * mx_row_bytes(FMT, c.D);
        if constexpr (FMT == HS_MX_E4M3) w[x] = *reinterpret_cast<const uint2*>(p);
        else w[x].x = *reinterpret_cast<const unsigned*>(p), w[x].y = 0u;
        byte[x] = scales[at[x] * (c.D / MX_BLOCK)];
      }
    }
#pragma unroll
    for (int x = 0; x < MXC_AT_ONCE; ++x) {
      if (at[x] < 0) continue;
      const uint4 e = mx_eight<FMT>(w[x].x, w[x].y, mx_scale(byte[x]));
      T* const to = dst + (int64_t)(i + x * t.step) * c.Hkv * c.D;
      if constexpr (sizeof(T) == 2) {
        *reinterpret_cast<uint4*>(to) = e;
      } else {
        *reinterpret_cast<uint4*>(to) = make_uint4(e.x << 16, e.x & 0xffff0000u, e.y << 16, e.y & 0xffff0000u);
        *reinterpret_cast<uint4*>(to + 4) = make_uint4(e.z << 16, e.z & 0xffff0000u, e.w << 16, e.w & 0xffff0000u);
      }
    }
  }
}

hs_status mx_pool_check(const char* what, const MxPool& c, hs_mx_format fmt) {
  HS_REQUIRE(fmt == HS_MX_E4M3 || fmt == HS_MX_E2M1, HS_ERR_SHAPE, "%s: unknown format %d", what, (int)fmt);
  HS_REQUIRE(c.Hkv >= 1 && c.D >= 1 && c.max_blocks >= 0 && c.n_pages >= 0, HS_ERR_SHAPE, "%s: Hkv=%d D=%d max_blocks=%d n_pages=%d", what,
             c.Hkv, c.D, c.max_blocks, c.n_pages);
  HS_REQUIRE(c.D % MX_BLOCK == 0 && (int64_t)c.Hkv * c.D <= (1 << 24), HS_ERR_UNSUPPORTED, "%s: D=%d must be a multiple of %d (and Hkv * D at most 2^24)",
             what, c.D, MX_BLOCK);
  return HS_OK;
}
hs_status mx_pool_pointers(const char* what, const MxPool& c) {
  HS_REQUIRE(c.k_codes && c.k_scales && c.v_codes && c.v_scales && c.table, HS_ERR_NULL, "%s: NULL cache or block table", what);
  HS_REQUIRE(((reinterpret_cast<uintptr_t>(c.k_codes) | reinterpret_cast<uintptr_t>(c.v_codes)) & 15) == 0 &&
                 ((reinterpret_cast<uintptr_t>(c.k_scales) | reinterpret_cast<uintptr_t>(c.v_scales)) & 3) == 0,
             HS_ERR_UNSUPPORTED, "%s: codes must be 16-byte aligned, scales 4-byte aligned", what);
  return HS_OK;
}

}  // namespace hs

using namespace hs;

static hs_status mx_store_impl(const char* what, MxStoreArgs a, hs_mx_format fmt, hs_dtype dt, bool path, hs_stream stream) {
  MxPool& c = a.pool;
  HS_REQUIRE(a.B >= 0 && a.places >= 0, HS_ERR_SHAPE, "%s: a size is negative", what);
  HS_REQUIRE(dt == HS_F32 || dt == HS_BF16, HS_ERR_SHAPE, "%s: unknown dtype %d", what, (int)dt);
  hs_status st = mx_pool_check(what, c, fmt);
  if (st != HS_OK) return st;
  if (a.B == 0) {
    HS_REQUIRE(a.places == 0, HS_ERR_SHAPE, "%s: rows of no sequence", what);
    return HS_OK;
  }
  HS_REQUIRE(a.node_offsets && a.lens, HS_ERR_NULL, "%s: NULL argument", what);
  HS_REQUIRE(!path || (a.path && a.path_len), HS_ERR_NULL, "%s: NULL accepted path", what);
  HS_REQUIRE(a.new_lens == nullptr || a.new_lens + a.B <= a.lens || a.lens + a.B <= a.new_lens, HS_ERR_SHAPE,
             "%s: new_lens overlaps cache_lens", what);
  // without rows only the lengths are written
  const bool any = a.places > 0;
  if (any) {
    st = mx_pool_pointers(what, c);
    if (st != HS_OK) return st;
    HS_REQUIRE(a.k && a.v, HS_ERR_NULL, "%s: NULL tensor", what);
    const int64_t row = (int64_t)c.Hkv * c.D;
    HS_REQUIRE(a.k_stride >= row && a.v_stride >= row, HS_ERR_SHAPE, "%s: a row stride is less than Hkv * D = %lld", what, (long long)row);
    const int per16 = dt == HS_F32 ? 4 : 8;
    HS_REQUIRE(((reinterpret_cast<uintptr_t>(a.k) | reinterpret_cast<uintptr_t>(a.v)) & 15) == 0 && a.k_stride % per16 == 0 && a.v_stride % per16 == 0,
               HS_ERR_UNSUPPORTED, "%s: rows must begin at multiples of 16 bytes", what);
  } else if (a.new_lens == nullptr) {
    return HS_OK;
  }
  a.per = mxc_rows(a.places, c);
  const int64_t blocks = any ? (a.places + a.per - 1) / a.per : 1, units = 2ll * c.Hkv * (c.D / 8);
  HS_REQUIRE(blocks < ((int64_t)1 << 24), HS_ERR_UNSUPPORTED, "%s: %lld rows are too many for one call", what, (long long)a.places);
  const dim3 grid((unsigned)blocks, any ? (unsigned)((units + MXC_THREADS - 1) / MXC_THREADS) : 1u), block(MXC_THREADS);
#define MXC_LAUNCH(T, F, P) hipLaunchKernelGGL((k_mx_store<T, F, P>), grid, block, 0, static_cast<hipStream_t>(stream), a)
#define MXC_FMT(T, P)                                    \
  do {                                                   \
    if (fmt == HS_MX_E4M3) MXC_LAUNCH(T, HS_MX_E4M3, P); \
    else MXC_LAUNCH(T, HS_MX_E2M1, P);                   \
  } while (0)
  if (dt == HS_F32) {
    if (path) MXC_FMT(float, true);
    else MXC_FMT(float, false);
  } else {
    if (path) MXC_FMT(bf16_t, true);
    else MXC_FMT(bf16_t, false);
  }
#undef MXC_FMT
#undef MXC_LAUNCH
  return launch_status(what);
}

static MxPool mx_pool(const void* kc, const void* ks, const void* vc, const void* vs, const int32_t* table, int32_t max_blocks,
                      int32_t n_pages, int32_t Hkv, int32_t D) {
  auto bytes = [](const void* p) { return static_cast<unsigned char*>(const_cast<void*>(p)); };
  return MxPool{bytes(kc), bytes(ks), bytes(vc), bytes(vs), table, max_blocks, n_pages, Hkv, D};
}

extern "C" hs_status hs_kv_append_mx(const void* k, int64_t k_stride, const void* v, int64_t v_stride, const int32_t* node_offsets,
                                     int32_t NN, void* k_codes, void* k_scales, void* v_codes, void* v_scales, hs_mx_format fmt,
                                     const int32_t* block_table, int32_t max_blocks, int32_t n_pages, const int64_t* cache_lens,
                                     int64_t* new_lens, int32_t B, int32_t Hkv, int32_t D, hs_dtype dt, hs_stream stream) {
  clear_error();
  MxStoreArgs a = {};
  a.k = k, a.v = v, a.k_stride = k_stride, a.v_stride = v_stride, a.node_offsets = node_offsets;
  a.lens = cache_lens, a.new_lens = new_lens, a.B = B, a.places = NN;
  a.pool = mx_pool(k_codes, k_scales, v_codes, v_scales, block_table, max_blocks, n_pages, Hkv, D);
  return mx_store_impl("hs_kv_append_mx", a, fmt, dt, false, stream);
}

extern "C" hs_status hs_kv_commit_mx(const void* k_tree, int64_t k_stride, const void* v_tree, int64_t v_stride,
                                     const int32_t* node_offsets, const int32_t* accept_path, const int32_t* accept_len,
                                     int32_t max_depth, void* k_codes, void* k_scales, void* v_codes, void* v_scales,
                                     hs_mx_format fmt, const int32_t* block_table, int32_t max_blocks, int32_t n_pages,
                                     const int64_t* cache_lens, int64_t* new_lens, int32_t B, int32_t Hkv, int32_t D, hs_dtype dt,
                                     hs_stream stream) {
  clear_error();
  HS_REQUIRE(max_depth >= 1 && B >= 0, HS_ERR_SHAPE, "hs_kv_commit_mx: B=%d max_depth=%d", B, max_depth);
  HS_REQUIRE((int64_t)B * ((int64_t)max_depth + 1) < ((int64_t)1 << 31), HS_ERR_UNSUPPORTED, "hs_kv_commit_mx: B=%d paths of %d rows", B, max_depth);
  MxStoreArgs a = {};
  a.k = k_tree, a.v = v_tree, a.k_stride = k_stride, a.v_stride = v_stride, a.node_offsets = node_offsets;
  a.path = accept_path, a.path_len = accept_len, a.max_depth = max_depth;
  a.lens = cache_lens, a.new_lens = new_lens, a.B = B, a.places = (int64_t)B * (max_depth + 1);
  a.pool = mx_pool(k_codes, k_scales, v_codes, v_scales, block_table, max_blocks, n_pages, Hkv, D);
  return mx_store_impl("hs_kv_commit_mx", a, fmt, dt, true, stream);
}

extern "C" hs_status hs_kv_read_mx(const void* k_codes, const void* k_scales, const void* v_codes, const void* v_scales,
                                   hs_mx_format fmt, const int32_t* block_table, int32_t max_blocks, int32_t n_pages,
                                   const int64_t* first, const int64_t* out_offsets, int64_t total, void* k_out, void* v_out,
                                   int32_t B, int32_t Hkv, int32_t D, hs_dtype dt, hs_stream stream) {
  clear_error();
  MxReadArgs a = {out_offsets, first, B, 1, total, k_out, v_out, mx_pool(k_codes, k_scales, v_codes, v_scales, block_table, max_blocks, n_pages, Hkv, D)};
  HS_REQUIRE(B >= 0 && total >= 0, HS_ERR_SHAPE, "hs_kv_read_mx: B=%d total=%lld", B, (long long)total);
  HS_REQUIRE(dt == HS_F32 || dt == HS_BF16, HS_ERR_SHAPE, "hs_kv_read_mx: unknown dtype %d", (int)dt);
  hs_status st = mx_pool_check("hs_kv_read_mx", a.pool, fmt);
  if (st != HS_OK) return st;
  HS_REQUIRE(B > 0 || total == 0, HS_ERR_SHAPE, "hs_kv_read_mx: rows of no sequence");
  if (total == 0) return HS_OK;
  st = mx_pool_pointers("hs_kv_read_mx", a.pool);
  if (st != HS_OK) return st;
  HS_REQUIRE(out_offsets && k_out && v_out, HS_ERR_NULL, "hs_kv_read_mx: NULL argument");
  HS_REQUIRE(((reinterpret_cast<uintptr_t>(k_out) | reinterpret_cast<uintptr_t>(v_out)) & 15) == 0, HS_ERR_UNSUPPORTED,
             "hs_kv_read_mx: outputs must be 16-byte aligned");
  a.per = mxc_rows(total, a.pool);
  const int64_t blocks = (total + a.per - 1) / a.per, units = 2ll * Hkv * (D / 8);
  HS_REQUIRE(blocks < ((int64_t)1 << 24), HS_ERR_UNSUPPORTED, "hs_kv_read_mx: %lld rows are too many for one call", (long long)total);
  const dim3 grid((unsigned)blocks, (unsigned)((units + MXC_THREADS - 1) / MXC_THREADS)), block(MXC_THREADS);
#define MXC_LAUNCH(T, F) hipLaunchKernelGGL((k_mx_read<T, F>), grid, block, 0, static_cast<hipStream_t>(stream), a)
  if (dt == HS_F32) {
    if (fmt == HS_MX_E4M3) MXC_LAUNCH(float, HS_MX_E4M3);
    else MXC_LAUNCH(float, HS_MX_E2M1);
  } else {
    if (fmt == HS_MX_E4M3) MXC_LAUNCH(bf16_t, HS_MX_E4M3);
    else MXC_LAUNCH(bf16_t, HS_MX_E2M1);
  }
#undef MXC_LAUNCH
  return launch_status("hs_kv_read_mx");
}
