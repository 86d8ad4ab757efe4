// hs_latent_store, hs_latent_read: rows of latents into and out of a pool, by slots.
//
// A row is R + Dr elements, which come from (go to) two tensors: the latent and the rotary part.  Copies of 16 bytes a thread:
// bound by memory, each row's bytes once in and once out: 30528 rows of 1152 bytes go in in 14.2 us and out in 13.5
// (5.0 and 5.2 TB/s, counting both sides).
#include "attn_common.h"

namespace hs {

constexpr int LR_THREADS = 256;
constexpr int LR_MOST = 4;  // pieces to a thread

struct LrArgs {
  char* c;
  char* r;
  int64_t c_stride, r_stride;  // bytes
  const int64_t* slots;
  char* pool;
  int64_t n_slots, pieces;  // pieces: of all rows
  int c_pieces, row_pieces;
};

template <bool STORE>
__global__ __launch_bounds__(LR_THREADS) void k_latent_rows(LrArgs a) {
  const int64_t first = (int64_t)blockIdx.x * LR_THREADS * LR_MOST;
  const int64_t row0 = first / a.row_pieces;  // (the same for all: a scalar division; a thread's row is few rows on)
  const unsigned rest = (unsigned)(first - row0 * a.row_pieces);
#pragma unroll
  for (int x = 0; x < LR_MOST; ++x) {
    const unsigned at = rest + x * LR_THREADS + threadIdx.x;
    if (first + x * LR_THREADS + threadIdx.x >= a.pieces) return;
    const unsigned dr = at / (unsigned)a.row_pieces, p = at - dr * (unsigned)a.row_pieces;
    const int64_t row = row0 + dr, slot = a.slots[row];
    if (slot < 0 || slot >= a.n_slots) continue;
    char* const in_rows = p < (unsigned)a.c_pieces ? a.c + row * a.c_stride + 16 * (int64_t)p : a.r + row * a.r_stride + 16 * (int64_t)(p - a.c_pieces);
    char* const in_pool = a.pool + (slot * a.row_pieces + p) * 16;
    if (STORE) *reinterpret_cast<uint4*>(in_pool) = *reinterpret_cast<const uint4*>(in_rows);
    else *reinterpret_cast<uint4*>(in_rows) = *reinterpret_cast<const uint4*>(in_pool);
  }
}

static hs_status latent_rows(const char* who, bool store, char* c, int64_t c_stride, char* r, int64_t r_stride, const int64_t* slots, int32_t N, char* pool,
                             int64_t n_slots, int32_t R, int32_t Dr, hs_dtype dt, hs_stream stream) {
  HS_REQUIRE(N >= 0 && n_slots >= 0 && R >= 1 && Dr >= 0, HS_ERR_SHAPE, "%s: N=%d n_slots=%lld R=%d Dr=%d", who, N, (long long)n_slots, R, Dr);
  HS_REQUIRE(dt == HS_F32 || dt == HS_BF16, HS_ERR_SHAPE, "%s: unknown dtype %d", who, (int)dt);
  const int size = dt == HS_F32 ? 4 : 2;
  if (Dr == 0) r = nullptr, r_stride = 0;
  HS_REQUIRE((int64_t)R + Dr <= 1 << 20 && R * size % 16 == 0 && Dr * size % 16 == 0, HS_ERR_UNSUPPORTED, "%s: R and Dr must be multiples of 16 bytes", who);
  HS_REQUIRE(n_slots < (int64_t)1 << 40, HS_ERR_UNSUPPORTED, "%s: n_slots must be below 2^40", who);
  HS_REQUIRE((N <= 1 || c_stride >= R || (store && c_stride >= 0)) && (N <= 1 || Dr == 0 || r_stride >= Dr || (store && r_stride >= 0)), HS_ERR_SHAPE,
             "%s: rows overlap (strides %lld, %lld)", who, (long long)c_stride, (long long)r_stride);
  HS_REQUIRE(c_stride < (int64_t)1 << 40 && r_stride < (int64_t)1 << 40, HS_ERR_UNSUPPORTED, "%s: strides must be below 2^40", who);
  if (N == 0) return HS_OK;
  HS_REQUIRE(c && (r || Dr == 0) && slots && (pool || n_slots == 0), HS_ERR_NULL, "%s: NULL argument", who);
  auto odd = [](const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 != 0; };
  HS_REQUIRE(!odd(c) && !odd(r) && !odd(pool) && (N == 1 || (c_stride * size % 16 == 0 && r_stride * size % 16 == 0)), HS_ERR_UNSUPPORTED,
             "%s: rows must begin at multiples of 16 bytes", who);
  LrArgs a = {c, r, N > 1 ? c_stride * size : 0, N > 1 ? r_stride * size : 0, slots, pool, n_slots, 0, R * size / 16, (R + Dr) * size / 16};
  a.pieces = (int64_t)N * a.row_pieces;
  const int64_t grid = (a.pieces + LR_THREADS * LR_MOST - 1) / (LR_THREADS * LR_MOST);
  HS_REQUIRE(grid < (int64_t)1 << 24, HS_ERR_UNSUPPORTED, "%s: %lld pieces are too many for a call", who, (long long)a.pieces);
  if (store) hipLaunchKernelGGL(k_latent_rows<true>, dim3((unsigned)grid), dim3(LR_THREADS), 0, static_cast<hipStream_t>(stream), a);
  else hipLaunchKernelGGL(k_latent_rows<false>, dim3((unsigned)grid), dim3(LR_THREADS), 0, static_cast<hipStream_t>(stream), a);
  return launch_status(who);
}

}  // namespace hs

using namespace hs;

extern "C" hs_status hs_latent_store(const void* c, int64_t c_stride, const void* r, int64_t r_stride, const int64_t* slots, int32_t N, void* pool,
                                     int64_t n_slots, int32_t R, int32_t Dr, hs_dtype dt, hs_stream stream) {
  clear_error();
  return latent_rows("hs_latent_store", true, const_cast<char*>(static_cast<const char*>(c)), c_stride, const_cast<char*>(static_cast<const char*>(r)), r_stride,
                     slots, N, static_cast<char*>(pool), n_slots, R, Dr, dt, stream);
}

extern "C" hs_status hs_latent_read(const void* pool, int64_t n_slots, const int64_t* slots, int32_t N, void* c, int64_t c_stride, void* r, int64_t r_stride,
                                    int32_t R, int32_t Dr, hs_dtype dt, hs_stream stream) {
  clear_error();
  return latent_rows("hs_latent_read", false, static_cast<char*>(c), c_stride, static_cast<char*>(r), r_stride, slots, N,
                     const_cast<char*>(static_cast<const char*>(pool)), n_slots, R, Dr, dt, stream);
}
