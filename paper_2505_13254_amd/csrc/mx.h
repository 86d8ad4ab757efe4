// Quantised KV caches (internal): what their bytes mean, and the conversions.
//
// A cache is a pool of pages of 64 tokens, codes [n_pages, Hkv, 64, D] and scales [n_pages, Hkv, 64, D / 32]: a head's
// tokens of a page are one piece of memory, which is what an attention workgroup streams.  32 neighbours of a row
// share a power of two 2^e, stored as the byte e + 127, and an element is an 8-bit (e4m3) or 4-bit (e2m1) floating
// point number x / 2^e.  e is the least one for which the largest magnitude of the 32 is representable (nothing
// saturates), -100 at least, so that no product is subnormal.  A code times a power of two has at most four significant
// bits: it is a bfloat16 without rounding, and one conversion instruction of the card takes two codes and the scale to
// two bfloat16.  Byte 255 (a NaN or an infinity was among the 32) reads as NaN in every element.
#pragma once
#include "attn_common.h"

namespace hs {

constexpr int MX_PAGE = HS_MX_PAGE;
constexpr int MX_BLOCK = HS_MX_BLOCK;
constexpr int MX_LEAST = 27;  // least scale byte: 2^-100

typedef __bf16 mx_bf16x2 __attribute__((ext_vector_type(2)));
typedef short mx_s16x2 __attribute__((ext_vector_type(2)));

template <int FMT>
struct Mx;
template <>
struct Mx<HS_MX_E4M3> {
  static constexpr int BITS = 8, EMAX = 8;            // largest 448 = 1.75 * 2^8
  static constexpr unsigned TOP = 0x600000u;          // mantissa of 1.75
};
template <>
struct Mx<HS_MX_E2M1> {
  static constexpr int BITS = 4, EMAX = 2;            // largest 6 = 1.5 * 2^2
  static constexpr unsigned TOP = 0x400000u;          // mantissa of 1.5
};
__host__ __device__ constexpr int mx_row_bytes(int fmt, int D) { return fmt == HS_MX_E4M3 ? D : D / 2; }

// Memory that a pointer out of an asm statement is known to be (of a generic one the loads would be waited for all together).
typedef const __attribute__((address_space(1))) unsigned char* mx_mem;
typedef __attribute__((ext_vector_type(4))) unsigned mx_u4;
__device__ __forceinline__ uint4 mx_load16(mx_mem p) {
  const mx_u4 v = *reinterpret_cast<const __attribute__((address_space(1))) mx_u4*>(p);
  return make_uint4(v[0], v[1], v[2], v[3]);
}

// A cache as the kernels see it.
struct MxPool {
  unsigned char* k_codes;
  unsigned char* k_scales;
  unsigned char* v_codes;
  unsigned char* v_scales;
  const int32_t* table;  // [B, max_blocks]
  int max_blocks, n_pages, Hkv, D;
};

// Scale byte of 32 values whose largest magnitude has these bits (NaN and infinity compare largest).
template <int FMT>
__device__ __forceinline__ unsigned mx_scale_byte(unsigned amax) {
  const int e = (int)(amax >> 23) - Mx<FMT>::EMAX + ((amax & 0x7fffffu) > Mx<FMT>::TOP ? 1 : 0);
  return amax >= 0x7f800000u ? 255u : (unsigned)(e < MX_LEAST ? MX_LEAST : e);
}
__device__ __forceinline__ float mx_scale(unsigned byte) { return __builtin_bit_cast(float, byte << 23); }

// Two elements of four (e4m3) or eight (e2m1) in a word: pair P as bfloat16, exact.
template <int FMT, int P>
__device__ __forceinline__ unsigned mx_pair(unsigned word, float scale) {
  if constexpr (FMT == HS_MX_E4M3)
    return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)word, scale, P & 1));
  else
    return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, P & 3));
}
// Eight elements as four words of bfloat16 pairs: of e4m3 from two words, of e2m1 from one.
template <int FMT>
__device__ __forceinline__ uint4 mx_eight(unsigned w0, unsigned w1, float scale) {
  uint4 r;
  if constexpr (FMT == HS_MX_E4M3) {
    r.x = mx_pair<FMT, 0>(w0, scale);
    r.y = mx_pair<FMT, 1>(w0, scale);
    r.z = mx_pair<FMT, 0>(w1, scale);
    r.w = mx_pair<FMT, 1>(w1, scale);
  } else {
    r.x = mx_pair<FMT, 0>(w0, scale);
    r.y = mx_pair<FMT, 1>(w0, scale);
    r.z = mx_pair<FMT, 2>(w0, scale);
    r.w = mx_pair<FMT, 3>(w0, scale);
  }
  return r;
}

// The sequence of row `row` among B sequences packed by off [B+1] (rising): the last s with off[s] <= row.  Every lane of
// the wave takes part, `row` is the same for all of them.
template <typename T>
__device__ __forceinline__ int seq_of_row(const T* off, int B, int64_t row) {
  const int lane = (int)(threadIdx.x & 63);
  int s = 0;
  for (int base = 0; base < B; base += 64) {
    const bool below = base + lane < B && (int64_t)off[base + lane] <= row;
    const int n = __builtin_popcountll(__ballot(below));
    s = base + n - 1;
    if (n < 64) break;
  }
  return s < 0 ? 0 : s;
}

}  // namespace hs
