// The attention kernel on a quantised cache (internal): a work item to a workgroup, in the form that its size asks for.
#pragma once
#include "attn_mx_private.h"
#include "attn_mx_shared.h"

namespace hs {

template <int FMT, int D>
__global__ __launch_bounds__(MXA_THREADS) void k_attn_mx(MxAttnArgs a) {
  __shared__ MxLds<D> mem;
  MxItem it;
  if (!mx_item<FMT>(a, blockIdx.x, it)) return;
  switch (it.form) {
    case MX_PRIVATE_1: return attn_mx_private<FMT, D, 1>(a, it, mem);
    case MX_PRIVATE_2: return attn_mx_private<FMT, D, 2>(a, it, mem);
    case MX_SHARED_4: return attn_mx_shared<FMT, D, 2>(a, it, mem);
    default: return attn_mx_shared<FMT, D, 1>(a, it, mem);
  }
}

template <int FMT>
inline void attn_mx_launch(const MxAttnArgs& a, unsigned items, hipStream_t stream) {
  if (a.pool.D == 128) hipLaunchKernelGGL((k_attn_mx<FMT, 128>), dim3(items), dim3(MXA_THREADS), 0, stream, a);
  else hipLaunchKernelGGL((k_attn_mx<FMT, 64>), dim3(items), dim3(MXA_THREADS), 0, stream, a);
}

}  // namespace hs
