// The attention kernel on a quantised cache (internal): a work item to a workgroup, in the form that its size asks for.
#pragma once
#include "attn_mx_follow.h"
#include "attn_mx_private.h"
#include "attn_mx_shared.h"

namespace hs {

template <int FMT, int D>
__global__ __launch_bounds__(MXA_THREADS) void k_attn_mx(MxAttnArgs a) {
  __shared__ MxLds<D> mem;
  // the arguments in one batch: left to itself the compiler fetches each where it is first used, one trip after another
  asm volatile("" ::"s"(a.q), "s"(a.k_tree), "s"(a.v_tree), "s"(a.q_stride), "s"(a.k_stride), "s"(a.v_stride), "s"(a.pool.k_codes),
               "s"(a.pool.k_scales), "s"(a.pool.v_codes), "s"(a.pool.v_scales), "s"(a.pool.table), "s"(a.pool.max_blocks), "s"(a.pool.n_pages),
               "s"(a.pool.Hkv), "s"(a.parent), "s"(a.Hq), "s"(a.G), "s"(a.inv_G), "s"(a.c2), "s"(a.o), "s"(a.lse), "s"(a.part), "s"(a.n_entries),
               "s"(a.entries[0].n0), "s"(a.entries[0].M), "s"(a.entries[0].L), "s"(a.entries[0].pages), "s"(a.entries[0].n_sp_form), "s"(a.entries[0].groups));
  MxItem it;
  if (!mx_item(a, blockIdx.x, it)) return;
  bool held;
  switch (it.form) {
    case MX_PRIVATE_1: held = attn_mx_private<FMT, D, 1>(a, it, mem); break;
    case MX_PRIVATE_2: held = attn_mx_private<FMT, D, 2>(a, it, mem); break;
    case MX_SHARED_4: held = attn_mx_shared<FMT, D, 2>(a, it, mem); break;
    default: held = attn_mx_shared<FMT, D, 1>(a, it, mem); break;
  }
  if (!held) {  // (its rows are written again: behind everything that was written)
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    attn_mx_follow<FMT, D>(a, it, mem);
  }
}

template <int FMT>
inline void attn_mx_launch(const MxAttnArgs& a, unsigned items, hipStream_t stream) {
  if (a.pool.D == 128) hipLaunchKernelGGL((k_attn_mx<FMT, 128>), dim3(items), dim3(MXA_THREADS), 0, stream, a);
  else hipLaunchKernelGGL((k_attn_mx<FMT, 64>), dim3(items), dim3(MXA_THREADS), 0, stream, a);
}

}  // namespace hs
