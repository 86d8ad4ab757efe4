// hs_tree_attention_mx: the kernel for caches of 4-bit elements.
#include "attn_mx_kernel.h"

namespace hs {
void attn_mx_launch_e2m1(const MxAttnArgs& a, unsigned items, hipStream_t stream) { attn_mx_launch<HS_MX_E2M1>(a, items, stream); }
}  // namespace hs
