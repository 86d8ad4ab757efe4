// hs_tree_attention_mx: the kernel for caches of 8-bit elements.
#include "attn_mx_kernel.h"

namespace hs {
void attn_mx_launch_e4m3(const MxAttnArgs& a, unsigned items, hipStream_t stream) { attn_mx_launch<HS_MX_E4M3>(a, items, stream); }
}  // namespace hs
