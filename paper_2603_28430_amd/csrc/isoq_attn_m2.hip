// Matrix-core attention kernels of 2-bit caches (the kernel template is in
// isoq_attn_m.h).
#include "isoq_attn_m_pick.h"

namespace isoq {

AttnKernel attn_m_kernel_b2(int d, int rows, bool f16) { return attn_m_d<2>(d, rows, f16); }

}  // namespace isoq
