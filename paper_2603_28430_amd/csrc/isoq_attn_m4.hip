// Matrix-core attention kernels of 4-bit caches (the kernel template is in
// isoq_attn_m.h).
#include "isoq_attn_m_pick.h"

namespace isoq {

AttnKernel attn_m_kernel_b4(int d, int rows, bool f16) { return attn_m_d<4>(d, rows, f16); }

}  // namespace isoq
