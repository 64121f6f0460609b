// Attention kernels of many rows on the fp16 matrix cores (the kernel template
// is in isoq_attn_c.h).
#include "isoq_attn_c.h"

namespace isoq {
namespace {

template <int D, int BITS>
AttnKernel attn_c_entry()
{
    using C = AttnCShape<D, BITS>;
    return {reinterpret_cast<const void *>(&attn_c_kernel<D, BITS>), (size_t)C::lds_bytes(), C::ROWS, true};
}

template <int D>
AttnKernel attn_c_bits(int bits)
{
    switch (bits) {
    case 2: return attn_c_entry<D, 2>();
    case 3: return attn_c_entry<D, 3>();
    case 4: return attn_c_entry<D, 4>();
    }
    return {};
}

}  // namespace

AttnKernel attn_c_kernel_for(int d, int bits)
{
    switch (d) {
    case 64: return attn_c_bits<64>(bits);
    case 80: return attn_c_bits<80>(bits);
    case 96: return attn_c_bits<96>(bits);
    case 128: return attn_c_bits<128>(bits);
    }
    return {};
}

}  // namespace isoq
