// Attention kernels of many rows on the fp16 matrix cores (the kernel template
// is in isoq_attn_c.h).
#include "isoq_attn_c.h"

namespace isoq {
namespace {

template <int D, int BITS, bool LO>
AttnKernel attn_c_entry()
{
    using C = AttnCShape<D, BITS, LO>;
    return {reinterpret_cast<const void *>(&attn_c_kernel<D, BITS, LO>), (size_t)C::lds_bytes(), C::ROWS, true};
}

template <int D, bool LO>
AttnKernel attn_c_bits(int bits)
{
    switch (bits) {
    case 2: return attn_c_entry<D, 2, LO>();
    case 3: return attn_c_entry<D, 3, LO>();
    case 4: return attn_c_entry<D, 4, LO>();
    }
    return {};
}

template <bool LO>
AttnKernel attn_c_d(int d, int bits)
{
    switch (d) {
    case 64: return attn_c_bits<64, LO>(bits);
    case 80: return attn_c_bits<80, LO>(bits);
    case 96: return attn_c_bits<96, LO>(bits);
    case 128: return attn_c_bits<128, LO>(bits);
    }
    return {};
}

}  // namespace

AttnKernel attn_c_kernel_for(int d, int bits, bool half_keys)
{
    return half_keys ? attn_c_d<false>(d, bits) : attn_c_d<true>(d, bits);
}

}  // namespace isoq
