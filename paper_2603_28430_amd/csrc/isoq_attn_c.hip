// Attention kernels of many rows on the fp16 matrix cores (the kernel template
// is in isoq_attn_c.h).
#include "isoq_attn_c.h"

namespace isoq {
namespace {

template <int D, int BITS, int REST>
AttnKernel attn_c_entry()
{
    using C = AttnCShape<D, BITS, REST>;
    return {reinterpret_cast<const void *>(&attn_c_kernel<D, BITS, REST>), (size_t)C::lds_bytes(), C::ROWS, true};
}

template <int D, int REST>
AttnKernel attn_c_bits(int bits)
{
    switch (bits) {
    case 2: return attn_c_entry<D, 2, REST>();
    case 3: return attn_c_entry<D, 3, REST>();
    case 4: return attn_c_entry<D, 4, REST>();
    }
    return {};
}

template <int REST>
AttnKernel attn_c_d(int d, int bits)
{
    switch (d) {
    case 64: return attn_c_bits<64, REST>(bits);
    case 80: return attn_c_bits<80, REST>(bits);
    case 96: return attn_c_bits<96, REST>(bits);
    case 128: return attn_c_bits<128, REST>(bits);
    }
    return {};
}

}  // namespace

AttnKernel attn_c_kernel_for(int d, int bits, int rest)
{
    return rest == kRestNone    ? attn_c_d<kRestNone>(d, bits)
           : rest == kRestBytes ? attn_c_d<kRestBytes>(d, bits)
                                : attn_c_d<kRestHalves>(d, bits);
}

}  // namespace isoq
