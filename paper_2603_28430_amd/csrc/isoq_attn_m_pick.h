// Compile-time dispatch of the matrix-core attention kernels over width, rows
// per workgroup and level digits, for one number of bits; shared by the
// translation units that instantiate them (isoq_attn_m2.hip, _m3, _m4: 2, 3
// and 4 bits).
#pragma once

#include "isoq_attn_m.h"

namespace isoq {
namespace {

template <int D, int BITS, int NT>
AttnKernel attn_m_entry(bool f16)
{
    const size_t lds = sizeof(uint32_t) * AttnMShape<D, BITS, NT>::lds_words();
    return {f16 ? reinterpret_cast<const void *>(&attn_m_kernel<D, BITS, NT, 2>)
                : reinterpret_cast<const void *>(&attn_m_kernel<D, BITS, NT, 3>),
            lds, 4 * NT, false};
}

template <int D, int BITS>
AttnKernel attn_m_rows(int rows, bool f16)
{
    if constexpr (D <= 128) {
        if (rows > 4)
            return attn_m_entry<D, BITS, 2>(f16);
    }
    return attn_m_entry<D, BITS, 1>(f16);
}

template <int BITS>
AttnKernel attn_m_d(int d, int rows, bool f16)
{
    switch (d) {
    case 64: return attn_m_rows<64, BITS>(rows, f16);
    case 80: return attn_m_rows<80, BITS>(rows, f16);
    case 96: return attn_m_rows<96, BITS>(rows, f16);
    case 128: return attn_m_rows<128, BITS>(rows, f16);
    case 160: return attn_m_rows<160, BITS>(rows, f16);
    case 192: return attn_m_rows<192, BITS>(rows, f16);
    case 256: return attn_m_rows<256, BITS>(rows, f16);
    case 512: return attn_m_rows<512, BITS>(rows, f16);
    }
    return {};
}

}  // namespace
}  // namespace isoq
