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

// 4, 8 or 12 rows a workgroup.  A tile is decoded once for them, and the rest of
// its work grows by half of that decoding for every four (about 470 + 255 a four
// vector instructions): 8 in place of two times 4, 12 in place of two times 8 for 9
// to 12 rows.  (For 17 to 24 two times 12 in place of three times 8 gained as often
// as it lost: the registers leave half of the waves.)  Registers allow 12 up to d =
// 128, and 8 up to 256, where 8 rows of 4 bits take all of them and pay from 9 rows on.
// (us with 4 / 8: 4 x 8 heads, 4,096 positions, d = 256, 3 bits: 5 rows 21 / 19, 16
// 34 / 28, 64 99 / 68; 4 bits: 8 rows 29 / 32, 16 44 / 44, 64 129 / 106.  d = 192, 4
// bits, 1 x 8 x 16,384: 8 rows 24 / 23, 16 36 / 29.  12 rows with 8 / 12: d = 128, 3 bits,
// 16 x 8 heads, 4,096 44 / 40; 1 x 8, 32,768 29 / 23; 8 ragged x 8, up to 8,000 34 / 31;
// fp32, 4 bits, 8 x 4, 4,096 24 / 21.  16 rows at once were no faster than two times
// 8: 43 / 44, 30 / 26, 24 / 29.)
template <int D, int BITS>
AttnKernel attn_m_rows(int rows, bool f16)
{
    if constexpr (D <= 128) {
        if (rows > 8 && rows <= 12)
            return attn_m_entry<D, BITS, 3>(f16);
    }
    if constexpr (D <= 256) {
        if (rows > (D == 256 && BITS == 4 ? 8 : 4))
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
