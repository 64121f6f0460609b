// Attention kernels of many rows on the fp16 matrix cores (the kernel template
// is in isoq_attn_c.h).
#include "isoq_attn_c.h"

namespace isoq {
namespace {

template <int D, int BITS, int REST, int W>
AttnKernel attn_c_entry()
{
    using C = AttnCShape<D, BITS, REST, W>;
    return {reinterpret_cast<const void *>(&attn_c_kernel<D, BITS, REST, W>), nullptr, (size_t)C::lds_bytes(), C::ROWS, true, 64 * W};
}

template <int D, int REST, int W>
AttnKernel attn_c_bits(int bits)
{
    switch (bits) {
    case 2: return attn_c_entry<D, 2, REST, W>();
    case 3: return attn_c_entry<D, 3, REST, W>();
    case 4: return attn_c_entry<D, 4, REST, W>();
    }
    return {};
}

template <int REST, int W>
AttnKernel attn_c_d(int d, int bits)
{
    switch (d) {
    case 64: return attn_c_bits<64, REST, W>(bits);
    case 80: return attn_c_bits<80, REST, W>(bits);
    case 96: return attn_c_bits<96, REST, W>(bits);
    case 128: return attn_c_bits<128, REST, W>(bits);
    }
    return {};
}

// 256 rows a workgroup where there are more than 128 (us with 128 / 256 rows; 8 ragged x 16
// heads, up to 1,500 positions: d = 64, 4 bits, 448 rows 76 / 63; d = 128 98 / 84, 400 rows 57 / 53;
// 1,200 rows, d = 64 71 / 60; one sequence's 256 rows 46 / 46, 240 44 / 43, 192 52 / 45; 256 rows
// at 131,071 positions, 8 heads 335 / 268).
template <int REST>
AttnKernel attn_c_rows(int d, int bits, int rows)
{
    return rows > 128 ? attn_c_d<REST, 8>(d, bits) : attn_c_d<REST, 4>(d, bits);
}

}  // namespace

AttnKernel attn_c_kernel_for(int d, int bits, int rest, int rows)
{
    return rest == kRestNone    ? attn_c_rows<kRestNone>(d, bits, rows)
           : rest == kRestBytes ? attn_c_rows<kRestBytes>(d, bits, rows)
                                : attn_c_rows<kRestHalves>(d, bits, rows);
}

}  // namespace isoq
