// The join of attention's splits: m = max m_j, l = sum l_j 2^(m_j - m), and the
// sums of values likewise; then the last step of the row (isoq_attn_device.h).
// One wave per row, a rotation slot per lane.  Reads n_splits (width + 2) floats
// a row and writes the row: small next to the cache of any call that splits.
#include "isoq_attn_device.h"

namespace isoq {
namespace {

template <int VAR>
__global__ __launch_bounds__(64 * kAttnJoinRows) void attn_join_kernel(const AttnArgs a)
{
    constexpr int SW = kGenSW<VAR>;
    __shared__ float weight[kAttnJoinRows][kAttnMaxSplits];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const AttnSeq sq = attn_seq(a, blockIdx.y);
    const int r = blockIdx.x * kAttnJoinRows + w;   // token (r / n_q_heads), head (r mod n_q_heads)
    const int i = r / a.n_q_heads, hq = r - i * a.n_q_heads;
    const bool on = i < sq.rows;
    const int64_t row = (int64_t)(sq.first + i) * a.n_q_heads + hq;
    const int lim = on ? sq.limit(i, a.cap) : 0;
    const int ns = (lim + a.chunk - 1) / a.chunk;   // splits that have positions of this row
    const float *ml = a.part_ml + row * a.n_splits * 2;
    float m = -INFINITY;
    for (int j = lane; j < ns; j += 64)
        m = fmaxf(m, ml[2 * j]);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1)
        m = fmaxf(m, __shfl_xor(m, o));
    const float mref = m == -INFINITY ? 0.f : m;
    float l = 0.f;
    for (int j = lane; j < ns; j += 64) {
        const float f = __builtin_amdgcn_exp2f(ml[2 * j] - mref);
        weight[w][j] = f;
        l = fmaf(f, ml[2 * j + 1], l);
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1)
        l += __shfl_xor(l, o);
    __syncthreads();
    if (!on)
        return;
    const float inv = l == 0.f ? 0.f : 1.f / l;
    for (int j = lane; j < a.slots; j += 64) {
        float y[SW];
#pragma unroll
        for (int c = 0; c < SW; c++)
            y[c] = 0.f;
        const float *p = a.part + row * a.n_splits * a.width + SW * j;
#pragma unroll 4
        for (int k = 0; k < ns; k++) {
            const float f = weight[w][k];
            const f32x4 v = *reinterpret_cast<const f32x4 *>(p + (int64_t)k * a.width);
#pragma unroll
            for (int c = 0; c < 4; c++)
                y[c] = fmaf(f, v[c], y[c]);
            if constexpr (SW == 8) {
                const f32x4 u = *reinterpret_cast<const f32x4 *>(p + (int64_t)k * a.width + 4);
#pragma unroll
                for (int c = 0; c < 4; c++)
                    y[4 + c] = fmaf(f, u[c], y[4 + c]);
            }
        }
#pragma unroll
        for (int c = 0; c < SW; c++)
            y[c] *= inv;
        attn_emit<VAR, SW>(a, row, hq / a.group, j, y);
    }
    if (lane == 0 && a.lse)
        a.lse[row] = attn_lse(m, l);
}

}  // namespace

const void *attn_join_kernel_for(int variant)
{
    switch (variant) {
    case VAR_FULL: return reinterpret_cast<const void *>(&attn_join_kernel<VAR_FULL>);
    case VAR_FAST: return reinterpret_cast<const void *>(&attn_join_kernel<VAR_FAST>);
    case VAR_PLANAR2D: return reinterpret_cast<const void *>(&attn_join_kernel<VAR_PLANAR2D>);
    case VAR_BLOCK8: return reinterpret_cast<const void *>(&attn_join_kernel<VAR_BLOCK8>);
    }
    return nullptr;
}

}  // namespace isoq
