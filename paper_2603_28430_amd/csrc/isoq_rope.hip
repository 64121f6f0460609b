// Norms and rotary positions of queries and keys (isoq_qk_norm_rope).  Per row
// (a head of a token) y = weight x / sqrt(mean x^2 + eps), and each of the
// rotated pairs (a, b) becomes
//     amplitude (a cos - b sin, a sin + b cos),  angle = position frequency.
// The angle is exact at any position: a frequency is held as turns in units of
// 2^-64, the product with the position taken modulo 2^64, so whole turns drop out
// without a rounding and the fraction is off by 2^-34 of a turn at most.
#include <hip/hip_runtime.h>

#include "isoq_device.h"
#include "isoq_step.h"

namespace isoq {
namespace {

// cos and sin of p 2^-32 turns: by the Taylor series on an eighth of a turn
// either side of the nearest quarter (cut at x^11 / 11! and x^12 / 12!, 2e-9 and
// 1e-10 at the ends).
__device__ __forceinline__ void turn_cos_sin(uint32_t p, float &c, float &s)
{
    const uint32_t quarter = (p + 0x20000000u) >> 30;
    const float x = (float)(int32_t)(p - (quarter << 30)) * 1.4629180792671596e-9f;   // 2 pi / 2^32
    const float z = x * x;
    float u = fmaf(z, 2.7557319e-6f, -1.9841270e-4f);
    u = fmaf(u, z, 8.3333333e-3f);
    u = fmaf(u, z, -1.6666667e-1f);
    const float sx = fmaf(u * z, x, x);
    float v = fmaf(z, -2.7557319e-7f, 2.4801587e-5f);
    v = fmaf(v, z, -1.3888889e-3f);
    v = fmaf(v, z, 4.1666667e-2f);
    v = fmaf(v, z, -0.5f);
    const float cx = fmaf(v, z, 1.f);
    const float a = quarter & 1 ? sx : cx, b = quarter & 1 ? cx : sx;
    c = (quarter + 1) & 2 ? -a : a;
    s = quarter & 2 ? -b : b;
}

__device__ __forceinline__ uint32_t turns_of(uint64_t per_position, int32_t position)
{
    return (uint32_t)((per_position * (uint64_t)(int64_t)position) >> 32);
}

// A row a wave: lane i has the coordinates i, 64 + i, ... and, for each, the other
// of its pair.
template <bool F16, bool HALVES, int N>
__global__ __launch_bounds__(256) void rope_rows_kernel(const RopeArgs a)
{
    using T = std::conditional_t<F16, _Float16, float>;
    const int lane = threadIdx.x & 63;
    const int64_t r = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int heads = a.heads[0] + a.heads[1];
    const int64_t t = r / heads;
    if (t >= a.n_tokens)
        return;
    const int hh = (int)(r - t * heads), k = hh >= a.heads[0], h = hh - (k ? a.heads[0] : 0);
    const T *x = static_cast<const T *>(a.x[k]) + t * a.stride[k] + (int64_t)h * a.d;
    T *out = static_cast<T *>(a.out[k]) + (t * a.heads[k] + h) * a.d;
    const float *weight = a.weight[k];
    float own[N], other[N], sum = 0.f;
    int partner[N];
#pragma unroll
    for (int i = 0; i < N; i++) {
        const int e = lane + 64 * i;
        partner[i] = e >= 2 * a.half ? e : HALVES ? (e < a.half ? e + a.half : e - a.half) : e ^ 1;
        own[i] = e < a.d ? (float)x[e] : 0.f;
        other[i] = e < a.d ? (float)x[partner[i]] : 0.f;
        sum = fmaf(own[i], own[i], sum);
    }
    float scale = 1.f;
    if (weight) {
#pragma unroll
        for (int o = 32; o > 0; o >>= 1)
            sum += __shfl_xor(sum, o);
        scale = 1.f / sqrtf(sum / (float)a.d + a.eps);
    }
    const int32_t pos = a.positions[t];
#pragma unroll
    for (int i = 0; i < N; i++) {
        const int e = lane + 64 * i;
        if (e >= a.d)
            continue;
        float y = own[i] * scale, z = other[i] * scale;
        if (weight) {
            y *= weight[e];
            z *= weight[partner[i]];
        }
        if (e < 2 * a.half) {
            const int p = HALVES ? (e < a.half ? e : e - a.half) : e >> 1;
            float c, s;
            turn_cos_sin(turns_of(a.turns[p], pos), c, s);
            const bool first = HALVES ? e < a.half : (e & 1) == 0;
            y = a.amplitude * fmaf(y, c, first ? -z * s : z * s);
        }
        out[e] = (T)y;
    }
}

template <bool F16, bool HALVES>
const void *rope_steps(int log2_steps)
{
    switch (log2_steps) {
    case 0: return reinterpret_cast<const void *>(&rope_rows_kernel<F16, HALVES, 1>);
    case 1: return reinterpret_cast<const void *>(&rope_rows_kernel<F16, HALVES, 2>);
    case 2: return reinterpret_cast<const void *>(&rope_rows_kernel<F16, HALVES, 4>);
    case 3: return reinterpret_cast<const void *>(&rope_rows_kernel<F16, HALVES, 8>);
    case 4: return reinterpret_cast<const void *>(&rope_rows_kernel<F16, HALVES, 16>);
    }
    return nullptr;
}

}  // namespace

const void *rope_kernel(bool f16, bool halves, int log2_steps)
{
    return f16 ? (halves ? rope_steps<true, true>(log2_steps) : rope_steps<true, false>(log2_steps))
               : (halves ? rope_steps<false, true>(log2_steps) : rope_steps<false, false>(log2_steps));
}

}  // namespace isoq
