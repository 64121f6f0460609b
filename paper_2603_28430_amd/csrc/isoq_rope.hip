// Norms and rotary positions of queries and keys (isoq_qk_norm_rope).  Per row
// (a head of a token) y = weight x / sqrt(mean x^2 + eps), and each of the
// rotated pairs (a, b) becomes
//     amplitude (a cos - b sin, a sin + b cos),  angle = position frequency.
// A frequency is held as turns in units of 2^-64 (off by up to two of them, the division's
// and the cut), the product with the position taken modulo 2^64, so whole turns drop out
// without a rounding; its upper 32 bits are what is used.  At the farthest positions, 2^31, the
// angle is off by 2^-32 of a turn of the first and 2^-32 of the second at most (1.5 2^-32 the
// worst of 700 frequencies up to a turn a position at 8 positions each).
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

// Any other width (pairs of an odd width or place): a row a wave; lane i has the coordinates i,
// 64 + i, ... and, for each, the other of its pair.  Bound by its instructions, cos and sin of every
// element among them.
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

// CH elements as one access.
template <bool F16, int CH>
struct RopeChunk {
    using T = std::conditional_t<F16, _Float16, float>;
    T x[CH];
    __device__ __forceinline__ void load(const T *p)
    {
        if constexpr (CH * sizeof(T) == 16) {
            const u32x4 v = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(p));
            __builtin_memcpy(x, &v, 16);
        } else {
            __builtin_memcpy(x, __builtin_assume_aligned(p, CH * sizeof(T)), CH * sizeof(T));
        }
    }
    __device__ __forceinline__ void store(T *p) const
    {
        __builtin_memcpy(__builtin_assume_aligned(p, CH * sizeof(T)), x, CH * sizeof(T));
    }
};

// Rows by chunks of CH coordinates (16 bytes where widths and places allow it).  L
// lanes have a row, a wave 64 / L rows of one token at a time; a lane has two chunks,
// half of the rotated part (or of the rest) apart, so that both layouts have their pairs
// in one lane: coordinates i of both chunks, or 2 i and 2 i + 1 of each.  cos and sin
// are a lane's own for all of its token's rows, with the weight and the amplitude
// multiplied in: a pair is four products of its two coordinates.
//
// What bounds it: memory.  32,768 tokens of 32 + 8 heads, d = 128, fp16, 671 MB: 125
// us, 5.4 TB/s, where a large copy moves 4.8.  (A row a wave with cos and sin for every
// element, rope_rows_kernel: 789.)  32 tokens: 4 us, next to its launch; the binding's
// host time, 9 us, is what a call takes.  4,133 tokens of 10 heads, d = 90, fp32, in chunks of
// two: 30 MB, 9 us (rope_rows_kernel 14).
template <bool F16, bool HALVES, int CH, int L>
__global__ __launch_bounds__(256) void rope_tile_kernel(const RopeArgs a)
{
    static_assert(HALVES || CH % 2 == 0, "pairs inside a chunk");
    constexpr int V = 64 / L;
    using Chunk = RopeChunk<F16, CH>;
    using T = typename Chunk::T;
    const int lane = threadIdx.x & 63, sub = lane & (L - 1), g = lane / L;
    const uint32_t wid = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t t = wid / (uint32_t)a.parts, part = wid - t * a.parts;
    if (t >= (uint32_t)a.n_tokens)
        return;
    // chunks that rotate, that are passed on; lanes for each
    const int cr = 2 * a.half / CH, cz = (a.d - 2 * a.half) / CH, nr = (cr + 1) / 2, nz = (cz + 1) / 2;
    const bool turned = sub < nr, there = sub < nr + nz;
    const int ka = turned ? sub : sub - nr, kb = ka + (turned ? nr : nz);
    const bool both = kb < (turned ? cr : cz);   // (an odd chunk has no other)
    const int oa = (turned ? 0 : 2 * a.half) + ka * CH, ob = oa + (both ? (kb - ka) * CH : 0);

    float c[CH], s[CH];
    if (turned) {
        const int32_t pos = a.positions[t];
#pragma unroll
        for (int i = 0; i < CH; i++) {
            const int p = HALVES ? oa + i : i < CH / 2 ? oa / 2 + i : ob / 2 + i - CH / 2;
            turn_cos_sin(turns_of(a.turns[p], pos), c[i], s[i]);
        }
    }
    const int its[2] = {(a.heads[0] + V - 1) / V, (a.heads[1] + V - 1) / V}, all = its[0] + its[1];
    const int from = (int)(part * (uint32_t)all / (uint32_t)a.parts), to = (int)((part + 1) * (uint32_t)all / (uint32_t)a.parts);
#pragma unroll 1
    for (int k = 0; k < 2; k++) {
        const int lo = max(from - (k ? its[0] : 0), 0), hi = min(to - (k ? its[0] : 0), its[k]);
        if (lo >= hi)
            continue;
        const float *weight = a.weight[k];
        float wa[CH], wb[CH];
#pragma unroll
        for (int i = 0; i < CH; i++)
            wa[i] = wb[i] = 1.f;
        if (weight && there) {
#pragma unroll
            for (int i = 0; i < CH; i++) {
                wa[i] = weight[oa + i];
                wb[i] = weight[ob + i];
            }
        }
        // pair i: (x, y) -> (x cx - y sy, x sx + y cy)
        float cx[CH], sx[CH], cy[CH], sy[CH];
#pragma unroll
        for (int i = 0; i < CH; i++) {
            const float wx = HALVES ? wa[i] : i < CH / 2 ? wa[2 * i % CH] : wb[2 * i % CH];
            const float wy = HALVES ? wb[i] : i < CH / 2 ? wa[(2 * i + 1) % CH] : wb[(2 * i + 1) % CH];
            const float ca = a.amplitude * c[i], sa = a.amplitude * s[i];
            cx[i] = wx * ca;
            sx[i] = wx * sa;
            cy[i] = wy * ca;
            sy[i] = wy * sa;
        }
        const int heads = a.heads[k];
        const T *x = static_cast<const T *>(a.x[k]) + t * a.stride[k];
        T *out = static_cast<T *>(a.out[k]) + (int64_t)t * heads * a.d;
        Chunk ra, rb, na{}, nb{};
        auto load = [&](int it) {
            const int h = it * V + g;
            if (there && h < heads) {
                na.load(x + (int64_t)h * a.d + oa);
                nb.load(x + (int64_t)h * a.d + ob);
            }
        };
        load(lo);
        for (int it = lo; it < hi; it++) {
            ra = na;
            rb = nb;
            if (it + 1 < hi)
                load(it + 1);
            float xa[CH], xb[CH];
#pragma unroll
            for (int i = 0; i < CH; i++) {
                xa[i] = (float)ra.x[i];
                xb[i] = (float)rb.x[i];
            }
            if (weight) {   // (uniform)
                float sum = 0.f;
                if (there) {
#pragma unroll
                    for (int i = 0; i < CH; i++) {
                        const float other = both ? xb[i] : 0.f;   // (in both factors: 0 times an infinity is no number)
                        sum = fmaf(other, other, fmaf(xa[i], xa[i], sum));
                    }
                }
                const float scale = 1.f / sqrtf(row_sum<L>(sum) / (float)a.d + a.eps);
#pragma unroll
                for (int i = 0; i < CH; i++) {
                    xa[i] *= scale;
                    xb[i] *= scale;
                }
            }
            float ya[CH], yb[CH];
            if (turned) {
#pragma unroll
                for (int i = 0; i < CH; i++) {
                    const float px = HALVES ? xa[i] : i < CH / 2 ? xa[2 * i % CH] : xb[2 * i % CH];
                    const float py = HALVES ? xb[i] : i < CH / 2 ? xa[(2 * i + 1) % CH] : xb[(2 * i + 1) % CH];
                    const float u = fmaf(px, cx[i], -(py * sy[i])), v = fmaf(px, sx[i], py * cy[i]);
                    if constexpr (HALVES) {
                        ya[i] = u;
                        yb[i] = v;
                    } else {
                        (i < CH / 2 ? ya : yb)[2 * i % CH] = u;
                        (i < CH / 2 ? ya : yb)[(2 * i + 1) % CH] = v;
                    }
                }
            } else {
#pragma unroll
                for (int i = 0; i < CH; i++) {
                    ya[i] = xa[i] * wa[i];
                    yb[i] = xb[i] * wb[i];
                }
            }
#pragma unroll
            for (int i = 0; i < CH; i++) {
                ra.x[i] = (T)ya[i];
                rb.x[i] = (T)yb[i];
            }
            const int h = it * V + g;
            if (there && h < heads) {
                ra.store(out + (int64_t)h * a.d + oa);
                if (both)
                    rb.store(out + (int64_t)h * a.d + ob);
            }
        }
    }
}

template <bool F16, bool HALVES, int CH>
const void *rope_lanes(int lanes)
{
    switch (lanes) {
    case 4: return reinterpret_cast<const void *>(&rope_tile_kernel<F16, HALVES, CH, 4>);
    case 8: return reinterpret_cast<const void *>(&rope_tile_kernel<F16, HALVES, CH, 8>);
    case 16: return reinterpret_cast<const void *>(&rope_tile_kernel<F16, HALVES, CH, 16>);
    case 32: return reinterpret_cast<const void *>(&rope_tile_kernel<F16, HALVES, CH, 32>);
    case 64: return reinterpret_cast<const void *>(&rope_tile_kernel<F16, HALVES, CH, 64>);
    }
    return nullptr;
}

template <bool F16, bool HALVES>
const void *rope_chunks(int chunk, int lanes)
{
    if constexpr (HALVES)
        if (chunk == 1)
            return rope_lanes<F16, HALVES, 1>(lanes);
    return chunk == 2 ? rope_lanes<F16, HALVES, 2>(lanes) : rope_lanes<F16, HALVES, F16 ? 8 : 4>(lanes);
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

const void *rope_tile_kernel_for(bool f16, bool halves, int chunk, int lanes)
{
    return f16 ? (halves ? rope_chunks<true, true>(chunk, lanes) : rope_chunks<true, false>(chunk, lanes))
               : (halves ? rope_chunks<false, true>(chunk, lanes) : rope_chunks<false, false>(chunk, lanes));
}

const void *rope_kernel(bool f16, bool halves, int log2_steps)
{
    return f16 ? (halves ? rope_steps<true, true>(log2_steps) : rope_steps<true, false>(log2_steps))
               : (halves ? rope_steps<false, true>(log2_steps) : rope_steps<false, false>(log2_steps));
}

}  // namespace isoq
