// Attention over the paged quantized cache at any width from 1 to 1024 and with
// any codebook, in fp32 without matrix instructions: the compatibility path of
// widths (and of codebooks with levels of very different sizes) that
// isoq_attn_m.h does not take.  It is not tuned (4 sequences x 8 x 4 heads x 4,096
// positions, 3 bits: d = 100 66 us, d = 1000 1,150; d = 128 with a codebook of
// distant levels 80, where isoq_attn_m.h takes 12 with an ordinary one).
//
// Workgroup (row = query head of a token, sequence, split), 256 positions at a
// time: each lane sums one key's logit over its record, slot by slot as the
// generic stage-1 kernels write it (the query rotated once into LDS, zero
// padded as in Sec. 5.1); then the lanes are dealt to the rotation slots of the
// values, 256 / slots groups of positions each, and sum p rho c[idx].  The
// running maximum rescales both sums (fp32).
#include "isoq_attn_device.h"

namespace isoq {
namespace {

template <int VAR, int BITS, bool PRE>
__global__ __launch_bounds__(256) void generic_attn_kernel(const AttnArgs a)
{
    constexpr int SW = kGenSW<VAR>;
    constexpr int PS = SW == 8 ? 64 : kSlotParams<VAR>;
    constexpr int K = 1 << BITS;
    extern __shared__ __align__(16) float gsm[];
    float *klev = gsm, *vlev = gsm + 16;
    float *red = gsm + 32;                                    // [8]
    float *wt = gsm + 40;                                     // [256] p rho_v
    int *place = reinterpret_cast<int *>(gsm + 40 + 256);     // [256][2] cache block, position in it
    float *qt = gsm + 40 + 3 * 256;                           // T q scale, slots * SW
    float *sum = qt + a.slots * SW;                           // [256][SW] at the end

    const int s = blockIdx.y, tid = threadIdx.x;
    const int i = blockIdx.x / a.n_q_heads, hq = blockIdx.x - i * a.n_q_heads;
    const int h = hq / a.group;
    const AttnSeq sq = attn_seq<PRE>(a, s);
    if (i >= sq.rows)   // (block-uniform, as every early return here)
        return;
    const int64_t row = (int64_t)(sq.first + i) * a.n_q_heads + hq;
    const int lim = sq.limit(i, a.cap);
    const int64_t t0 = (int64_t)blockIdx.z * a.chunk;
    if (t0 >= lim && blockIdx.z > 0)
        return;   // the join looks at the splits below lim only
    const int tend = (int)min(t0 + a.chunk, (int64_t)lim);

    if (tid < K) {
        klev[tid] = a.k_lev[tid];
        vlev[tid] = a.v_lev[tid];
    }
    const int set = a.k_sets == 1 ? 0 : h;
    bool odd = false;   // an infinity or NaN in the rotated query
    for (int j = tid; j < a.slots; j += 256) {
        float x[SW], y[SW], P[PS];
#pragma unroll
        for (int c = 0; c < SW; c++) {
            const int e = SW * j + c;
            x[c] = e >= a.d    ? 0.f
                   : a.q_f16 ? (float)static_cast<const _Float16 *>(a.q)[row * a.d + e]
                               : static_cast<const float *>(a.q)[row * a.d + e];
        }
        load_params<PS>(a.k_params + set * a.set_stride + (int64_t)j * PS, P);
        if constexpr (SW == 8)
            rotate_forward<VAR>(P, x, y);
        else
            rotate4_forward<VAR>(P, x, y);
#pragma unroll
        for (int c = 0; c < SW; c++)
            y[c] *= a.scale;
#pragma unroll
        for (int c = 0; c < SW; c++) {
            qt[SW * j + c] = y[c];
            odd |= !(fabsf(y[c]) < INFINITY);
        }
    }
    odd = __syncthreads_or(odd);

    // lanes of the second step: slot vj of the positions vg, vg + groups, ...
    const int groups = max(1, 256 / a.slots);
    const int vg = tid / a.slots, vj = tid - vg * a.slots;
    float acc[SW], m = -INFINITY, l = 0.f;
    bool seen = false;   // a position that is there
#pragma unroll
    for (int c = 0; c < SW; c++)
        acc[c] = 0.f;
    const int32_t *table = a.block_table + (int64_t)s * a.max_blocks;

    auto read = [&](const CacheSrcRt &rec, int j) {
        if constexpr (SW == 8)
            return gen_read_slot8<BITS>(rec, j);
        else
            return gen_read_slot_bytes<BITS>(rec, j, a.rec);
    };
    auto source = [&](const uint8_t *base, int blk, int pos) {
        return CacheSrcRt{base + ((int64_t)blk * a.n_kv_heads + h) * a.block_size * a.rec, pos, a.block_size, a.rec_lp,
                          a.rec};
    };
    for (int64_t tb = t0; tb < tend; tb += 256) {
        const int64_t t = tb + tid;
        float v = -INFINITY, rho_k = 0.f, rho_v = 0.f;
        bool ok = false;
        int blk = 0, pos = 0;
        if (t < tend) {
            const AttnEntry e = attn_entry<PRE>(a, sq, table, (int)t);
            blk = e.blk;
            pos = e.pos;
            ok = blk >= 0 && blk < a.n_blocks;
        }
        seen |= ok;
        if (ok) {
            const CacheSrcRt rec = source(a.k_idx, blk, pos);
            float dot = 0.f;
#pragma unroll 4
            for (int j = 0; j < a.slots; j++) {
                const uint32_t p = read(rec, j);
#pragma unroll
                for (int c = 0; c < SW; c++)
                    dot = fmaf(qt[SW * j + c], klev[(p >> (BITS * c)) & (K - 1)], dot);
            }
            const int64_t crow = ((int64_t)blk * a.n_kv_heads + h) * a.block_size + pos;
            rho_k = a.k_rho[crow];
            v = rho_k * dot;
            rho_v = a.v_rho[crow];
        }
        float top = v;
#pragma unroll
        for (int o = 32; o > 0; o >>= 1)
            top = fmaxf(top, __shfl_xor(top, o));
        if ((tid & 63) == 0)
            red[tid >> 6] = top;
        __syncthreads();
        const float mnew = fmaxf(m, fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3])));
        const float mref = mnew == -INFINITY ? 0.f : mnew;
        const float alpha = __builtin_amdgcn_exp2f(m - mref);   // (m = -inf: 0)
        const float p = ok ? __builtin_amdgcn_exp2f(v - mref) : 0.f;
        // (a norm that is an infinity or NaN: NaN in out and lse)
        l = fmaf(l, alpha, fabsf(rho_k) < INFINITY && fabsf(rho_v) < INFINITY ? p : NAN);
        m = mnew;
        wt[tid] = ok ? p * rho_v : 0.f;
        place[2 * tid] = ok ? blk : -1;
        place[2 * tid + 1] = pos;
#pragma unroll
        for (int c = 0; c < SW; c++)
            acc[c] *= alpha;
        __syncthreads();
        const int n = (int)min((int64_t)256, tend - tb);
        if (vg < groups) {
            for (int k = vg; k < n; k += groups) {
                const int b = place[2 * k];
                if (b < 0)
                    continue;
                const uint32_t x = read(source(a.v_idx, b, place[2 * k + 1]), vj);
                const float f = wt[k];
#pragma unroll
                for (int c = 0; c < SW; c++)
                    acc[c] = fmaf(f, vlev[(x >> (BITS * c)) & (K - 1)], acc[c]);
            }
        }
        __syncthreads();
    }
    // l over the lanes, the sums of values over the groups
#pragma unroll
    for (int o = 32; o > 0; o >>= 1)
        l += __shfl_xor(l, o);
    if ((tid & 63) == 0)
        red[4 + (tid >> 6)] = l;
#pragma unroll
    for (int c = 0; c < SW; c++)
        sum[tid * SW + c] = acc[c];
    __syncthreads();
    l = (red[4] + red[5]) + (red[6] + red[7]);
    if (odd && __syncthreads_or(seen))   // (odd is the same in all lanes; the logits may all be -inf: no NaN came up by itself)
        l = NAN;
    const float inv = a.part ? 1.f : l == 0.f ? 0.f : 1.f / l;
    for (int j = tid; j < a.slots; j += 256) {
        float y[SW];
#pragma unroll
        for (int c = 0; c < SW; c++) {
            y[c] = 0.f;
            for (int g = 0; g < groups; g++)
                y[c] += sum[(g * a.slots + j) * SW + c];
            y[c] *= inv;
        }
        if (a.part) {
            float *dst = a.part + attn_part(a, row, blockIdx.z) * a.width + SW * j;
#pragma unroll
            for (int c = 0; c < SW; c++)
                dst[c] = y[c];
        } else {
            attn_emit<VAR, SW>(a, row, h, j, y);
        }
    }
    if (tid == 0) {
        if (a.part) {
            float *ml = a.part_ml + attn_part(a, row, blockIdx.z) * 2;
            ml[0] = m;
            ml[1] = l;
        } else if (a.lse) {
            a.lse[row] = attn_lse(m, l);
        }
    }
}

template <int VAR, bool PRE>
const void *gen_attn_bits(int bits)
{
    switch (bits) {
    case 2: return reinterpret_cast<const void *>(&generic_attn_kernel<VAR, 2, PRE>);
    case 3: return reinterpret_cast<const void *>(&generic_attn_kernel<VAR, 3, PRE>);
    case 4: return reinterpret_cast<const void *>(&generic_attn_kernel<VAR, 4, PRE>);
    }
    return nullptr;
}

}  // namespace

const void *attn_generic_kernel_for(int variant, int bits, bool pre)
{
    switch (variant) {
    case VAR_FULL: return pre ? gen_attn_bits<VAR_FULL, true>(bits) : gen_attn_bits<VAR_FULL, false>(bits);
    case VAR_FAST: return pre ? gen_attn_bits<VAR_FAST, true>(bits) : gen_attn_bits<VAR_FAST, false>(bits);
    case VAR_PLANAR2D: return pre ? gen_attn_bits<VAR_PLANAR2D, true>(bits) : gen_attn_bits<VAR_PLANAR2D, false>(bits);
    case VAR_BLOCK8: return pre ? gen_attn_bits<VAR_BLOCK8, true>(bits) : gen_attn_bits<VAR_BLOCK8, false>(bits);
    }
    return nullptr;
}

size_t attn_generic_lds(int slots, int variant)
{
    const size_t sw = variant == VAR_BLOCK8 ? 8 : 4;
    return sizeof(float) * (40 + 3 * 256 + slots * sw + 256 * sw);
}

}  // namespace isoq
