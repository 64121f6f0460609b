// The join of attention's splits: m = max m_j, l = sum l_j 2^(m_j - m), and the
// sums of values likewise; then the last step of the row (isoq_attn_device.h).
//
// Up to kAttnJoinFew splits (attn_join_few_kernel): a lane has a rotation slot of
// a row, reads every split's m and l itself, and adds up; 256 / slots rows per
// workgroup.  Bound by what it reads and writes (a chunk of 512 tokens, 32
// heads, d = 128: n_splits x 8 MB; two of them in 2 splits 9 to 11 us), and by its
// launch where that is little (3 to 5 us).
//
// More (attn_join_kernel): one workgroup per row.  A lane has a split's m and l (kAttnMaxSplits of them
// at most), then a rotation slot of the splits g, g + groups, ... (256 / slots
// groups, summed through LDS).  It reads n_splits (width + 2) floats a row: little
// next to the cache of any call that splits, so the chain of dependent loads
// is what it takes, 4 to 5 us (64 rows of 86 splits, 512 rows of 11): the first
// splits' sums are asked for together with m and l.  Behind a prefix a row's further splits
// are the prefix's (2,048 rows of 32 + 4 splits, 38 MB, 10 us: memory).
#include "isoq_attn_device.h"

namespace isoq {
namespace {

// A row's splits: `own` of its sequence from `at` on, then `all - own` of its
// prefix, `jump` places further (in part and part_ml).
struct RowSplits {
    int64_t at;
    int own, all, jump;
    __device__ __forceinline__ int64_t place(int k) const { return at + k + (k < own ? 0 : jump); }
};
// (without a prefix jump is 0, and place() waits for no length)

// The splits that have positions of token i of sequence s (all = -1: the row is left
// as it is).
template <bool PREFIX>
__device__ __forceinline__ RowSplits row_splits(const AttnArgs &a, const AttnPrefix &p, const AttnSeq &sq, int s, int i,
                                                int64_t row)
{
    const int own = splits_of(sq.limit(i, a.cap), attn_chunk(a, sq));
    RowSplits r{row * a.part_splits, PREFIX ? own : 0, own, 0};
    if constexpr (PREFIX) {
        const PrefixOf g = prefix_of(a, p.start, p.n, p.n_seqs, s);
        if (g.any) {
            if (sq.first + i - g.token >= p.max_tokens) {
                r.all = -1;
                return r;
            }
            const int len = p.lens[g.index];
            r.all += splits_of(min(max(len, 0), p.cap), attn_chunk(len, p.even, p.cap, p.n_splits, p.chunk));
            r.jump = a.n_splits - r.own;
        }
    }
    return r;
}

template <int VAR, bool PREFIX, bool PRE>
__device__ __forceinline__ void attn_join_row(const AttnArgs &a, const AttnPrefix &pre)
{
    constexpr int SW = kGenSW<VAR>, AHEAD = 4;
    __shared__ float weight[kAttnMaxSplits], red[8];
    __shared__ float sum[256 * SW];
    static_assert(kAttnMaxSplits <= 256, "a split per lane");
    const int tid = threadIdx.x;
    const AttnSeq sq = attn_seq<PRE>(a, blockIdx.y);
    const int i = blockIdx.x / a.n_q_heads, hq = blockIdx.x - i * a.n_q_heads;
    if (i >= sq.rows)
        return;
    const int64_t row = (int64_t)(sq.first + i) * a.n_q_heads + hq;
    const RowSplits rs = row_splits<PREFIX>(a, pre, sq, blockIdx.y, i, row);
    const int ns = rs.all;
    if (PREFIX && ns < 0)   // (block-uniform)
        return;
    const int groups = max(1, 256 / a.slots);
    const int g = tid / a.slots, j = tid - g * a.slots;
    f32x4 v[AHEAD][SW / 4];
    const int last = PREFIX ? max(0, ns - 1) : a.n_splits - 1;   // (of one sequence's own splits: before their number is known)
    auto load = [&](int k, f32x4 *x) {   // (past the last split: that one again, not used)
        const f32x4 *src = reinterpret_cast<const f32x4 *>(a.part + rs.place(min(k, last)) * a.width + SW * j);
#pragma unroll
        for (int c = 0; c < SW / 4; c++)
            x[c] = src[c];
    };
#pragma unroll
    for (int u = 0; u < AHEAD; u++)
        load(g + u * groups, v[u]);
    const float *ml = a.part_ml + rs.place(min(tid, last)) * 2;
    float m = ml[0], l = ml[1];
    if (tid >= ns) {
        m = -INFINITY;
        l = 0.f;
    }
    float top = m;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1)
        top = fmaxf(top, __shfl_xor(top, o));
    if ((tid & 63) == 0)
        red[tid >> 6] = top;
    __syncthreads();
    top = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
    const float f = __builtin_amdgcn_exp2f(m - (top == -INFINITY ? 0.f : top));
    weight[tid] = f;
    l *= f;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1)
        l += __shfl_xor(l, o);
    if ((tid & 63) == 0)
        red[4 + (tid >> 6)] = l;
    __syncthreads();
    l = (red[4] + red[5]) + (red[6] + red[7]);
    float y[SW];
#pragma unroll
    for (int c = 0; c < SW; c++)
        y[c] = 0.f;
    if (g < groups) {
        for (int k0 = g; k0 < ns; k0 += AHEAD * groups) {
#pragma unroll
            for (int u = 0; u < AHEAD; u++) {
                const int k = k0 + u * groups;
                if (k < ns) {
                    const float w = weight[k];
#pragma unroll
                    for (int c = 0; c < SW; c++)
                        y[c] = fmaf(w, v[u][c / 4][c % 4], y[c]);
                }
            }
#pragma unroll
            for (int u = 0; u < AHEAD; u++)
                if (k0 + AHEAD * groups < ns)
                    load(k0 + (AHEAD + u) * groups, v[u]);
        }
    }
#pragma unroll
    for (int c = 0; c < SW; c++)
        sum[tid * SW + c] = y[c];
    __syncthreads();
    if (tid < a.slots) {
        const float inv = l == 0.f ? 0.f : 1.f / l;
        for (int x = 1; x < groups; x++)
#pragma unroll
            for (int c = 0; c < SW; c++)
                y[c] += sum[(x * a.slots + tid) * SW + c];
#pragma unroll
        for (int c = 0; c < SW; c++)
            y[c] *= inv;
        attn_emit<VAR, SW>(a, row, hq / a.group, tid, y);
    }
    if (tid == 0 && a.lse)
        a.lse[row] = attn_lse(top, l);
}

template <int VAR, bool PREFIX, bool PRE>
__device__ __forceinline__ void attn_join_rows(const AttnArgs &a, const AttnPrefix &pre)
{
    constexpr int SW = kGenSW<VAR>, N = kAttnJoinFew;
    const AttnSeq sq = attn_seq<PRE>(a, blockIdx.y);
    const int g = threadIdx.x / a.slots, j = threadIdx.x - g * a.slots, per = 256 / a.slots;
    const int r = blockIdx.x * per + g, i = r / a.n_q_heads, hq = r - i * a.n_q_heads;
    if (g >= per || i >= sq.rows)
        return;
    const int64_t row = (int64_t)(sq.first + i) * a.n_q_heads + hq;
    const RowSplits rs = row_splits<PREFIX>(a, pre, sq, blockIdx.y, i, row);
    const int ns = rs.all;
    if (PREFIX && ns < 0)
        return;
    float m[N], top = -INFINITY, l = 0.f, y[SW];
    f32x4 v[N][SW / 4];
#pragma unroll
    for (int k = 0; k < N; k++)
        if (k < ns) {
            m[k] = a.part_ml[rs.place(k) * 2];
#pragma unroll
            for (int c = 0; c < SW / 4; c++)
                v[k][c] = *reinterpret_cast<const f32x4 *>(a.part + rs.place(k) * a.width + SW * j + 4 * c);
        }
#pragma unroll
    for (int k = 0; k < N; k++)
        if (k < ns)
            top = fmaxf(top, m[k]);
    const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll
    for (int c = 0; c < SW; c++)
        y[c] = 0.f;
#pragma unroll
    for (int k = 0; k < N; k++)
        if (k < ns) {
            const float f = __builtin_amdgcn_exp2f(m[k] - ref);
            l = fmaf(f, a.part_ml[rs.place(k) * 2 + 1], l);
#pragma unroll
            for (int c = 0; c < SW; c++)
                y[c] = fmaf(f, v[k][c / 4][c % 4], y[c]);
        }
    const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
    for (int c = 0; c < SW; c++)
        y[c] *= inv;
    attn_emit<VAR, SW>(a, row, hq / a.group, j, y);
    if (j == 0 && a.lse)
        a.lse[row] = attn_lse(top, l);
}

template <int VAR, bool PRE>
__global__ __launch_bounds__(256) void attn_join_kernel(const AttnArgs a)
{
    attn_join_row<VAR, false, PRE>(a, AttnPrefix{});
}

template <int VAR, bool PRE>
__global__ __launch_bounds__(256) void attn_join_few_kernel(const AttnArgs a)
{
    attn_join_rows<VAR, false, PRE>(a, AttnPrefix{});
}

template <int VAR>
__global__ __launch_bounds__(256) void attn_prefix_join_kernel(const AttnArgs a, const AttnPrefix p)
{
    attn_join_row<VAR, true, false>(a, p);
}

template <int VAR>
__global__ __launch_bounds__(256) void attn_prefix_join_few_kernel(const AttnArgs a, const AttnPrefix p)
{
    attn_join_rows<VAR, true, false>(a, p);
}

// Splits of the sequences' own positions (kOwn), with a prefix ahead of them (kAhead), and of
// both (kBoth).
enum JoinOf { kOwn, kAhead, kBoth };

template <int VAR>
const void *join_kernel(JoinOf of, bool few)
{
    switch (of) {
    case kOwn:
        return few ? reinterpret_cast<const void *>(&attn_join_few_kernel<VAR, false>)
                   : reinterpret_cast<const void *>(&attn_join_kernel<VAR, false>);
    case kAhead:
        return few ? reinterpret_cast<const void *>(&attn_join_few_kernel<VAR, true>)
                   : reinterpret_cast<const void *>(&attn_join_kernel<VAR, true>);
    case kBoth:
        return few ? reinterpret_cast<const void *>(&attn_prefix_join_few_kernel<VAR>)
                   : reinterpret_cast<const void *>(&attn_prefix_join_kernel<VAR>);
    }
    return nullptr;
}

const void *join_of(int variant, JoinOf of, bool few)
{
    switch (variant) {
    case VAR_FULL: return join_kernel<VAR_FULL>(of, few);
    case VAR_FAST: return join_kernel<VAR_FAST>(of, few);
    case VAR_PLANAR2D: return join_kernel<VAR_PLANAR2D>(of, few);
    case VAR_BLOCK8: return join_kernel<VAR_BLOCK8>(of, few);
    }
    return nullptr;
}

}  // namespace

const void *attn_join_kernel_for(int variant, bool few, bool pre) { return join_of(variant, pre ? kAhead : kOwn, few); }
const void *attn_prefix_join_kernel_for(int variant, bool few) { return join_of(variant, kBoth, few); }

}  // namespace isoq
