// Device helpers shared by the attention kernels: which rows a sequence has,
// and the last step of a row.
#pragma once

#include "isoq_attn.h"
#include "isoq_device.h"
#include "isoq_generic.h"

namespace isoq {
namespace {

// The new tokens of sequence s: rows first .. first + n - 1 of q, of which
// `rows` are computed (max_q_len at most), and its length.
struct AttnSeq {
    int first, n, rows, len;
    // Positions that token i attends to: those up to its own, the newest token
    // being the last position.
    __device__ __forceinline__ int limit(int i, int cap) const
    {
        const int64_t l = (int64_t)len - (n - 1 - i);
        return (int)(l < 0 ? 0 : l < cap ? l : cap);
    }
};

__device__ __forceinline__ AttnSeq attn_seq(const AttnArgs &a, int s)
{
    AttnSeq q{s, 1, 1, a.seq_lens[s]};
    if (a.q_start) {   // (clamped: no row outside q is touched, whatever q_start holds)
        q.first = min(max(a.q_start[s], 0), a.n_tokens);
        q.n = min(max(a.q_start[s + 1], q.first), a.n_tokens) - q.first;
        q.rows = min(q.n, a.max_q_len);
    }
    return q;
}

// Positions per split of a sequence: a.chunk, which the longest possible one needs, or
// (even) what cuts its own length into n_splits equal parts.  Equal parts keep
// the workgroups of a few sequences of many rows busy to the end (two ragged
// chunks of up to 512 tokens and 8,192 positions 185 us instead of 194, mean of six;
// four of 128 and 4,096 88 instead of 98); with one to eight rows a key head they changed
// nothing where the block table is as wide as the longest sequence (16 ragged sequences
// of up to 8,192 positions 44 and 44 us, of others 36 and 36).  Where it is wider and the
// caller gives no max_len, a.chunk is longer than the sequences need (16 sequences of
// 8,192 positions, 8 x 4 heads, a table of 131,072: 86 us instead of 42, one sequence 22
// instead of 11): even parts were not measured there.
__device__ __forceinline__ int attn_chunk(const AttnArgs &a, const AttnSeq &sq)
{
    if (!a.even)
        return a.chunk;
    const uint32_t len = (uint32_t)min(max(sq.len, 0), a.cap), n = (uint32_t)a.n_splits;
    return min(max(128, (int)((len + n - 1) / n + 63) & ~63), a.chunk);
}

// Slot j (SW coordinates) of row `row` (head hq of its token): the sum of
// values y, rotated, rotated back and stored.
template <int VAR, int SW>
__device__ __forceinline__ void attn_emit(const AttnArgs &a, int64_t row, int h, int j, const float y[SW])
{
    constexpr int PS = SW == 8 ? 64 : kSlotParams<VAR>;
    float P[PS], o[SW];
    load_params<PS>(a.v_params + (a.v_sets == 1 ? 0 : h) * a.set_stride + (int64_t)j * PS, P);
    if constexpr (SW == 8)
        rotate_inverse<VAR>(P, y, o);
    else
        rotate4_inverse<VAR>(P, y, o);
    const bool vec = a.d % SW == 0;
    if (a.q_f16)
        gen_store<true, SW>(static_cast<char *>(a.out) + row * a.d * 2, j, a.d, vec, o);
    else
        gen_store<false, SW>(static_cast<char *>(a.out) + row * a.d * 4, j, a.d, vec, o);
}

// lse from m (in units of ln 2) and l.
__device__ __forceinline__ float attn_lse(float m, float l)
{
    return l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * 0.69314718055994531f;
}

}  // namespace
}  // namespace isoq
