// Device helpers shared by the attention kernels: which rows a sequence has,
// and the last step of a row.
#pragma once

#include "isoq_attn.h"
#include "isoq_device.h"
#include "isoq_generic.h"

namespace isoq {
namespace {

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
__device__ __forceinline__ int attn_chunk(int len, int even, int cap, int n_splits, int chunk)
{
    if (!even)
        return chunk;
    const uint32_t l = (uint32_t)min(max(len, 0), cap), n = (uint32_t)n_splits;
    return min(max(128, (int)((l + n - 1) / n + 63) & ~63), chunk);
}

__device__ __forceinline__ int splits_of(int positions, int chunk)
{
    return (int)(((uint32_t)positions + (uint32_t)chunk - 1u) / (uint32_t)chunk);
}

// The prefix that sequence s has of `n` (start[p] .. start[p + 1] - 1 share prefix p;
// start null: all share one), or none, and the first of its tokens.
struct PrefixOf {
    int index, token;
    bool any;
};

__device__ __forceinline__ PrefixOf prefix_of(const AttnArgs &a, const int32_t *start, int n, int n_seqs, int s)
{
    PrefixOf p{0, 0, true};
    int first = 0, end = n_seqs;
    if (start) {
        for (int hi = n; p.index + 1 < hi;) {
            const int mid = (p.index + hi) >> 1;
            if (start[mid] <= s)
                p.index = mid;
            else
                hi = mid;
        }
        first = max(start[p.index], 0);
        end = start[p.index + 1];
    }
    p.any = s >= first && s < end;
    p.token = a.q_start ? min(max(a.q_start[min(first, n_seqs)], 0), a.n_tokens) : first;
    return p;
}

// The new tokens of sequence s: rows first .. first + n - 1 of q, of which
// `rows` are computed (max_q_len at most), and its length.
struct AttnSeq {
    int first, n, rows, len, full;
    int base, prefix;   // positions of its prefix that come first, which prefix (0: none, or the first)
    int folded;         // splits of its prefix to be added
    // Positions that token i attends to: all, or those up to its own, the newest
    // token being the last position.
    __device__ __forceinline__ int limit(int i, int cap) const
    {
        const int64_t l = (int64_t)len - (full ? 0 : n - 1 - i);
        return base + (int)(l < 0 ? 0 : l < cap ? l : cap);
    }
};

// (PRE: launches with n_pre > 0, whose kernels are instantiations of their own: what they ask
// for took the others 1 to 2%)
template <bool PRE>
__device__ __forceinline__ AttnSeq attn_seq(const AttnArgs &a, int s)
{
    AttnSeq q{s, 1, 1, a.seq_lens[s], a.full, 0, 0, 0};
    if (a.n_all > 0) {   // (clamped likewise)
        const int from = a.shared ? min(max(a.shared[s], 0), a.n_all) : 0;
        const int to = a.shared ? min(max(a.shared[s + 1], from), a.n_all) : a.n_all;
        q.first = a.q_start ? min(max(a.q_start[from], 0), a.n_tokens) : from;
        q.n = (a.q_start ? min(max(a.q_start[to], q.first), a.n_tokens) : to) - q.first;
        q.rows = min(q.n, a.max_q_len);
    } else if (a.q_start) {   // (clamped: no row outside q is touched, whatever q_start holds)
        q.first = min(max(a.q_start[s], 0), a.n_tokens);
        q.n = min(max(a.q_start[s + 1], q.first), a.n_tokens) - q.first;
        q.rows = min(q.n, a.max_q_len);
    }
    if constexpr (PRE) {
        const PrefixOf p = prefix_of(a, a.pre_start, a.n_pre, a.n_seqs, s);
        if (p.any) {
            q.prefix = p.index;
            const int len = min(max(a.pre_lens[p.index], 0), a.pre_cap);
            if (a.fold > 0)
                q.folded = splits_of(len, attn_chunk(len, a.pre_even, a.pre_cap, a.fold, a.pre_chunk));
            else
                q.base = len;
            q.rows = min(q.rows, max(a.pre_tokens - (q.first - p.token), 0));
        }
    }
    return q;
}

// Position t's entry of the block tables: its prefix's, then its own.
struct AttnEntry {
    int32_t blk, pos;   // cache block and position in it
};

template <bool PRE>
__device__ __forceinline__ AttnEntry attn_entry(const AttnArgs &a, const AttnSeq &sq, const int32_t *table, int t)
{
    uint32_t tt = (uint32_t)min(t, a.cap - 1);
    if constexpr (PRE) {
        const bool own = t >= sq.base && a.cap > 0;
        tt = (uint32_t)(own ? min(t - sq.base, a.cap - 1) : min(t, a.pre_cap - 1));
        table = own ? table : a.pre_table + (int64_t)sq.prefix * a.pre_blocks;
    }
    const uint32_t bi = fast_div(tt, a.div_block);
    return AttnEntry{table[bi], (int)(tt - bi * a.block_size)};
}

__device__ __forceinline__ int attn_chunk(const AttnArgs &a, const AttnSeq &sq)
{
    return attn_chunk(sq.len, a.even, a.cap, a.n_splits, a.chunk);
}

// Where a launch's split z of a row is, in part and part_ml.
__device__ __forceinline__ int64_t attn_part(const AttnArgs &a, int64_t row, int z)
{
    return row * a.part_splits + a.part_first + z;
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
