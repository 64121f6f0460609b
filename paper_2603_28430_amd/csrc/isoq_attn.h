// Attention over a paged cache of quantized keys and values: what its kernels
// (isoq_attn_m.h, isoq_attn_generic.hip, isoq_attn_join.hip) and the host code
// (isoq_attn_api.cpp) share.
//
// A row is a new token's query head.  With k_hat = rho T_k^{-1} c[idx] and
// v_hat = rho T_v^{-1} c[idx] for the cached rows and T orthogonal (Prop. 1),
//     s_t = scale <q, k_hat_t> = rho_kt <scale T_k q, c[idx_kt]>
//     o   = sum_t p_t v_hat_t / l = T_v^{-1} (sum_t p_t rho_vt c[idx_vt]) / l,
//     p_t = exp(s_t - m),  l = sum_t p_t,  lse = m + ln l:
// the query is rotated once, the sum of values is rotated back once, and no
// cached row is ever decompressed.  (Logits and m are kept in units of ln 2.)
// A long cache is cut into splits of `chunk` positions (attn_chunk); each leaves m, l and its
// sum of values, which attn_join_kernel joins.  With one split a workgroup
// finishes its rows by itself.
#pragma once

#include "isoq_attn_tables.h"
#include "isoq_internal.h"

namespace isoq {

struct AttnArgs {
    const void *q;               // [n_tokens][n_q_heads][d]
    void *out;                   // the same
    float *lse;                  // [n_tokens][n_q_heads], or null
    float *part;                 // splits (or null: rows are finished by the kernel): sums of values [row][n_splits][width], row = token n_q_heads + head
    float *part_ml;              // splits: m, l [row][n_splits][2]
    const uint8_t *k_idx, *v_idx;
    const float *k_rho, *v_rho;
    const int32_t *block_table;  // [n_seqs][max_blocks]
    const int32_t *seq_lens;     // [n_seqs]
    const int32_t *q_start;      // [n_seqs + 1], or null: one token each
    const float *k_params, *v_params;
    int64_t n_blocks;
    int64_t set_stride;          // parameter floats per set
    int32_t n_tokens, max_q_len, n_q_heads, n_kv_heads, group;
    int32_t block_size, max_blocks;
    int32_t cap;                 // positions a sequence has at most (0: no cache)
    int32_t k_sets, v_sets, variant, q_f16;
    int32_t chunk, n_splits;     // positions per split (at most, if even: attn_chunk)
    int32_t even;
    float scale;                 // times log2(e)
    FastDiv div_block;
    int32_t d, width, slots;     // coordinates per row, padded width, its rotation slots (8 coordinates for 8-D, else 4)
    int32_t rec, rec_lp;         // record bytes, the cache layout's pieces (1 << rec_lp bytes, or whole: < 0)
    float k_lev[16], v_lev[16];  // codebooks (width-generic kernel)
    LevelDigits k_dig;           // the same as digits (matrix-core kernel)
    ValueDigits v_dig;
    HalfLevels k_half, v_half;   // and in fp16 (kernel of many rows)
};

constexpr int kAttnMaxSplits = 256;

// Width-generic kernel: one row per workgroup, grid (query head + n_q_heads
// token, sequence, split).
const void *attn_generic_kernel_for(int variant, int bits);
size_t attn_generic_lds(int slots, int variant);
// Matrix-core kernel (isoq_attn_m.h; widths of the tuned decoding kernels) for
// `rows` rows per sequence and key head: its entry, its dynamic LDS, and the
// rows that a workgroup takes.  Grid (key head + n_kv_heads row tile,
// sequence, split).
struct AttnKernel {
    const void *fn;
    size_t lds;
    int rows;
    bool parts;   // the kernel of many rows
};
AttnKernel attn_m_kernel_b2(int d, int rows, bool f16);
AttnKernel attn_m_kernel_b3(int d, int rows, bool f16);
AttnKernel attn_m_kernel_b4(int d, int rows, bool f16);
// Kernel of many rows (isoq_attn_c.h; fp16 queries, widths up to 128), with what
// fp16 leaves of the keys' levels in the form `rest` (kRestNone ..); or {}.
AttnKernel attn_c_kernel_for(int d, int bits, int rest);
// Join of the splits, 256 threads: up to kAttnJoinFew splits (few) grid (rows of
// a sequence / (256 / slots), sequence), more (row, sequence); a row being query
// head + n_q_heads token.
constexpr int kAttnJoinFew = 8;
const void *attn_join_kernel_for(int variant, bool few);

}  // namespace isoq
