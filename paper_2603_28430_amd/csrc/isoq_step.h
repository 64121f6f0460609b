// What a serving step takes before its append: blocks and slots of its tokens
// (isoq_plan.hip), norms and rotary positions of its queries and keys
// (isoq_rope.hip).  Arguments and entries; the host code is isoq_step_api.cpp.
#pragma once

#include "isoq_internal.h"

namespace isoq {

struct PlanArgs {
    const int32_t *lens, *new_lens;   // [n_seqs] positions before, after
    int32_t *block_table;             // [n_seqs][max_blocks]
    int32_t *free_blocks;             // [max_free], of which the first *n_free count
    const int32_t *n_free;
    int32_t *seq_lens;                // [n_seqs] (may be lens)
    int32_t *q_start;                 // [n_seqs + 1]
    int64_t *slots;                   // [n_tokens]
    int32_t *positions;               // [n_tokens]
    int32_t *n_free_out;              // (may be n_free)
    int64_t max_free;
    int32_t n_seqs, max_blocks, block_size;
    int32_t n_tokens;
    int32_t cap;                      // max_blocks * block_size
    int32_t tokens_too;               // the one workgroup writes slots and positions as well
    FastDiv div_block;
};
// One workgroup of kPlanThreads; then, where it does not do that itself, slots and
// positions: 256 threads, a token each.
constexpr int kPlanThreads = 1024;
const void *plan_kernel(int n_seqs);
const void *plan_tokens_kernel();

struct RopeArgs {
    const void *x[2];              // queries, keys: token t's heads at x + t stride
    void *out[2];                  // [n_tokens][heads][d]
    const float *weight[2];        // [d], or null: no norm
    int64_t stride[2];             // elements between tokens
    int32_t heads[2];
    const int32_t *positions;      // [n_tokens]
    const uint64_t *turns;         // [half] turns a position, in units of 2^-64
    int32_t n_tokens, d, half;     // half: pairs that are rotated
    float eps, amplitude;
    int32_t parts;                 // waves that share a token's rows (rope_tile_kernel)
};
// Rows by chunks of `chunk` coordinates (16 bytes, 2 or, in halves, 1), which divide the width and
// the rotated part (in halves each half), lanes (4 .. 64, a power of two) a row. Grid
// of four waves, `parts` a token.
const void *rope_tile_kernel_for(bool f16, bool halves, int chunk, int lanes);
// A row a wave, rows token by token (queries, then keys), four waves a workgroup;
// for widths up to 64 << log2_steps (log2_steps <= 4).
const void *rope_kernel(bool f16, bool halves, int log2_steps);

}  // namespace isoq
