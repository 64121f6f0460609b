// C ABI of attention over the paged cache and of the cache's pages (declared in
// include/isoquant.h): argument validation, the choice of kernel and splits,
// and launches.
#include <hip/hip_runtime_api.h>

#include <algorithm>
#include <cmath>

#include "isoq_attn.h"
#include "isoq_handles.h"

namespace {

using namespace isoq;

// Rows (query heads of a sequence's tokens): a grid of one workgroup of 256 a row
// stays below 2^32 threads.
constexpr int kAttnMaxRows = 1 << 23;
// Positions: a workgroup's first one past them still fits 31 bits.
constexpr int64_t kAttnMaxPos = 0x7FFFFFFF - 1023;

// How a call is cut up; from its sizes alone, so that isoq_kv_attn_workspace
// answers for the call that follows.
struct AttnPlan {
    AttnKernel kern;   // fn null: the width-generic kernel, a row per workgroup
    int64_t max_pos;   // positions a sequence has at most
    int64_t groups;    // workgroups per sequence and split
    int width, slots;  // rotated coordinates per row (a multiple of the slot), slots
    int chunk, n_splits;
};

AttnPlan attn_plan(const isoq_params *pk, const isoq_params *pv, int dtype, int n_seqs, int max_q_len, int n_q_heads,
                   int n_kv_heads, int block_size, int max_blocks_per_seq, int64_t max_len)
{
    AttnPlan p{};
    const int sw = pk->variant == VAR_BLOCK8 ? 8 : 4;
    p.slots = (padded_width(pk->variant, pk->d) + sw - 1) / sw;
    p.width = p.slots * sw;
    p.max_pos = std::min<int64_t>(max_len, (int64_t)max_blocks_per_seq * block_size);
    const bool f16 = dtype == ISOQ_F16;
    const int64_t rows = (int64_t)(n_q_heads / n_kv_heads) * max_q_len;
    p.groups = (int64_t)n_q_heads * max_q_len;
    // (wide codebooks: levels that one set of digits does not hold)
    if (decode_d(pk->d) && !pk->wide && !pv->wide) {
        const int r = (int)std::min<int64_t>(rows, 1 << 20);
        p.kern = pk->bits == 2   ? attn_m_kernel_b2(pk->d, r, f16)
                 : pk->bits == 3 ? attn_m_kernel_b3(pk->d, r, f16)
                                 : attn_m_kernel_b4(pk->d, r, f16);
        p.groups = n_kv_heads * ((rows + p.kern.rows - 1) / p.kern.rows);
    }
    const int64_t want = 2048, blocks = p.groups * n_seqs;
    const int64_t splits = std::min<int64_t>((want + blocks - 1) / blocks, kAttnMaxSplits);
    int64_t chunk = (p.max_pos + splits - 1) / splits;
    chunk = std::max<int64_t>(256, (chunk + 255) / 256 * 256);
    p.chunk = (int)std::min<int64_t>(chunk, 0x7FFFFF00);
    p.n_splits = (int)std::max<int64_t>(1, (p.max_pos + p.chunk - 1) / p.chunk);
    return p;
}

size_t plan_bytes(const AttnPlan &p, int64_t n_tokens, int n_q_heads)
{
    return p.n_splits == 1 ? 0 : sizeof(float) * (size_t)n_tokens * n_q_heads * p.n_splits * (p.width + 2);
}

// Argument values of isoq_kv_attn that do not need its pointers.
isoq_status check_attn(const isoq_params *pk, const isoq_params *pv, int dtype, int64_t n_tokens, int max_q_len,
                       int n_seqs, int n_q_heads, int n_kv_heads, int block_size, int max_blocks_per_seq,
                       int64_t max_len)
{
    if (!pk || !pv)
        return ISOQ_E_NULL;
    if (dtype != ISOQ_F32 && dtype != ISOQ_F16)
        return ISOQ_E_INVALID;
    if (pv->variant != pk->variant || pv->d != pk->d || pv->bits != pk->bits || pv->device != pk->device)
        return ISOQ_E_INVALID;
    if (n_tokens < 0 || n_seqs < 0 || max_q_len < 1 || n_q_heads < 1 || n_kv_heads < 1 ||
        n_q_heads % n_kv_heads != 0 || block_size < 1 || max_blocks_per_seq < 0 || max_len < 0)
        return ISOQ_E_INVALID;
    if ((pk->n_sets != 1 && pk->n_sets != n_kv_heads) || (pv->n_sets != 1 && pv->n_sets != n_kv_heads))
        return ISOQ_E_INVALID;
    if (n_seqs > 65535 || (int64_t)max_blocks_per_seq * block_size > kAttnMaxPos ||
        n_tokens > 0x7FFFFFFF / n_q_heads || max_q_len > kAttnMaxRows / n_q_heads)
        return ISOQ_E_UNSUPPORTED;
    return ISOQ_OK;
}

}  // namespace

extern "C" {

size_t isoq_kv_attn_workspace(const isoq_params *pk, const isoq_params *pv, int dtype, int64_t n_tokens, int max_q_len,
                              int n_seqs, int n_q_heads, int n_kv_heads, int block_size, int max_blocks_per_seq,
                              int64_t max_len)
{
    if (check_attn(pk, pv, dtype, n_tokens, max_q_len, n_seqs, n_q_heads, n_kv_heads, block_size, max_blocks_per_seq,
                   max_len) != ISOQ_OK ||
        n_tokens == 0 || n_seqs == 0)
        return 0;
    return plan_bytes(attn_plan(pk, pv, dtype, n_seqs, max_q_len, n_q_heads, n_kv_heads, block_size, max_blocks_per_seq, max_len),
                      n_tokens, n_q_heads);
}

isoq_status isoq_kv_attn(const isoq_params *pk, const isoq_params *pv, int dtype, const void *q,
                         const int32_t *q_start, int64_t n_tokens, int max_q_len, int n_seqs, int n_q_heads,
                         int n_kv_heads, const uint8_t *k_idx, const float *k_rho, const uint8_t *v_idx,
                         const float *v_rho, int64_t n_blocks, int block_size, const int32_t *block_table,
                         int max_blocks_per_seq, const int32_t *seq_lens, int64_t max_len, float scale, void *out,
                         float *lse, void *workspace, size_t workspace_bytes, void *stream)
{
    isoq_status st = check_attn(pk, pv, dtype, n_tokens, max_q_len, n_seqs, n_q_heads, n_kv_heads, block_size,
                                max_blocks_per_seq, max_len);
    if (st != ISOQ_OK)
        return st;
    if (n_blocks < 0 || !std::isfinite(scale) || (!q_start && (n_tokens != n_seqs || max_q_len != 1)))
        return ISOQ_E_INVALID;
    if (n_tokens == 0 || n_seqs == 0)
        return ISOQ_OK;
    const bool no_keys = n_blocks == 0 || max_blocks_per_seq == 0 || max_len == 0;
    if (!q || !out || !seq_lens || (!no_keys && (!k_idx || !k_rho || !v_idx || !v_rho || !block_table)))
        return ISOQ_E_NULL;
    if (!aligned(q, 16) || !aligned(out, 16) || !aligned(k_idx, 16) || !aligned(v_idx, 16) || !aligned(k_rho, 4) ||
        !aligned(v_rho, 4) || !aligned(block_table, 4) || !aligned(seq_lens, 4) || !aligned(q_start, 4) ||
        !aligned(lse, 4) || !aligned(workspace, 16))
        return ISOQ_E_ALIGN;
    const AttnPlan plan =
        attn_plan(pk, pv, dtype, n_seqs, max_q_len, n_q_heads, n_kv_heads, block_size, max_blocks_per_seq, max_len);
    const size_t need = plan_bytes(plan, n_tokens, n_q_heads);
    if (need > 0 && !workspace)
        return ISOQ_E_NULL;
    if (need > workspace_bytes)
        return ISOQ_E_INVALID;
    st = check_device(pk);
    if (st != ISOQ_OK)
        return st;

    AttnArgs a{};
    a.q = q;
    a.out = out;
    a.lse = lse;
    a.part = static_cast<float *>(workspace);
    a.part_ml = need ? a.part + (size_t)n_tokens * n_q_heads * plan.n_splits * plan.width : nullptr;
    a.k_idx = k_idx;
    a.v_idx = v_idx;
    a.k_rho = k_rho;
    a.v_rho = v_rho;
    a.block_table = block_table;
    a.seq_lens = seq_lens;
    a.q_start = q_start;
    a.k_params = pk->dparams;
    a.v_params = pv->dparams;
    a.n_blocks = n_blocks;
    a.set_stride = (int64_t)slots_per_set(pk->variant, pk->d) * params_per_slot(pk->variant);
    a.n_tokens = (int32_t)n_tokens;
    a.max_q_len = max_q_len;
    a.n_q_heads = n_q_heads;
    a.n_kv_heads = n_kv_heads;
    a.group = n_q_heads / n_kv_heads;
    a.block_size = block_size;
    a.max_blocks = max_blocks_per_seq;
    a.cap = no_keys ? 0 : (int32_t)plan.max_pos;
    a.k_sets = pk->n_sets;
    a.v_sets = pv->n_sets;
    a.variant = pk->variant;
    a.q_f16 = dtype == ISOQ_F16;
    a.chunk = plan.chunk;
    a.n_splits = plan.n_splits;
    a.scale = (float)((double)scale * 1.4426950408889634);
    a.div_block = make_fastdiv((uint32_t)block_size);
    a.d = pk->d;
    a.width = plan.width;
    a.slots = plan.slots;
    a.rec = (int32_t)record_bytes(pk->variant, pk->d, pk->bits);
    a.rec_lp = a.rec % 16 == 0 ? 4 : a.rec % 8 == 0 ? 3 : -1;   // cache_piece
    for (int k = 0; k < (1 << pk->bits); k++) {
        a.k_lev[k] = pk->levels[k];
        a.v_lev[k] = pv->levels[k];
    }
    a.k_dig = pk->lv;
    a.v_dig = pv->vd[dtype == ISOQ_F16 ? 0 : 1];
    void *args[] = {&a};
    const void *fn = plan.kern.fn ? plan.kern.fn : attn_generic_kernel_for(pk->variant, pk->bits);
    const size_t lds = plan.kern.fn ? plan.kern.lds : attn_generic_lds(plan.slots, pk->variant);
    if (!fn)
        return ISOQ_E_UNSUPPORTED;
    if (lds > 65536) {
        const hipError_t e = hipFuncSetAttribute(fn, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (e != hipSuccess)
            return hip_fail(e, "hipFuncSetAttribute");
    }
    st = launch_lds(fn, dim3((unsigned)plan.groups, (unsigned)plan.n_splits, (unsigned)n_seqs), 256, args, lds, stream);
    if (st != ISOQ_OK || plan.n_splits == 1)
        return st;
    const unsigned rows = (unsigned)n_q_heads * (unsigned)max_q_len;
    return launch_lds(attn_join_kernel_for(pk->variant),
                      dim3((rows + kAttnJoinRows - 1) / kAttnJoinRows, (unsigned)n_seqs), 64 * kAttnJoinRows, args, 0,
                      stream);
}

}  // extern "C"
