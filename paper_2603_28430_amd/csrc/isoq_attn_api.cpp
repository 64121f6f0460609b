// C ABI of attention over the paged cache and of the cache's pages (declared in
// include/isoquant.h): argument validation, the choice of kernel and splits,
// and launches.
#include <hip/hip_runtime_api.h>

#include <algorithm>
#include <cmath>
#include <new>

#include "isoq_attn.h"
#include "isoq_handles.h"
#include "isoq_pages.h"

namespace {

using namespace isoq;

// Rows (query heads of a sequence's tokens): a grid of one workgroup of 256 a row
// stays below 2^32 threads.
constexpr int kAttnMaxRows = 1 << 23;
// Positions: a workgroup's first one past them still fits 31 bits.
constexpr int64_t kAttnMaxPos = 0x7FFFFFFF - 1023;

// Kept positions: a workgroup's first one past them still fits 31 bits.
constexpr int kCompactMaxKeep = 0x7FFFFFFF - 8191;

// The handle's tables, made by the first call that asks for them; null if there is
// no memory.  (Host threads that come first together all make them, the same ones,
// and keep one.)
const AttnTables *tables_of(const isoq_params *p)
{
    const AttnTables *held = p->attn_tables.load(std::memory_order_acquire);
    if (held)
        return held;
    AttnTables *t = new (std::nothrow) AttnTables;
    if (!t)
        return nullptr;
    build_value_digits(p->bits, p->levels, 2, t->vd[0]);
    build_value_digits(p->bits, p->levels, 3, t->vd[1]);
    const double left = build_half_levels(p->bits, p->levels, t->half);
    t->key_rest = left <= kLeftNone ? kRestNone : left <= kLeftBytes ? kRestBytes : kRestHalves;
    if (p->attn_tables.compare_exchange_strong(held, t, std::memory_order_acq_rel))
        return t;
    delete t;
    return held;
}

// How a call is cut up; from its sizes alone, so that isoq_kv_attn_workspace
// answers for the call that follows.
struct AttnPlan {
    const AttnTables *kt, *vt;   // null where the width-generic kernel runs, or without memory
    AttnKernel kern;   // fn null: the width-generic kernel, a row per workgroup
    int64_t max_pos;   // positions a sequence has at most
    int64_t groups;    // workgroups per sequence and split
    int width, slots;  // rotated coordinates per row (a multiple of the slot), slots
    int chunk, n_splits;
    bool join;         // the kernel leaves parts for a join
};

AttnPlan attn_plan(const isoq_params *pk, const isoq_params *pv, int dtype, int n_seqs, int max_q_len, int n_q_heads,
                   int n_kv_heads, int64_t max_pos, bool few_rows = false, int max_splits = kAttnMaxSplits)
{
    AttnPlan p{};
    const int sw = pk->variant == VAR_BLOCK8 ? 8 : 4;
    p.slots = (padded_width(pk->variant, pk->d) + sw - 1) / sw;
    p.width = p.slots * sw;
    p.max_pos = max_pos;
    const bool f16 = dtype == ISOQ_F16;
    const int64_t rows = (int64_t)(n_q_heads / n_kv_heads) * max_q_len;
    p.groups = (int64_t)n_q_heads * max_q_len;
    if (pk->attn_by_tables && pv->attn_by_tables) {
        p.kt = tables_of(pk);
        p.vt = tables_of(pv);
        if (!p.kt || !p.vt)
            return p;
        const int r = (int)std::min<int64_t>(rows, 1 << 20);
        p.kern = pk->bits == 2   ? attn_m_kernel_b2(pk->d, r, f16)
                 : pk->bits == 3 ? attn_m_kernel_b3(pk->d, r, f16)
                                 : attn_m_kernel_b4(pk->d, r, f16);
        // Many rows: where decoding a tile for 128 rows at once pays for what
        // fewer leave idle (us by digits / in fp16.  16 x 8 heads, 4,096
        // positions, d = 128, 3 bits: 24 rows 64 / 74, 32 78 / 69, 64 141 / 81, 128
        // 256 / 103.  2 x 8 heads, 8,192: 24 28 / 33, 32 30 / 33, 48 39 / 38, 128 70
        // / 55.  4 x 4 heads, 8,192, d = 64, 4 bits: 32 25 / 24, 64 40 / 28.)
        if (f16 && rows >= 32 && !few_rows) {
            const AttnKernel many = attn_c_kernel_for(pk->d, pk->bits, p.kt->key_rest, r);
            if (many.fn)
                p.kern = many;
        }
        p.groups = n_kv_heads * ((rows + p.kern.rows - 1) / p.kern.rows);
    }
    // Splits: as many as give so many workgroups, of which a compute unit holds two
    // to four at once (two above d = 128 and in fp16): more than one round of them
    // evens out sequences of different lengths, and is not wanted where there is
    // one sequence, or in fp16, which cuts them evenly (attn_chunk).  None up to
    // 768 positions, three tiles a wave (one sequence, 8 x 4 heads, on the GPU / with
    // the host's calls: 700 positions 9.8 / 12.1 us with one split, 8.7 / 15.6 with
    // three; 1,000: 12.4 / 12.4, 8.7 / 14.5).
    // (us at 512 / 768 / 1,024 / 1,536 / 2,048 wanted: 1 x 8 x 8 heads, 131,071
    // positions 49 / 51 / 49 / 53 / 53; 8 x 32 x 32,768 231 / 210 / 203 / 202 / 208; 16
    // ragged x 8 x 4 of up to 8,192 45 / 44 / 40 / 42 / 42, with 5 tokens of up to
    // 4,096 51 / 50 / 44 / 40 / 41; 4 x 8 x 2, 8,190, d = 256 25 / 25 / 27 / 27 / 27.
    // In fp16 at 384 / 512 / 640 / 768 / 1,024: two ragged chunks of up to 512 tokens and
    // 8,192 positions 231 / 220 / 254 / 253 / 234, two equal ones 308 / 303 / 334 / 337
    // / 318; 16 of up to 16 tokens and 4,096 positions 89 / 78 / 77 / 89 / 84; 8 prompts
    // of 1,024 tokens 103 / 102 / 112 / 111 / 110: one round of workgroups, which is
    // three a compute unit at d = 64 (512 / 768 / 1,024: two ragged chunks 138 / 126 / 137,
    // two equal ones 219 / 190 / 206, the 16 57 / 48 / 56).)
    // (Those figures are of 128 rows a workgroup.  Of 256, one a compute unit: one round is 256.)
    // (Workgroups of 8 rows at 768 / 1,280 / 1,536: 8 x 8 heads, 4,096 positions 18 / 22 /
    // 22; 16 ragged x 8 x 4 of 5 tokens, mean of three 47 / 38 / 38; 4 ragged x 2 x 16, up
    // to 20,000 20 / 23 / 23; 8 ragged x 4 x 4 of 5 tokens, fp32 23 / 23 / 27.  Of 12: 8 x
    // 8 heads, 4,096 23 / 28 / 28, 8 ragged x 8, up to 8,000 34 / 35 / 35.)
    // (Of 4, ragged, at 1,024 / 1,280 / 1,536: 16 x 16 heads, up to 1,500 17.5 / 17.5 / 19.1,
    // 32 x 8 x 4 18.3 / 18.1 / 20.2, fp32 18.2 / 18.3 / 20.1; 32 x 8 x 4 of up to 8,000 54 / 52 / 48,
    // 8 x 32, up to 32,768 160 / 159 / 140.)
    const int64_t want = p.kern.parts                                          ? (p.kern.rows > 128 ? 256 : pk->d <= 64 ? 768 : 512)
                         : n_seqs == 1 || pk->d > 128 || p.kern.rows == 12     ? 768
                         : p.kern.rows == 8 || p.max_pos <= 2048               ? 1280
                                                                               : 1536;
    const int64_t blocks = p.groups * n_seqs;
    // In fp16 as many splits as fit one round, down to 128 positions each up to 768 and
    // 256 past that: a tile takes a workgroup 4 us however few there are (32 tokens of
    // one sequence, 8 x 4 heads, 700 positions: one split 51 us, of 256 30, of 128 25; 300
    // tokens of 4 sequences: one 67, two 82; four of 64 tokens and 4,000, d = 64, 2 bits: of
    // 512 39, of 384 50).
    const bool short_many = p.kern.parts && p.max_pos <= 768;
    const int64_t unit = short_many ? 128 : 256;
    int64_t splits = p.kern.parts        ? std::max<int64_t>(1, want / blocks)
                     : p.max_pos <= 768 ? 1
                                         : (want + blocks - 1) / blocks;
    splits = std::min<int64_t>(splits, max_splits);
    int64_t chunk = (p.max_pos + splits - 1) / splits;
    chunk = std::max<int64_t>(unit, (chunk + unit - 1) / unit * unit);
    p.chunk = (int)std::min<int64_t>(chunk, 0x7FFFFF00);
    p.n_splits = (int)std::max<int64_t>(1, (p.max_pos + p.chunk - 1) / p.chunk);
    p.join = p.n_splits > 1 || (p.kern.parts && pk->variant == VAR_BLOCK8);
    return p;
}

size_t plan_bytes(const AttnPlan &p, int64_t n_tokens, int n_q_heads)
{
    return !p.join ? 0 : sizeof(float) * (size_t)n_tokens * n_q_heads * p.n_splits * (p.width + 2);
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

// The planes of a cache that a page call was given: records and norms of K, of
// V (or null), signs and gamma of a sketch (or null).
struct Planes {
    uint8_t *base[kCachePlanes];
    int64_t row[kCachePlanes];   // bytes of a position of a head
    bool record[kCachePlanes];   // stored in the cache's pieces
    int n;
};

isoq_status cache_planes(const isoq_params *pk, const isoq_sketch *sk, uint8_t *k_idx, float *k_rho, uint8_t *v_idx,
                         float *v_rho, uint8_t *k_signs, float *k_gamma, Planes &p)
{
    if (!k_idx || !k_rho || !v_idx != !v_rho)
        return ISOQ_E_NULL;
    if (sk ? !k_signs || !k_gamma : k_signs || k_gamma)
        return ISOQ_E_NULL;
    if (sk && (sk->variant != pk->variant || sk->d != pk->d || sk->device != pk->device))
        return ISOQ_E_INVALID;
    if (!aligned(k_idx, 16) || !aligned(v_idx, 16) || !aligned(k_rho, 4) || !aligned(v_rho, 4) ||
        !aligned(k_signs, 4) || !aligned(k_gamma, 4))
        return ISOQ_E_ALIGN;
    p.n = 0;
    auto add = [&](void *base, int64_t row, bool record) {
        if (base) {
            p.base[p.n] = static_cast<uint8_t *>(base);
            p.row[p.n] = row;
            p.record[p.n++] = record;
        }
    };
    const int64_t rec = (int64_t)record_bytes(pk->variant, pk->d, pk->bits);
    add(k_idx, rec, true);
    add(v_idx, rec, true);
    add(k_rho, 4, false);
    add(v_rho, 4, false);
    add(k_signs, sk ? sk->m / 8 : 0, false);
    add(k_gamma, 4, false);
    return ISOQ_OK;
}

// One attention call's arguments; the prefix's where n_prefixes > 0.
struct AttnCall {
    const isoq_params *pk, *pv;
    int dtype;
    const void *q;
    const int32_t *q_start;
    int64_t n_tokens;
    int max_q_len, n_seqs, n_q_heads, n_kv_heads;
    const uint8_t *k_idx;
    const float *k_rho;
    const uint8_t *v_idx;
    const float *v_rho;
    int64_t n_blocks;
    int block_size;
    const int32_t *block_table;
    int max_blocks;
    const int32_t *seq_lens;
    int64_t max_len;
    const int32_t *prefix_table;
    int max_prefix_blocks;
    const int32_t *prefix_lens;
    int64_t max_prefix_len;
    const int32_t *prefix_start;
    int n_prefixes;
    int64_t max_prefix_tokens;
    float scale;
    void *out;
    float *lse;
    void *workspace;
    size_t workspace_bytes;
    void *stream;
    bool full;
};

// A launch's arguments, but for the parts' places.
AttnArgs attn_args(const AttnCall &c, const AttnPlan &plan, float scale2)
{
    const isoq_params *pk = c.pk, *pv = c.pv;
    AttnArgs a{};
    a.q = c.q;
    a.out = c.out;
    a.lse = c.lse;
    a.k_idx = c.k_idx;
    a.v_idx = c.v_idx;
    a.k_rho = c.k_rho;
    a.v_rho = c.v_rho;
    a.block_table = c.block_table;
    a.seq_lens = c.seq_lens;
    a.q_start = c.q_start;
    a.k_params = pk->dparams;
    a.v_params = pv->dparams;
    a.n_blocks = c.n_blocks;
    a.set_stride = (int64_t)slots_per_set(pk->variant, pk->d) * params_per_slot(pk->variant);
    a.n_tokens = (int32_t)c.n_tokens;
    a.max_q_len = c.max_q_len;
    a.n_q_heads = c.n_q_heads;
    a.n_kv_heads = c.n_kv_heads;
    a.group = c.n_q_heads / c.n_kv_heads;
    a.block_size = c.block_size;
    a.max_blocks = c.max_blocks;
    a.cap = c.n_blocks == 0 ? 0 : (int32_t)std::min<int64_t>(c.max_len, (int64_t)c.max_blocks * c.block_size);
    a.k_sets = pk->n_sets;
    a.v_sets = pv->n_sets;
    a.variant = pk->variant;
    a.q_f16 = c.dtype == ISOQ_F16;
    a.chunk = plan.chunk;
    a.n_splits = a.part_splits = plan.n_splits;
    a.n_seqs = c.n_seqs;
    a.even = plan.kern.parts;
    a.full = c.full;
    a.scale = scale2;
    a.div_block = make_fastdiv((uint32_t)c.block_size);
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
    if (plan.kern.fn) {
        a.v_dig = plan.vt->vd[c.dtype == ISOQ_F16 ? 0 : 1];
        a.k_half = plan.kt->half;
        a.v_half = plan.vt->half;
    }
    return a;
}

// The kernel of a plan (pre: of launches with n_pre > 0), or null where there is none.
const void *attn_fn(const AttnCall &c, const AttnPlan &plan, bool pre)
{
    return !plan.kern.fn ? attn_generic_kernel_for(c.pk->variant, c.pk->bits, pre)
           : pre         ? plan.kern.fn_pre
                         : plan.kern.fn;
}

isoq_status launch_attn(const AttnCall &c, const AttnPlan &plan, const void *fn, AttnArgs &a, int n_seqs)
{
    void *args[] = {&a};
    const size_t lds = plan.kern.fn ? plan.kern.lds : attn_generic_lds(plan.slots, c.pk->variant);
    if (lds > 65536) {
        const hipError_t e = hipFuncSetAttribute(fn, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (e != hipSuccess)
            return hip_fail(e, "hipFuncSetAttribute");
    }
    // (splits last: those that some sequences do not reach come after those that all do)
    return launch_lds(fn, dim3((unsigned)plan.groups, (unsigned)n_seqs, (unsigned)plan.n_splits),
                      plan.kern.fn ? plan.kern.threads : 256, args, lds, c.stream);
}

// The plans of a call: of the sequences' own positions, and of the prefixes'.
struct AttnPlans {
    AttnPlan own, pre;
    bool prefix;   // in launches and parts of their own
    bool fold;     // which the kernel of the own positions, in one split, adds itself
    bool ahead;    // before each sequence's own positions, in one launch (own is the plan of both)
    size_t bytes;
    bool ok;   // (false: no memory for a handle's tables)
};

// What a tile of keys (64 positions) of a key head costs a workgroup of `rows` rows of a
// kernel, four rows by digits being 1: a third more for each further four by digits
// (isoq_attn_m_pick.h), 10 for 128 rows in fp16, by its waves that have rows.
double tile_cost(const AttnPlan &p, int64_t rows)
{
    if (!p.kern.fn)
        return (double)rows;
    if (p.kern.parts)
        return 2.5 * (double)std::max<int64_t>(4, (rows + 31) / 32);
    return (double)((rows + p.kern.rows - 1) / p.kern.rows) * (0.6 + 0.1 * p.kern.rows);
}

// Whether the prefix is read anew by every sequence, in front of its own positions, in
// one launch: `ahead` of both together, against `pre` of the prefix for all its rows
// together (a launch and parts of its own).  Where the products differ by less than the
// further launch and the parts take, 4 us by digits and 13 and more in fp16, a unit of
// work being 22 us in a million, in fp16 half of that.  (us, shared / ahead, behind one
// prefix, 100 positions of their own: 8 x 4 heads, d = 128, fp16: 16 sequences of 2,000 28
// / 20, of 8,000 31 / 38, 32 of 2,000 30 / 24, of 4,000 31 / 36, 64 of 1,000 37 / 25, of
// 2,000 38 / 36, of 4,000 40 / 57; 5 tokens each: 8 of 2,000 31 / 23, 16 40 / 35, 64 56 / 93, 4 of
// 8,000 33 / 39; fp32: 4 of 2,000 15 / 13, 32 23 / 24, 64 35 / 38, of 4,000 52 / 59; 8 x 1, d =
// 64: 16 of 2,000 13 / 15, 64 23 / 28; 4 x 5, d = 96, fp32, 5 tokens: 16 of 2,000 31 / 30, of 4,000
// 41 / 44, of 8,000 57 / 72; d = 256, 2 x 4: 16 of 8,000 31 / 27, 64 of 4,000 37 / 39.)
bool prefix_ahead(const AttnCall &c, const AttnPlan &ahead, const AttnPlan &pre)
{
    const int64_t group = c.n_q_heads / c.n_kv_heads;
    const double tiles = (double)pre.max_pos * c.n_kv_heads;
    const double anew = tiles * c.n_seqs * tile_cost(ahead, group * c.max_q_len);
    const double once = tiles * c.n_prefixes * tile_cost(pre, group * c.max_prefix_tokens);
    const double rows = (double)c.n_tokens * c.n_q_heads;
    return ahead.max_pos <= kAttnMaxPos && anew <= (pre.kern.parts ? 0.5 * once + 0.6e6 + 130.0 * rows : once + 0.2e6);
}

// Whether a call has a prefix to attend to.
bool has_prefix(const AttnCall &c)
{
    return c.n_prefixes > 0 && c.max_prefix_blocks > 0 && c.max_prefix_len > 0 && c.max_prefix_tokens > 0;
}

AttnPlans attn_plans(const AttnCall &c)
{
    AttnPlans p{};
    const isoq_params *pk = c.pk;
    p.prefix = has_prefix(c);
    const bool tables = pk->attn_by_tables && c.pv->attn_by_tables;
    const int most = p.prefix ? kAttnMaxSplits / 2 : kAttnMaxSplits;   // (a row's join takes both kinds)
    const int64_t own = std::min<int64_t>(c.max_len, (int64_t)c.max_blocks * c.block_size);
    if (p.prefix) {
        const int64_t shared = std::min<int64_t>(c.max_prefix_len, (int64_t)c.max_prefix_blocks * c.block_size);
        p.pre = attn_plan(pk, c.pv, c.dtype, c.n_prefixes, (int)c.max_prefix_tokens, c.n_q_heads, c.n_kv_heads, shared,
                          false, most);
        p.own = attn_plan(pk, c.pv, c.dtype, c.n_seqs, c.max_q_len, c.n_q_heads, c.n_kv_heads, own + shared, true);
        p.ok = !tables || (p.own.kern.fn && p.pre.kern.fn);
        if (prefix_ahead(c, p.own, p.pre)) {
            p.prefix = false;
            p.ahead = true;
            p.bytes = plan_bytes(p.own, c.n_tokens, c.n_q_heads);
            return p;
        }
    }
    auto plan_own = [&](int splits) {
        return attn_plan(pk, c.pv, c.dtype, c.n_seqs, c.max_q_len, c.n_q_heads, c.n_kv_heads, own, false, splits);
    };
    p.own = plan_own(most);
    // (One split, whose kernel needs no join, where that leaves two workgroups a compute unit and
    // few tiles a wave: us in splits / in one, behind 8,000 positions, 64 x 8 x 4 heads, up to
    // 1,000 positions of their own 70 / 61, 2,000 78 / 75, 4,000 98 / 102, fp32, 1,500 114 /
    // 112; 32 x 8 x 4 behind 30,000, 1,000 74 / 72, 2,000 79 / 82; 16 x 4 x 8, 1,000 97 / 113.)
    if (p.prefix && p.own.kern.fn && !p.own.kern.parts && p.own.n_splits > 1 && own <= 2048 &&
        p.own.groups * c.n_seqs >= 512)
        p.own = plan_own(1);
    p.ok = !tables || (p.own.kern.fn && (!p.prefix || p.pre.kern.fn));
    if (!p.prefix) {
        p.bytes = plan_bytes(p.own, c.n_tokens, c.n_q_heads);
        return p;
    }
    p.fold = p.own.kern.fn_pre && !p.own.join;   // (the kernel of many rows has no form that adds them)
    p.bytes = sizeof(float) * (size_t)c.n_tokens * c.n_q_heads * ((p.fold ? 0 : p.own.n_splits) + p.pre.n_splits) *
              (p.own.width + 2);
    return p;
}

isoq_status check_prefix(const AttnCall &c)
{
    if (c.n_prefixes < 0 || c.max_prefix_blocks < 0 || c.max_prefix_len < 0 || c.max_prefix_tokens < 0 ||
        (c.n_prefixes > 0 && c.max_prefix_tokens == 0 && c.n_tokens > 0) || (!c.prefix_start && c.n_prefixes > 1))
        return ISOQ_E_INVALID;
    if (c.n_prefixes > 65535 || (int64_t)c.max_prefix_blocks * c.block_size > kAttnMaxPos ||
        (has_prefix(c) && c.max_prefix_tokens > kAttnMaxRows / c.n_q_heads))
        return ISOQ_E_UNSUPPORTED;
    return ISOQ_OK;
}

isoq_status attn_call(AttnCall c)
{
    isoq_status st = check_attn(c.pk, c.pv, c.dtype, c.n_tokens, c.max_q_len, c.n_seqs, c.n_q_heads, c.n_kv_heads,
                                c.block_size, c.max_blocks, c.max_len);
    c.max_prefix_tokens = std::min(c.max_prefix_tokens, c.n_tokens);
    if (st == ISOQ_OK)
        st = check_prefix(c);
    if (st != ISOQ_OK)
        return st;
    const float scale2 = (float)((double)c.scale * 1.4426950408889634);   // (logits in units of ln 2)
    if (c.n_blocks < 0 || !std::isfinite(scale2) || (!c.q_start && (c.n_tokens != c.n_seqs || c.max_q_len != 1)))
        return ISOQ_E_INVALID;
    if (c.n_tokens == 0 || c.n_seqs == 0)
        return ISOQ_OK;
    const bool no_keys = c.n_blocks == 0 || c.max_blocks == 0 || c.max_len == 0;
    AttnPlans plans = attn_plans(c);
    if (c.n_blocks == 0 && (plans.prefix || plans.ahead)) {   // (less than isoq_kv_attn_prefix_workspace says)
        plans.prefix = plans.ahead = plans.fold = false;
        plans.bytes = plan_bytes(plans.own, c.n_tokens, c.n_q_heads);
    }
    if (!c.q || !c.out || !c.seq_lens || (!no_keys && !c.block_table) ||
        ((plans.prefix || plans.ahead) && (!c.prefix_table || !c.prefix_lens)) ||
        ((!no_keys || plans.prefix || plans.ahead) && (!c.k_idx || !c.k_rho || !c.v_idx || !c.v_rho)))
        return ISOQ_E_NULL;
    if (!aligned(c.q, 16) || !aligned(c.out, 16) || !aligned(c.k_idx, 16) || !aligned(c.v_idx, 16) || !aligned(c.k_rho, 4) ||
        !aligned(c.v_rho, 4) || !aligned(c.block_table, 4) || !aligned(c.seq_lens, 4) || !aligned(c.q_start, 4) ||
        !aligned(c.lse, 4) || !aligned(c.workspace, 16) || !aligned(c.prefix_table, 4) || !aligned(c.prefix_lens, 4) ||
        !aligned(c.prefix_start, 4))
        return ISOQ_E_ALIGN;
    if (!plans.ok)
        return ISOQ_E_NOMEM;
    const size_t need = plans.bytes;
    if (need > 0 && !c.workspace)
        return ISOQ_E_NULL;
    if (need > c.workspace_bytes)
        return ISOQ_E_INVALID;
    st = check_device(c.pk);
    if (st != ISOQ_OK)
        return st;

    const AttnPlan &plan = plans.own;
    const void *fn = attn_fn(c, plan, plans.ahead || plans.fold), *fn_prefix = plans.prefix ? attn_fn(c, plans.pre, false) : fn;
    if (!fn || !fn_prefix)   // (before anything is launched)
        return ISOQ_E_UNSUPPORTED;
    AttnArgs a = attn_args(c, plan, scale2);
    if (no_keys)
        a.cap = 0;
    if (plans.ahead || plans.fold) {
        a.n_pre = c.n_prefixes;
        a.pre_blocks = c.max_prefix_blocks;
        a.pre_tokens = (int32_t)c.max_prefix_tokens;
        a.pre_cap = (int32_t)std::min<int64_t>(c.max_prefix_len, (int64_t)c.max_prefix_blocks * c.block_size);
        a.pre_start = c.prefix_start;
        a.pre_table = c.prefix_table;
        a.pre_lens = c.prefix_lens;
    }
    if (plans.prefix)
        a.part_splits = (plans.fold ? 0 : a.n_splits) + plans.pre.n_splits;
    if (plans.fold) {
        a.fold = plans.pre.n_splits;
        a.pre_chunk = plans.pre.chunk;
        a.pre_even = plans.pre.kern.parts;
    }
    if (need) {
        a.part = static_cast<float *>(c.workspace);
        a.part_ml = a.part + (size_t)c.n_tokens * c.n_q_heads * a.part_splits * plan.width;
    }
    AttnPrefix p{};
    if (plans.prefix) {
        AttnCall shared = c;   // every token of a prefix's sequences, all its positions
        shared.block_table = c.prefix_table;
        shared.max_blocks = c.max_prefix_blocks;
        shared.max_len = c.max_prefix_len;
        shared.seq_lens = c.prefix_lens;
        shared.max_q_len = (int)c.max_prefix_tokens;
        shared.full = true;
        AttnArgs b = attn_args(shared, plans.pre, scale2);
        b.shared = c.prefix_start;
        b.n_all = c.n_seqs;
        b.part = a.part;
        b.part_ml = a.part_ml;
        b.part_splits = a.part_splits;
        b.part_first = plans.fold ? 0 : a.n_splits;
        p = AttnPrefix{c.prefix_start, c.prefix_lens, c.n_prefixes, c.n_seqs, (int32_t)c.max_prefix_tokens,
                       b.cap, b.chunk, b.n_splits, b.even};
        st = launch_attn(shared, plans.pre, fn_prefix, b, c.n_prefixes);
        if (st != ISOQ_OK)
            return st;
    }
    st = launch_attn(c, plan, fn, a, c.n_seqs);
    if (st != ISOQ_OK || need == 0 || plans.fold)
        return st;
    const bool few = a.part_splits <= kAttnJoinFew;
    const unsigned rows = (unsigned)c.n_q_heads * (unsigned)c.max_q_len, per = few ? 256 / plan.slots : 1;
    void *args[] = {&a, &p};
    const void *join = plans.prefix ? attn_prefix_join_kernel_for(c.pk->variant, few)
                                    : attn_join_kernel_for(c.pk->variant, few, plans.ahead);
    return launch_lds(join, dim3((rows + per - 1) / per, (unsigned)c.n_seqs), 256, args, 0, c.stream);
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
    return plan_bytes(attn_plan(pk, pv, dtype, n_seqs, max_q_len, n_q_heads, n_kv_heads,
                                std::min<int64_t>(max_len, (int64_t)max_blocks_per_seq * block_size)),
                      n_tokens, n_q_heads);
}

isoq_status isoq_kv_attn(const isoq_params *pk, const isoq_params *pv, int dtype, const void *q,
                         const int32_t *q_start, int64_t n_tokens, int max_q_len, int n_seqs, int n_q_heads,
                         int n_kv_heads, const uint8_t *k_idx, const float *k_rho, const uint8_t *v_idx,
                         const float *v_rho, int64_t n_blocks, int block_size, const int32_t *block_table,
                         int max_blocks_per_seq, const int32_t *seq_lens, int64_t max_len, float scale, void *out,
                         float *lse, void *workspace, size_t workspace_bytes, void *stream)
{
    return attn_call(AttnCall{pk, pv, dtype, q, q_start, n_tokens, max_q_len, n_seqs, n_q_heads, n_kv_heads, k_idx, k_rho,
                              v_idx, v_rho, n_blocks, block_size, block_table, max_blocks_per_seq, seq_lens, max_len,
                              nullptr, 0, nullptr, 0, nullptr, 0, 0, scale, out, lse, workspace, workspace_bytes, stream,
                              false});
}

isoq_status isoq_kv_attn_cross(const isoq_params *pk, const isoq_params *pv, int dtype, const void *q,
                               const int32_t *q_start, int64_t n_tokens, int max_q_len, int n_seqs, int n_q_heads,
                               int n_kv_heads, const uint8_t *k_idx, const float *k_rho, const uint8_t *v_idx,
                               const float *v_rho, int64_t n_blocks, int block_size, const int32_t *block_table,
                               int max_blocks_per_seq, const int32_t *seq_lens, int64_t max_len, float scale, void *out,
                               float *lse, void *workspace, size_t workspace_bytes, void *stream)
{
    return attn_call(AttnCall{pk, pv, dtype, q, q_start, n_tokens, max_q_len, n_seqs, n_q_heads, n_kv_heads, k_idx, k_rho,
                              v_idx, v_rho, n_blocks, block_size, block_table, max_blocks_per_seq, seq_lens, max_len,
                              nullptr, 0, nullptr, 0, nullptr, 0, 0, scale, out, lse, workspace, workspace_bytes, stream,
                              true});
}

size_t isoq_kv_attn_prefix_workspace(const isoq_params *pk, const isoq_params *pv, int dtype, int64_t n_tokens,
                                     int max_q_len, int n_seqs, int n_q_heads, int n_kv_heads, int block_size,
                                     int max_blocks_per_seq, int64_t max_len, int n_prefixes, int64_t max_prefix_tokens,
                                     int max_prefix_blocks, int64_t max_prefix_len)
{
    AttnCall c{};
    c.pk = pk;
    c.pv = pv;
    c.dtype = dtype;
    c.n_tokens = n_tokens;
    c.max_q_len = max_q_len;
    c.n_seqs = n_seqs;
    c.n_q_heads = n_q_heads;
    c.n_kv_heads = n_kv_heads;
    c.block_size = block_size;
    c.max_blocks = max_blocks_per_seq;
    c.max_len = max_len;
    c.max_prefix_blocks = max_prefix_blocks;
    c.max_prefix_len = max_prefix_len;
    c.n_prefixes = n_prefixes;
    c.max_prefix_tokens = std::min(max_prefix_tokens, n_tokens);
    static const int32_t some = 0;
    c.prefix_start = &some;   // (only whether there is one matters here)
    if (check_attn(pk, pv, dtype, n_tokens, max_q_len, n_seqs, n_q_heads, n_kv_heads, block_size, max_blocks_per_seq,
                   max_len) != ISOQ_OK ||
        check_prefix(c) != ISOQ_OK || n_tokens == 0 || n_seqs == 0)
        return 0;
    return attn_plans(c).bytes;
}

isoq_status isoq_kv_attn_prefix(const isoq_params *pk, const isoq_params *pv, int dtype, const void *q,
                                const int32_t *q_start, int64_t n_tokens, int max_q_len, int n_seqs, int n_q_heads,
                                int n_kv_heads, const uint8_t *k_idx, const float *k_rho, const uint8_t *v_idx,
                                const float *v_rho, int64_t n_blocks, int block_size, const int32_t *block_table,
                                int max_blocks_per_seq, const int32_t *seq_lens, int64_t max_len,
                                const int32_t *prefix_table, int max_prefix_blocks, const int32_t *prefix_lens,
                                int64_t max_prefix_len, const int32_t *prefix_start, int n_prefixes,
                                int64_t max_prefix_tokens, float scale, void *out, float *lse, void *workspace,
                                size_t workspace_bytes, void *stream)
{
    return attn_call(AttnCall{pk, pv, dtype, q, q_start, n_tokens, max_q_len, n_seqs, n_q_heads, n_kv_heads, k_idx, k_rho,
                              v_idx, v_rho, n_blocks, block_size, block_table, max_blocks_per_seq, seq_lens, max_len,
                              prefix_table, max_prefix_blocks, prefix_lens, max_prefix_len, prefix_start, n_prefixes,
                              max_prefix_tokens, scale, out, lse, workspace, workspace_bytes, stream, false});
}

isoq_status isoq_kv_copy_blocks(const isoq_params *pk, const isoq_sketch *sk, const int32_t *block_pairs,
                                int64_t n_pairs, int n_heads, uint8_t *k_idx, float *k_rho, uint8_t *v_idx,
                                float *v_rho, uint8_t *k_signs, float *k_gamma, int64_t n_blocks, int block_size,
                                void *stream)
{
    if (!pk)
        return ISOQ_E_NULL;
    if (n_pairs < 0 || n_heads < 1 || block_size < 1 || n_blocks < 0)
        return ISOQ_E_INVALID;
    if (n_pairs > 0xFFFFFF || n_blocks > 0x7FFFFFFF / block_size)
        return ISOQ_E_UNSUPPORTED;
    if (n_pairs == 0 || n_blocks == 0)
        return ISOQ_OK;
    if (!block_pairs)
        return ISOQ_E_NULL;
    Planes pl;
    isoq_status st = cache_planes(pk, sk, k_idx, k_rho, v_idx, v_rho, k_signs, k_gamma, pl);
    if (st != ISOQ_OK)
        return st;
    if (!aligned(block_pairs, 4))
        return ISOQ_E_ALIGN;
    CopyArgs a{};
    int64_t most = 0;
    for (int c = 0; c < pl.n; c++) {
        a.plane[c] = pl.base[c];
        a.stride[c] = pl.row[c] * n_heads * block_size;
        a.unit[c] = a.stride[c] >= 16 ? 16 : a.stride[c] % 4 == 0 ? 4 : 1;
        const int64_t units = (a.stride[c] + a.unit[c] - 1) / a.unit[c];
        if (units > 1 << 27)
            return ISOQ_E_UNSUPPORTED;
        a.units[c] = (int32_t)units;
        a.div_units[c] = make_fastdiv((uint32_t)units);
        most = std::max(most, (n_pairs * units + kCopyUnits - 1) / kCopyUnits);
    }
    const int64_t deep = (most + kCopyGrid - 1) / kCopyGrid;
    if (deep > 65535)
        return ISOQ_E_UNSUPPORTED;
    a.n_pairs = n_pairs;
    a.pairs = block_pairs;
    a.n_blocks = n_blocks;
    st = check_device(pk);
    if (st != ISOQ_OK)
        return st;
    void *args[] = {&a};
    return launch_lds(copy_blocks_kernel(), dim3((unsigned)std::min<int64_t>(most, kCopyGrid), (unsigned)pl.n, (unsigned)deep),
                      256, args, 0, stream);
}

isoq_status isoq_kv_compact(const isoq_params *pk, const isoq_sketch *sk, const int32_t *keep, int keep_heads,
                            int max_keep, const int32_t *n_keep, int n_seqs, const int32_t *block_table,
                            int max_blocks_per_seq, int n_heads, uint8_t *k_idx, float *k_rho, uint8_t *v_idx,
                            float *v_rho, uint8_t *k_signs, float *k_gamma, int64_t n_blocks, int block_size,
                            void *stream)
{
    if (!pk)
        return ISOQ_E_NULL;
    if (n_seqs < 0 || max_keep < 0 || n_heads < 1 || block_size < 1 || n_blocks < 0 || max_blocks_per_seq < 0 ||
        (keep_heads != 1 && keep_heads != n_heads))
        return ISOQ_E_INVALID;
    if (n_seqs > 65535 || n_heads > 0x3FFFFF || (int64_t)max_blocks_per_seq * block_size > 0x7FFFFFFF ||
        n_blocks > 0x7FFFFFFF / block_size || max_keep > kCompactMaxKeep)
        return ISOQ_E_UNSUPPORTED;
    if (n_seqs == 0 || max_keep == 0 || n_blocks == 0 || max_blocks_per_seq == 0)
        return ISOQ_OK;
    if (!keep || !n_keep || !block_table)
        return ISOQ_E_NULL;
    Planes pl;
    isoq_status st = cache_planes(pk, sk, k_idx, k_rho, v_idx, v_rho, k_signs, k_gamma, pl);
    if (st != ISOQ_OK)
        return st;
    if (!aligned(keep, 4) || !aligned(n_keep, 4) || !aligned(block_table, 4))
        return ISOQ_E_ALIGN;
    CompactArgs a{};
    const bool full = (int64_t)n_heads * n_seqs >= 64;   // (CompactArgs)
    bool whole = false;
    int n = 0;
    auto columns = [&](int c, int64_t offset, int width, int64_t count, int64_t step, int64_t pos_stride) {
        a.base[n] = pl.base[c] + offset;
        a.head_stride[n] = pl.row[c] * block_size;
        a.block_stride[n] = a.head_stride[n] * n_heads;
        a.width[n] = width;
        a.step[n] = step;
        a.pos_stride[n] = (int32_t)pos_stride;
        a.first[n + 1] = a.first[n] + (int32_t)count;
        n++;
    };
    for (int c = 0; c < pl.n; c++) {
        const int64_t row = pl.row[c], piece = pl.record[c] ? cache_piece(row) : row;
        if (piece != row) {   // pieces of 16 or 8 bytes, those of one position block_size of them apart
            columns(c, 0, (int)piece, row / piece, piece * block_size, piece);
            continue;
        }
        whole = whole || (row != 4 && row != 8 && row != 16);
        int64_t at = 0;
        for (int width = full ? 64 : 16; at < row; width /= 2) {
            if (full && width < 64)
                width = (int)(row - at);
            if (const int64_t count = (row - at) / width) {
                columns(c, at, width, count, width, row);
                at += count * width;
            }
        }
    }
    const int chains = a.first[n];
    for (; n < kCompactColumns; n++)
        a.first[n + 1] = chains;
    a.keep = keep;
    a.n_keep = n_keep;
    a.block_table = block_table;
    a.n_blocks = n_blocks;
    a.keep_heads = keep_heads;
    a.max_keep = max_keep;
    a.max_blocks = max_blocks_per_seq;
    a.block_size = block_size;
    a.div_block = make_fastdiv((uint32_t)block_size);
    st = check_device(pk);
    if (st != ISOQ_OK)
        return st;
    void *args[] = {&a};
    return launch_lds(compact_kernel(whole), dim3((unsigned)n_heads, (unsigned)n_seqs, (unsigned)chains),
                      kCompactThreads, args, 0, stream);
}

}  // extern "C"
