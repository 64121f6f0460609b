// C ABI of what a serving step takes before its append (declared in
// include/isoquant.h): blocks and slots of its tokens, and norms with rotary
// positions of its queries and keys.
#include <hip/hip_runtime_api.h>

#include <algorithm>
#include <cmath>
#include <new>
#include <vector>

#include "isoq_handles.h"
#include "isoq_step.h"

namespace {

using namespace isoq;

// Tokens up to which the one workgroup of the plan writes slots and positions too (us by a
// second launch / by itself: 512 single tokens 7.9 / 5.5, 2,048 11.7 / 9.7, 4,096 14.1 / 14.2, 8,192
// 33 / 47; a prompt of 2,048 7.4 / 6.0, of 4,096 7.7 / 6.9, two of 4,096 8.1 / 9.1).
constexpr int64_t kPlanTokensHere = 4096;

// Waves up to which a token's rows are shared out (us with one wave a token / up to 2,048 / 4,096 /
// 8,192 / 16,384; d = 128, fp16, 40 heads: 32 tokens 6.7 / 4.1 / 4.1 / 4.1 / 4.1, 512 7.4 / 6.0 /
// 5.7 / 5.7 / 5.7, 2,048 12.9 / 13.1 / 12.0 / 15.2 / 15.3, 4,096 17.9 / 18.0 / 18.1 / 20.1 / 25.9;
// fp32, 72 heads: 1,000 20.9 / 16.5 / 15.7 / 16.8 / 19.2).
constexpr int64_t kRopeWaves = 4096;

// Waves of a launch: a grid has fewer than 2^32 threads.
constexpr int64_t kRopeLaunch = (1 << 26) - 4;

// `waves` of them a token, four a workgroup; in launches of as many tokens as one takes, in
// multiples of 16, so that rows of any width stay at multiples of 16 bytes.
isoq_status launch_rope(const void *fn, const RopeArgs &all, int64_t n_tokens, int64_t waves, size_t es, void *stream)
{
    const int64_t most = kRopeLaunch / waves / 16 * 16;
    for (int64_t t = 0; t < n_tokens; t += most) {
        RopeArgs a = all;
        a.n_tokens = (int32_t)std::min(most, n_tokens - t);
        a.positions += t;
        for (int k = 0; k < 2; k++)
            if (a.heads[k] > 0) {
                a.x[k] = static_cast<const char *>(a.x[k]) + t * a.stride[k] * (int64_t)es;
                a.out[k] = static_cast<char *>(a.out[k]) + t * a.heads[k] * a.d * (int64_t)es;
            }
        void *args[] = {&a};
        const isoq_status st = launch_lds(fn, dim3((unsigned)((a.n_tokens * waves + 3) / 4)), 256, args, 0, stream);
        if (st != ISOQ_OK)
            return st;
    }
    return ISOQ_OK;
}

constexpr double kTwoPi = 6.283185307179586476925;

}  // namespace

struct isoq_rope {
    int d, rot_dim, layout;
    int device;
    float amplitude;
    uint64_t *turns;   // device, [rot_dim / 2] turns a position in units of 2^-64
};

extern "C" {

isoq_status isoq_kv_plan(const int32_t *lens, const int32_t *new_lens, int n_seqs, int32_t *block_table,
                         int max_blocks_per_seq, int block_size, int32_t *free_blocks, int64_t max_free,
                         const int32_t *n_free, int32_t *seq_lens, int32_t *q_start, int64_t *slot_mapping,
                         int32_t *positions, int64_t n_tokens, int32_t *n_free_out, void *stream)
{
    if (n_seqs < 0 || max_blocks_per_seq < 0 || block_size < 1 || max_free < 0 || n_tokens < 0)
        return ISOQ_E_INVALID;
    if (n_seqs > 65535 || (int64_t)max_blocks_per_seq * block_size > 0x7FFFFFFF - block_size || max_free > 0x7FFFFFFF ||
        n_tokens > 0x7FFFFFFF)
        return ISOQ_E_UNSUPPORTED;
    if (!n_free || !q_start || !n_free_out || (n_seqs > 0 && (!lens || !new_lens || !seq_lens)) ||
        (n_seqs > 0 && max_blocks_per_seq > 0 && !block_table) || (max_free > 0 && !free_blocks) ||
        (n_tokens > 0 && (!slot_mapping || !positions)))
        return ISOQ_E_NULL;
    if (!aligned(lens, 4) || !aligned(new_lens, 4) || !aligned(block_table, 4) || !aligned(free_blocks, 4) ||
        !aligned(n_free, 4) || !aligned(seq_lens, 4) || !aligned(q_start, 4) || !aligned(slot_mapping, 8) ||
        !aligned(positions, 4) || !aligned(n_free_out, 4))
        return ISOQ_E_ALIGN;
    if (seq_lens == new_lens && n_seqs > 0)
        return ISOQ_E_INVALID;
    PlanArgs a{};
    a.lens = lens;
    a.new_lens = new_lens;
    a.block_table = block_table;
    a.free_blocks = free_blocks;
    a.n_free = n_free;
    a.seq_lens = seq_lens;
    a.q_start = q_start;
    a.slots = slot_mapping;
    a.positions = positions;
    a.n_free_out = n_free_out;
    a.max_free = max_free;
    a.n_seqs = n_seqs;
    a.max_blocks = max_blocks_per_seq;
    a.block_size = block_size;
    a.n_tokens = (int32_t)n_tokens;
    a.cap = max_blocks_per_seq * block_size;
    a.tokens_too = n_tokens <= kPlanTokensHere;
    a.div_block = make_fastdiv((uint32_t)block_size);
    void *args[] = {&a};
    const isoq_status st = launch_lds(plan_kernel(n_seqs), dim3(1), kPlanThreads, args, 0, stream);
    if (st != ISOQ_OK || a.tokens_too)
        return st;
    return launch_lds(plan_tokens_kernel(), dim3((unsigned)((n_tokens + 255) / 256)), 256, args, 0, stream);
}

isoq_status isoq_rope_freqs(int rot_dim, double base, double factor, double original, double low, double high,
                            double *out)
{
    if (!out)
        return ISOQ_E_NULL;
    if (rot_dim < 2 || rot_dim % 2 != 0 || !(base > 0) || !std::isfinite(base) || !(factor > 0) || !std::isfinite(factor) ||
        !(original >= 0) || !std::isfinite(original) || !(low >= 0) || !(high >= low) || !std::isfinite(high))
        return ISOQ_E_INVALID;
    for (int i = 0; i < rot_dim / 2; i++) {
        const double f = std::pow(base, -2.0 * i / rot_dim);
        const double turns = f * original / kTwoPi;
        // how much of the pair's own frequency stays
        const double keep = turns <= low ? 0.0 : turns >= high ? 1.0 : (turns - low) / (high - low);
        out[i] = f * (keep + (1.0 - keep) / factor);
    }
    return ISOQ_OK;
}

isoq_status isoq_rope_init(isoq_rope **out, int d, int rot_dim, int layout, const double *freqs, double amplitude)
{
    if (!out)
        return ISOQ_E_NULL;
    *out = nullptr;
    if (d < 1 || rot_dim < 0 || rot_dim > d || rot_dim % 2 != 0 || (layout != ISOQ_ROPE_PAIRS && layout != ISOQ_ROPE_HALVES) ||
        !std::isfinite((float)amplitude))
        return ISOQ_E_INVALID;
    if (d > 1024)
        return ISOQ_E_UNSUPPORTED;
    if (rot_dim > 0 && !freqs)
        return ISOQ_E_NULL;
    std::vector<uint64_t> turns;
    isoq_rope *r = new (std::nothrow) isoq_rope{};
    if (!r)
        return ISOQ_E_NOMEM;
    try {
        turns.resize((size_t)std::max(1, rot_dim / 2));
    } catch (const std::bad_alloc &) {
        delete r;
        return ISOQ_E_NOMEM;
    }
    for (int i = 0; i < rot_dim / 2; i++) {
        if (!std::isfinite(freqs[i])) {
            delete r;
            return ISOQ_E_INVALID;
        }
        // (the 64 bits of long double hold what the division leaves)
        const long double t = (long double)freqs[i] / 6.283185307179586476925286766559L;
        const long double part = t - floorl(t);   // in [0, 1)
        const long double units = part * 18446744073709551616.0L;
        turns[i] = units >= 18446744073709551615.0L ? ~0ull : (uint64_t)units;
    }
    r->d = d;
    r->rot_dim = rot_dim;
    r->layout = layout;
    r->amplitude = (float)amplitude;
    hipError_t e = hipGetDevice(&r->device);
    if (e == hipSuccess)
        e = hipMalloc(reinterpret_cast<void **>(&r->turns), turns.size() * sizeof(uint64_t));
    if (e == hipSuccess)
        e = hipMemcpy(r->turns, turns.data(), turns.size() * sizeof(uint64_t), hipMemcpyHostToDevice);
    if (e != hipSuccess) {
        if (r->turns)
            (void)hipFree(r->turns);
        delete r;
        return hip_fail(e, "isoq_rope_init", e == hipErrorOutOfMemory ? ISOQ_E_NOMEM : ISOQ_E_HIP);
    }
    *out = r;
    return ISOQ_OK;
}

isoq_status isoq_rope_destroy(isoq_rope *r)
{
    if (!r)
        return ISOQ_OK;
    int prev = -1;
    (void)hipGetDevice(&prev);
    if (prev != r->device)
        (void)hipSetDevice(r->device);
    const isoq_status st = hipFree(r->turns) == hipSuccess ? ISOQ_OK : ISOQ_E_HIP;
    if (prev >= 0 && prev != r->device)
        (void)hipSetDevice(prev);
    delete r;
    return st;
}

isoq_status isoq_qk_norm_rope(const isoq_rope *r, int dtype, const void *q, int64_t q_stride, int n_q_heads,
                              const void *k, int64_t k_stride, int n_kv_heads, const int32_t *positions,
                              int64_t n_tokens, const float *q_weight, const float *k_weight, float eps, void *q_out,
                              void *k_out, void *stream)
{
    if (!r)
        return ISOQ_E_NULL;
    if (dtype != ISOQ_F32 && dtype != ISOQ_F16)
        return ISOQ_E_INVALID;
    if (n_tokens < 0 || n_q_heads < 0 || n_kv_heads < 0 || !(eps >= 0) || !std::isfinite(eps))
        return ISOQ_E_INVALID;
    if (n_q_heads > 65535 || n_kv_heads > 65535)
        return ISOQ_E_UNSUPPORTED;
    const int64_t heads = (int64_t)n_q_heads + n_kv_heads;
    if (n_tokens == 0 || heads == 0)
        return ISOQ_OK;
    if (n_tokens > 0x7FFFFFFF / heads)
        return ISOQ_E_UNSUPPORTED;
    if (!positions || (n_q_heads > 0 && (!q || !q_out)) || (n_kv_heads > 0 && (!k || !k_out)))
        return ISOQ_E_NULL;
    if ((n_q_heads > 0 && q_stride < (int64_t)n_q_heads * r->d) || (n_kv_heads > 0 && k_stride < (int64_t)n_kv_heads * r->d))
        return ISOQ_E_INVALID;
    const size_t es = dtype == ISOQ_F16 ? 2 : 4;
    if (!aligned(q, es) || !aligned(k, es) || !aligned(q_out, 16) || !aligned(k_out, 16) || !aligned(positions, 4) ||
        !aligned(q_weight, 4) || !aligned(k_weight, 4))
        return ISOQ_E_ALIGN;
    int dev = -1;
    const hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess)
        return hip_fail(e, "hipGetDevice");
    if (dev != r->device)
        return ISOQ_E_DEVICE;
    RopeArgs a{};
    a.x[0] = q;
    a.x[1] = k;
    a.out[0] = q_out;
    a.out[1] = k_out;
    a.weight[0] = q_weight;
    a.weight[1] = k_weight;
    a.stride[0] = q_stride;
    a.stride[1] = k_stride;
    a.heads[0] = n_q_heads;
    a.heads[1] = n_kv_heads;
    a.positions = positions;
    a.turns = r->turns;
    a.d = r->d;
    a.half = r->rot_dim / 2;
    a.eps = eps;
    a.amplitude = r->amplitude;
    const bool f16 = dtype == ISOQ_F16, halves = r->layout == ISOQ_ROPE_HALVES;
    // the largest chunks that all rows are made of
    for (const int chunk : {f16 ? 8 : 4, 2, 1}) {
        const int cr = 2 * a.half / chunk, cz = (r->d - 2 * a.half) / chunk, pairs = (cr + 1) / 2 + (cz + 1) / 2;
        const size_t bytes = chunk * es;
        auto placed = [&](const void *x, int64_t stride, int n) {
            return n == 0 || (aligned(x, bytes) && (n_tokens == 1 || stride % chunk == 0));
        };
        if (r->d % chunk != 0 || (halves ? a.half : 2 * a.half) % chunk != 0 || (!halves && chunk % 2 != 0) || pairs > 64 ||
            !placed(q, q_stride, n_q_heads) || !placed(k, k_stride, n_kv_heads))
            continue;
        int lanes = 4;
        while (lanes < pairs)
            lanes *= 2;
        const int64_t rows = 64 / lanes, most = (n_q_heads + rows - 1) / rows + (n_kv_heads + rows - 1) / rows;
        a.parts = (int32_t)std::max<int64_t>(1, std::min<int64_t>(most, kRopeWaves / n_tokens));
        return launch_rope(rope_tile_kernel_for(f16, halves, chunk, lanes), a, n_tokens, a.parts, es, stream);
    }
    int steps = 0;
    while ((64 << steps) < r->d)
        steps++;
    return launch_rope(rope_kernel(f16, halves, steps), a, n_tokens, heads, es, stream);
}

}  // extern "C"
