// Block tables and slots of a step's tokens, from the sequences' lengths before
// and after it (isoq_kv_plan).  With have and need the blocks of a sequence
// before and after,
//     released  blocks need .. have - 1 of a sequence that shrinks go on top of
//               the free list, sequence after sequence: `there` blocks are free;
//     taken     block i of a sequence that grows is
//               free[there - 1 - (what the sequences before it take) - i],
//               unless the sum up to and with it exceeds `there`;
//     tokens    token i of a sequence has position lens + i.
// Three prefix sums over the sequences (new tokens, blocks taken, blocks
// released), so the result does not depend on the order in which anything runs.
// Sums saturate at 2^31 - 1, past every list and every token.
//
// One workgroup of 1,024 threads: the sums need every sequence, and a second launch costs
// what the whole takes.  What bounds it is its chain of dependent accesses (lengths;
// released blocks; the free list, then the tables; tables, then slots), about 1 us each,
// and for many tokens one compute unit's stores: 64 single tokens take 4.2 us, a mixed
// step of 513 sequences 7.7, 8 prompts of 32,768 tokens (16,384 blocks, 3.3 MB) 7.1, each of the
// latter with 4 more for the slots, which a launch over all units writes
// (plan_slots_kernel).  Moves of more than two blocks go to a list in LDS that the waves work
// off, four at a time (a thread that moved its own: the mixed step 47 us on the GPU, the
// prompts 230; one at a time: 20 and 16).
#include <hip/hip_runtime.h>

#include "isoq_device.h"
#include "isoq_step.h"

namespace isoq {
namespace {

__device__ __forceinline__ int add_sat(int a, int b) { return __builtin_elementwise_add_sat(a, b); }

struct PlanSeq {
    int old, want, have, need;
    __device__ __forceinline__ int fresh() const { return max(0, want - old); }
    __device__ __forceinline__ int grow() const { return max(0, need - have); }
    __device__ __forceinline__ int drop() const { return max(0, have - need); }
};

__device__ __forceinline__ int plan_blocks(const PlanArgs &a, int len)
{
    return (int)fast_div((uint32_t)len + (uint32_t)a.block_size - 1u, a.div_block);
}

__device__ __forceinline__ PlanSeq plan_seq(const PlanArgs &a, int s)
{
    PlanSeq q;
    q.old = min(max(a.lens[s], 0), a.cap);
    q.want = min(max(a.new_lens[s], 0), a.cap);
    q.have = plan_blocks(a, q.old);
    q.need = plan_blocks(a, q.want);
    return q;
}

// Slot and position of token t of sequence s, which are there.
__device__ __forceinline__ void plan_place(const PlanArgs &a, int t, int s, int pos, bool fine)
{
    int64_t slot = -1;
    const uint32_t j = fast_div((uint32_t)pos, a.div_block);
    if (fine && pos >= 0 && j < (uint32_t)a.max_blocks) {
        const int blk = a.block_table[(int64_t)s * a.max_blocks + j];
        if (blk >= 0)
            slot = (int64_t)blk * a.block_size + (pos - (int)(j * (uint32_t)a.block_size));
    }
    a.slots[t] = slot;
    a.positions[t] = pos;
}

// The first sequence that ends past token t; start[s] .. start[s + 1] - 1 are those of s.
__device__ __forceinline__ int plan_find(const int *start, int n, int t)
{
    int lo = 0;
    for (int hi = n; lo < hi;) {
        const int mid = (lo + hi) >> 1;
        if (start[mid + 1] > t)
            hi = mid;
        else
            lo = mid + 1;
    }
    return lo;
}

// Slot and position of token t, once the sequences' lengths, first tokens and
// blocks are there.
__device__ __forceinline__ void plan_token(const PlanArgs &a, int t)
{
    const int s = plan_find(a.q_start, a.n_seqs, t);
    if (s >= a.n_seqs) {
        a.slots[t] = -1;
        a.positions[t] = 0;
        return;
    }
    const int first = a.q_start[s], len = a.seq_lens[s];
    const bool fine = len == min(max(a.new_lens[s], 0), a.cap);   // not refused
    plan_place(a, t, s, (fine ? len - (a.q_start[s + 1] - first) : len) + (t - first), fine);
}

// Inclusive sum over the wave's lanes.
__device__ __forceinline__ int wave_scan(int v)
{
#define ISOQ_SCAN_STEP(ctrl, rows) \
    v = add_sat(v, __builtin_amdgcn_update_dpp(0, v, ctrl, rows, 0xF, false))
    ISOQ_SCAN_STEP(0x111, 0xF);   // row_shr 1, 2, 4, 8: within 16 lanes
    ISOQ_SCAN_STEP(0x112, 0xF);
    ISOQ_SCAN_STEP(0x114, 0xF);
    ISOQ_SCAN_STEP(0x118, 0xF);
    ISOQ_SCAN_STEP(0x142, 0xA);   // row_bcast 15: lane 15's to 16 .. 31, lane 47's to 48 .. 63
    ISOQ_SCAN_STEP(0x143, 0xC);   // row_bcast 31: lane 31's to 32 .. 63
#undef ISOQ_SCAN_STEP
    return v;
}

// A sequence's blocks to move, a list of which the waves work off: free[from ..] to
// its row downwards (taken), or its row to free[from ..] (released).
struct PlanMove {
    int seq, at, from, count;   // count < 0: released
};

// N > 0: up to N consecutive sequences a thread, held in registers, and the token
// search in LDS; 0: any number, read again in every pass.  (2,000 single tokens 44 us read
// again, 9.7 in registers.)
template <int N>
__device__ __forceinline__ void plan_body(const PlanArgs &a)
{
    constexpr int WAVES = kPlanThreads / 64;
    // blocks that a thread moves by itself; more go to the list
    constexpr int FEW = 2;
    __shared__ int wave_sum[3][WAVES], most[WAVES], listed[4];
    __shared__ PlanMove list[kPlanThreads];
    __shared__ int start[N ? N * kPlanThreads + 1 : 1];
    __shared__ int begin[N ? N * kPlanThreads : 1];   // position of its first new token, or ~ that where it is refused
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int per = N ? N : (a.n_seqs + kPlanThreads - 1) / kPlanThreads;
    const int s0 = min(tid * per, a.n_seqs), s1 = min(s0 + per, a.n_seqs);

    if (tid < 4)
        listed[tid] = 0;
    const int n_free = *a.n_free;
    PlanSeq mine[N ? N : 1];
    if constexpr (N > 0) {
#pragma unroll
        for (int k = 0; k < N; k++)
            mine[k] = s0 + k < s1 ? plan_seq(a, s0 + k) : PlanSeq{0, 0, 0, 0};
    }
    auto seq = [&](int k) {
        if constexpr (N > 0)
            return mine[k];
        else
            return plan_seq(a, s0 + k);
    };
    int sum[3] = {0, 0, 0}, before[3], total[3];
#pragma unroll N > 0 ? N : 1
    for (int k = 0; k < per; k++) {
        if (s0 + k >= s1)
            break;
        const PlanSeq q = seq(k);
        sum[0] = add_sat(sum[0], q.fresh());
        sum[1] = add_sat(sum[1], q.grow());
        sum[2] = add_sat(sum[2], q.drop());
    }
#pragma unroll
    for (int k = 0; k < 3; k++) {
        const int x = wave_scan(sum[k]);
        const int y = __builtin_amdgcn_update_dpp(0, x, 0x138, 0xF, 0xF, false);   // wave_shr 1
        before[k] = lane == 0 ? 0 : y;
        if (lane == 63)
            wave_sum[k][w] = x;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 3; k++) {
        total[k] = 0;
#pragma unroll
        for (int x = 0; x < WAVES; x++) {
            if (x == w)
                before[k] = add_sat(before[k], total[k]);
            total[k] = add_sat(total[k], wave_sum[k][x]);
        }
    }
    const int max_free = (int)a.max_free;
    const int held = min(max(n_free, 0), max_free);
    const int there = min(add_sat(held, total[2]), max_free);

    auto blocks = [&](const PlanMove &m) { return m.count < 0 ? min(-m.count, max_free - m.from) : m.count; };   // (released: from <= max_free)
    auto source = [&](const PlanMove &m, int j) {
        return m.count < 0 ? a.block_table + (int64_t)m.seq * a.max_blocks + m.at + j : a.free_blocks + (m.from - j);
    };
    auto target = [&](const PlanMove &m, int j) {
        return m.count < 0 ? a.free_blocks + (m.from + j) : a.block_table + (int64_t)m.seq * a.max_blocks + m.at + j;
    };
    auto move = [&](const PlanMove &m, int first, int step) {
        const int n = blocks(m);
        for (int64_t j = first; j < n; j += 4 * step) {   // (four loads, then four stores: the lists do not overlap)
            int v[4];
#pragma unroll
            for (int u = 0; u < 4; u++)
                if (j + u * step < n)
                    v[u] = *source(m, (int)j + u * step);
#pragma unroll
            for (int u = 0; u < 4; u++)
                if (j + u * step < n)
                    *target(m, (int)j + u * step) = v[u];
        }
    };
    // few blocks at once; more by the lists: from the front those for a wave, from the back those for all
    auto put = [&](int which, const PlanMove &m) {
        const int n = blocks(m);
        if (n <= FEW)
            move(m, 0, 1);
        else if (n <= kPlanThreads / 2)
            list[atomicAdd(&listed[which], 1)] = m;
        else
            list[kPlanThreads - 1 - atomicAdd(&listed[2 + which], 1)] = m;
    };
    auto work_off = [&](int which) {
        constexpr int U = 4;   // moves at once: their loads wait together
        __syncthreads();
        const int n = listed[which], many = listed[2 + which];
        for (int x = 0; x < many; x++)
            move(list[kPlanThreads - 1 - x], tid, kPlanThreads);
        for (int x = U * w; x < n; x += U * WAVES) {
            PlanMove m[U];
            int v[U], count[U];
#pragma unroll
            for (int u = 0; u < U; u++) {
                m[u] = list[min(x + u, n - 1)];
                count[u] = x + u < n ? blocks(m[u]) : 0;
            }
#pragma unroll
            for (int u = 0; u < U; u++)
                if (lane < count[u])
                    v[u] = *source(m[u], lane);
#pragma unroll
            for (int u = 0; u < U; u++)
                if (lane < count[u])
                    *target(m[u], lane) = v[u];
#pragma unroll
            for (int u = 0; u < U; u++)
                if (count[u] > 64)
                    move(m[u], 64 + lane, 64);
        }
        __syncthreads();
        if constexpr (N != 1) {   // (the next sequences' moves take its place)
            if (tid < 4)
                listed[tid] = 0;
            __syncthreads();
        }
    };

    // what is released first: those that grow may take it
    if (total[2] > 0) {
        int at = add_sat(held, before[2]);
#pragma unroll N > 0 ? N : 1
        for (int k = 0; k < per; k++) {   // (a list of the threads' k-th sequences)
            const int s = s0 + k;
            if (s < s1) {
                const PlanSeq q = seq(k);
                if (q.drop() > 0 && at < max_free)
                    put(0, PlanMove{s, q.need, at, -q.drop()});
                at = add_sat(at, q.drop());
            }
            work_off(0);
        }
    }
    int first = before[0], taken = before[1], most_taken = 0;
#pragma unroll N > 0 ? N : 1
    for (int k = 0; k < per; k++) {
        const int s = s0 + k;
        if (s < s1) {
            const PlanSeq q = seq(k);
            const int upto = add_sat(taken, q.grow());
            const bool fine = q.grow() == 0 || upto <= there;
            if (fine && q.grow() > 0) {
                put(1, PlanMove{s, q.have, there - 1 - taken, q.grow()});
                most_taken = upto;
            }
            a.q_start[s] = first;
            a.seq_lens[s] = fine ? q.want : q.old;
            if constexpr (N > 0) {
                start[s] = first;
                begin[s] = fine ? q.old : ~q.old;
            }
            first = add_sat(first, q.fresh());
            taken = upto;
        }
        if (total[1] > 0)   // (uniform)
            work_off(1);
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1)
        most_taken = max(most_taken, __shfl_xor(most_taken, o));
    if (lane == 0)
        most[w] = most_taken;
    if (tid == 0) {
        a.q_start[a.n_seqs] = total[0];
        if constexpr (N > 0)
            start[a.n_seqs] = total[0];
    }
    __syncthreads();
    if (tid == 0) {
#pragma unroll
        for (int x = 1; x < WAVES; x++)
            most_taken = max(most_taken, most[x]);
        *a.n_free_out = there - most_taken;
    }
    if (!a.tokens_too)
        return;
    for (int t = tid; t < a.n_tokens; t += kPlanThreads) {
        if constexpr (N > 0) {
            const int s = plan_find(start, a.n_seqs, t);
            if (s >= a.n_seqs) {
                a.slots[t] = -1;
                a.positions[t] = 0;
                continue;
            }
            const int b = begin[s];
            plan_place(a, t, s, (b < 0 ? ~b : b) + (t - start[s]), b >= 0);
        } else {
            plan_token(a, t);
        }
    }
}

template <int N>
__global__ __launch_bounds__(kPlanThreads) void plan_all_kernel(const PlanArgs a)
{
    plan_body<N>(a);
}

__global__ __launch_bounds__(256) void plan_slots_kernel(const PlanArgs a)
{
    const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (t < a.n_tokens)
        plan_token(a, (int)t);
}

}  // namespace

const void *plan_kernel(int n_seqs)
{
    return n_seqs <= kPlanThreads       ? reinterpret_cast<const void *>(&plan_all_kernel<1>)
           : n_seqs <= 4 * kPlanThreads ? reinterpret_cast<const void *>(&plan_all_kernel<4>)
                                        : reinterpret_cast<const void *>(&plan_all_kernel<0>);
}
const void *plan_tokens_kernel() { return reinterpret_cast<const void *>(&plan_slots_kernel); }

}  // namespace isoq
