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
#include <hip/hip_runtime.h>

#include "isoq_device.h"
#include "isoq_step.h"

namespace isoq {
namespace {

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

// Slot and position of token t, once the sequences' lengths, first tokens and
// blocks are there.
__device__ __forceinline__ void plan_token(const PlanArgs &a, int t)
{
    int lo = 0, hi = a.n_seqs;   // the first sequence that ends past t
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (a.q_start[mid + 1] > t)
            hi = mid;
        else
            lo = mid + 1;
    }
    int64_t slot = -1;
    int pos = 0;
    if (lo < a.n_seqs) {
        const int first = a.q_start[lo], len = a.seq_lens[lo];
        const bool fine = len == min(max(a.new_lens[lo], 0), a.cap);   // not refused
        pos = (fine ? len - (a.q_start[lo + 1] - first) : len) + (t - first);
        const uint32_t j = fast_div((uint32_t)pos, a.div_block);
        if (fine && pos >= 0 && j < (uint32_t)a.max_blocks) {
            const int blk = a.block_table[(int64_t)lo * a.max_blocks + j];
            if (blk >= 0)
                slot = (int64_t)blk * a.block_size + (pos - (int)(j * (uint32_t)a.block_size));
        }
    }
    a.slots[t] = slot;
    a.positions[t] = pos;
}

__global__ __launch_bounds__(kPlanThreads) void plan_all_kernel(const PlanArgs a)
{
    constexpr int WAVES = kPlanThreads / 64;
    __shared__ int64_t wave_sum[3][WAVES], most[WAVES];
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const int per = (a.n_seqs + kPlanThreads - 1) / kPlanThreads;   // consecutive sequences a thread
    const int s0 = min(tid * per, a.n_seqs), s1 = min(s0 + per, a.n_seqs);

    int64_t sum[3] = {0, 0, 0}, before[3], total[3];
    for (int s = s0; s < s1; s++) {
        const PlanSeq q = plan_seq(a, s);
        sum[0] += q.fresh();
        sum[1] += q.grow();
        sum[2] += q.drop();
    }
    for (int k = 0; k < 3; k++) {
        int64_t x = sum[k];
        for (int o = 1; o < 64; o <<= 1) {
            const int64_t y = __shfl_up((long long)x, o);
            if (lane >= o)
                x += y;
        }
        before[k] = x - sum[k];
        if (lane == 63)
            wave_sum[k][w] = x;
    }
    __syncthreads();
    for (int k = 0; k < 3; k++) {
        total[k] = 0;
        for (int x = 0; x < WAVES; x++) {
            if (x == w)
                before[k] += total[k];
            total[k] += wave_sum[k][x];
        }
    }
    const int64_t held = min(max((int64_t)*a.n_free, (int64_t)0), a.max_free);
    const int64_t there = min(held + total[2], a.max_free);

    // what is released first: those that grow may take it
    int64_t at = held + before[2];
    for (int s = s0; s < s1; s++) {
        const PlanSeq q = plan_seq(a, s);
        for (int j = q.need; j < q.have; j++, at++)
            if (at < a.max_free)
                a.free_blocks[at] = a.block_table[(int64_t)s * a.max_blocks + j];
    }
    __syncthreads();
    int64_t first = before[0], taken = before[1], most_taken = 0;
    for (int s = s0; s < s1; s++) {
        const PlanSeq q = plan_seq(a, s);
        const bool fine = q.grow() == 0 || taken + q.grow() <= there;
        if (fine) {
            for (int j = q.have; j < q.need; j++)
                a.block_table[(int64_t)s * a.max_blocks + j] = a.free_blocks[there - 1 - (taken + j - q.have)];
            if (q.grow() > 0)
                most_taken = taken + q.grow();
        }
        a.q_start[s] = (int)min(first, (int64_t)0x7FFFFFFF);
        a.seq_lens[s] = fine ? q.want : q.old;
        first += q.fresh();
        taken += q.grow();
    }
    for (int o = 32; o > 0; o >>= 1)
        most_taken = max(most_taken, (int64_t)__shfl_xor((long long)most_taken, o));
    if (lane == 0)
        most[w] = most_taken;
    __syncthreads();
    if (tid == 0) {
        for (int x = 1; x < WAVES; x++)
            most_taken = max(most_taken, most[x]);
        a.q_start[a.n_seqs] = (int)min(total[0], (int64_t)0x7FFFFFFF);
        *a.n_free_out = (int)(there - most_taken);
    }
    if (a.tokens_too) {
        __syncthreads();
        for (int t = tid; t < a.n_tokens; t += kPlanThreads)
            plan_token(a, t);
    }
}

__global__ __launch_bounds__(256) void plan_slots_kernel(const PlanArgs a)
{
    const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (t < a.n_tokens)
        plan_token(a, (int)t);
}

}  // namespace

const void *plan_kernel() { return reinterpret_cast<const void *>(&plan_all_kernel); }
const void *plan_tokens_kernel() { return reinterpret_cast<const void *>(&plan_slots_kernel); }

}  // namespace isoq
