// Copies of cache blocks and compaction of sequences in place.  Both only move
// bytes: HBM traffic (each byte read once and written once) bounds them, and a
// call's launch the small ones.
//
// d = 128, 3 bits: 4,096 blocks of 32 heads x 16 positions (436 MB read and
// written) 89 us, 4.9 TB/s; 16 blocks of 8 heads 3 us (7.4 a call).  8 sequences of
// 32,768 positions compacted to half of them, chosen at random for each of 8 heads
// (174 MB), 71 us, 2.5 TB/s: of the 64-byte lines that are read half stays, and
// with all of them it is 3.7.  One of 1,000 positions 5 us (8.4 a call).
#include "isoq_pages.h"

#include <type_traits>

#include "isoq_device.h"

namespace isoq {
namespace {

// Workgroup (pair, plane, run of kCopyUnits accesses): every lane's loads go out
// before its stores.
template <typename T>
__device__ __forceinline__ void copy_run(const uint8_t *src, uint8_t *dst, int64_t units, int64_t u0)
{
    constexpr int N = kCopyUnits / 256;
    T x[N];
#pragma unroll
    for (int i = 0; i < N; i++) {   // (past the end: the last one again, not stored)
        const int64_t u = min(u0 + 256 * i + (int64_t)threadIdx.x, units - 1);
        x[i] = __builtin_nontemporal_load(reinterpret_cast<const T *>(src) + u);
    }
#pragma unroll
    for (int i = 0; i < N; i++) {
        const int64_t u = u0 + 256 * i + threadIdx.x;
        if (u < units)
            __builtin_nontemporal_store(x[i], reinterpret_cast<T *>(dst) + u);
    }
}

__global__ __launch_bounds__(256) void copy_kernel(const CopyArgs a)
{
    const int c = blockIdx.y;
    const int64_t stride = a.stride[c], units = stride / a.unit[c], u0 = (int64_t)blockIdx.z * kCopyUnits;
    if (u0 >= units)
        return;
    const int32_t from = a.pairs[2 * (int64_t)blockIdx.x], to = a.pairs[2 * (int64_t)blockIdx.x + 1];
    if (from < 0 || from >= a.n_blocks || to < 0 || to >= a.n_blocks || from == to)
        return;
    const uint8_t *src = a.plane[c] + from * stride;
    uint8_t *dst = a.plane[c] + to * stride;
    switch (a.unit[c]) {
    case 16: copy_run<u32x4>(src, dst, units, u0); break;
    case 4: copy_run<uint32_t>(src, dst, units, u0); break;
    default: copy_run<uint8_t>(src, dst, units, u0); break;
    }
}

// One chain of one head of one sequence, kTile positions at a time in order.
// In place: position i takes what was at keep[i] >= i, and keep ascends, so a
// tile's stores (positions i) can only meet sources of its own or of earlier
// tiles (those of later ones are at keep[j] >= j > i).  The tile's loads have
// arrived before any of its stores (the wait and the barrier); the next tile's
// loads need not wait for them.
constexpr int kPerLane = 4, kTile = kCompactThreads * kPerLane;

template <typename T>
__device__ __forceinline__ void compact_chain(const CompactArgs &a, uint8_t *base, int64_t bstride, int64_t pstride)
{
    const int s = blockIdx.y, n = min(max(a.n_keep[s], 0), a.max_keep);
    const int32_t *keep = a.keep + ((int64_t)s * a.keep_heads + (a.keep_heads == 1 ? 0 : blockIdx.x)) * a.max_keep;
    const int32_t *table = a.block_table + (int64_t)s * a.max_blocks;
    const uint32_t cap = (uint32_t)((int64_t)a.max_blocks * a.block_size);
    // The address of a position; ok is cleared where it has no page (the
    // address is then one in block 0, not written).  No branches: the loads of
    // a lane's entries go out together.
    auto at = [&](uint32_t pos, bool &ok) {
        ok = ok && pos < cap;
        pos = min(pos, cap - 1);
        const uint32_t bi = fast_div(pos, a.div_block);
        int32_t blk = table[bi];
        ok = ok && blk >= 0 && blk < a.n_blocks;
        blk = ok ? blk : 0;
        return reinterpret_cast<T *>(base + blk * bstride + (int64_t)(pos - bi * a.block_size) * pstride);
    };
    T *src[kPerLane], *dst[kPerLane];
    bool ok[kPerLane];
    auto places = [&](int i0) {
        int32_t from[kPerLane];
#pragma unroll
        for (int e = 0; e < kPerLane; e++)
            from[e] = keep[min(i0 + e * kCompactThreads + (int)threadIdx.x, n - 1)];
#pragma unroll
        for (int e = 0; e < kPerLane; e++) {
            const int i = i0 + e * kCompactThreads + (int)threadIdx.x;
            ok[e] = i < n && from[e] != i;
            dst[e] = at((uint32_t)i, ok[e]);
            src[e] = at((uint32_t)from[e], ok[e]);
        }
    };
    if (n == 0)
        return;
    places(0);
    for (int i0 = 0; i0 < n; i0 += kTile) {
        using R = std::conditional_t<(sizeof(T) < 4), uint32_t, T>;
        R x[kPerLane];
        T *to[kPerLane];
        bool on[kPerLane];
#pragma unroll
        for (int e = 0; e < kPerLane; e++) {
            x[e] = *src[e];
            to[e] = dst[e];
            on[e] = ok[e];
        }
        if (n - i0 > kTile)
            places(i0 + kTile);
#pragma unroll
        for (int e = 0; e < kPerLane; e++)
            asm volatile("" : "+v"(x[e])::"memory");   // the loads have arrived
        __syncthreads();
#pragma unroll
        for (int e = 0; e < kPerLane; e++)
            if (on[e])
                *to[e] = (T)x[e];
    }
}

__global__ __launch_bounds__(kCompactThreads) void compact_positions_kernel(const CompactArgs a)
{
    int c = 0;
    while ((int)blockIdx.z >= a.first[c + 1])
        c++;
    uint8_t *base = a.base[c] + blockIdx.x * a.head_stride[c] + ((int)blockIdx.z - a.first[c]) * a.step[c];
    const int64_t bs = a.block_stride[c], ps = a.pos_stride[c];
    switch (a.width[c]) {
    case 16: compact_chain<u32x4>(a, base, bs, ps); break;
    case 8: compact_chain<u32x2>(a, base, bs, ps); break;
    case 4: compact_chain<uint32_t>(a, base, bs, ps); break;
    case 2: compact_chain<uint16_t>(a, base, bs, ps); break;
    default: compact_chain<uint8_t>(a, base, bs, ps); break;
    }
}

}  // namespace

const void *copy_blocks_kernel() { return reinterpret_cast<const void *>(&copy_kernel); }
const void *compact_kernel() { return reinterpret_cast<const void *>(&compact_positions_kernel); }

}  // namespace isoq
