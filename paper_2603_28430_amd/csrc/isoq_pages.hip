// Copies of cache blocks and compaction of sequences in place.  Both only move
// bytes: HBM traffic (each byte read once and written once) bounds them, and a
// call's launch the small ones.
//
// d = 128, 3 bits: 4,096 blocks of 32 heads x 16 positions (436 MB read and
// written) 86 us, 5.0 TB/s; 16 blocks of 8 heads 4 us (7.5 a call); 20,000 blocks of
// one head 17 us, 3.8 TB/s.  8 sequences of
// 32,768 positions compacted to half of them, chosen at random for each of 8 heads
// (174 MB), 71 us, 2.5 TB/s: of the 64-byte lines that are read half stays, and
// with all of them it is 3.7.  One of 1,000 positions 5 us (8.4 a call).
#include "isoq_pages.h"

#include "isoq_device.h"

namespace isoq {
namespace {

// A 16-byte unit, or less, at any address: global memory takes unaligned accesses.
template <typename T>
struct Unaligned {
    T v;
} __attribute__((packed));

template <typename T>
__device__ __forceinline__ T load_at(const uint8_t *p) { return reinterpret_cast<const Unaligned<T> *>(p)->v; }
template <typename T>
__device__ __forceinline__ void store_at(uint8_t *p, T v) { reinterpret_cast<Unaligned<T> *>(p)->v = v; }

// kCopyUnits accesses of a plane, pair after pair: small blocks share a workgroup
// (one of their own cost more in launches than the copy: 20,000 blocks of 16
// positions of one head, d = 128, 3 bits, 80 us).  A block that is no multiple of 16
// bytes ends with an access that overlaps the one before.  Every lane's loads go out
// before its stores.
template <typename T>
__device__ __forceinline__ void copy_run(const CopyArgs &a, int c)
{
    typedef T Any __attribute__((aligned(1)));
    constexpr int N = kCopyUnits / 256;
    const uint32_t units = (uint32_t)a.units[c];
    const uint64_t first = ((uint64_t)blockIdx.z * gridDim.x + blockIdx.x) * kCopyUnits, total = (uint64_t)a.n_pairs * units;
    if (first >= total)
        return;
    const uint32_t count = (uint32_t)min((uint64_t)kCopyUnits, total - first);
    const uint64_t pair0 = first / units;
    const uint32_t unit0 = (uint32_t)(first - pair0 * units);
    const int64_t stride = a.stride[c];
    uint8_t *const base = a.plane[c];
    T x[N];
    uint8_t *dst[N];
    bool ok[N];
#pragma unroll
    for (int i = 0; i < N; i++) {   // (past the end: the last one again, not stored)
        const uint32_t j = 256 * i + threadIdx.x, at = unit0 + min(j, count - 1), pair = fast_div(at, a.div_units[c]);
        const int32_t *fromto = a.pairs + 2 * (pair0 + pair);
        const int32_t from = fromto[0], to = fromto[1];
        const bool here = from >= 0 && from < a.n_blocks;
        ok[i] = j < count && here && to >= 0 && to < a.n_blocks && from != to;
        const int64_t offset = min((int64_t)(at - pair * units) * (int64_t)sizeof(T), stride - (int64_t)sizeof(T));
        dst[i] = base + (ok[i] ? to : 0) * stride + offset;
        x[i] = __builtin_nontemporal_load(reinterpret_cast<const Any *>(base + (here ? from : 0) * stride + offset));
    }
#pragma unroll
    for (int i = 0; i < N; i++)
        if (ok[i])
            __builtin_nontemporal_store(x[i], reinterpret_cast<Any *>(dst[i]));
}

__global__ __launch_bounds__(256) void copy_kernel(const CopyArgs a)
{
    const int c = blockIdx.y;
    switch (a.unit[c]) {
    case 16: copy_run<u32x4>(a, c); break;
    case 4: copy_run<uint32_t>(a, c); break;
    default: copy_run<uint8_t>(a, c); break;
    }
}

// 16 NU + tail bytes (tail below 16) of a position, held in registers; calls with a
// constant tail have the conditions resolved.
template <int NU>
struct Bytes {
    u32x4 unit[NU > 0 ? NU : 1];
    u32x2 t8;
    uint32_t t4, t2, t1;
    __device__ __forceinline__ void load(const uint8_t *p, int tail)
    {
#pragma unroll
        for (int u = 0; u < NU; u++)
            unit[u] = load_at<u32x4>(p + 16 * u);
        p += 16 * NU;
        if (tail & 8)   // (uniform, as the others)
            t8 = load_at<u32x2>(p);
        if (tail & 4)
            t4 = load_at<uint32_t>(p + (tail & 8));
        if (tail & 2)
            t2 = load_at<uint16_t>(p + (tail & 12));
        if (tail & 1)
            t1 = p[tail & 14];
    }
    __device__ __forceinline__ void store(uint8_t *p, int tail) const
    {
#pragma unroll
        for (int u = 0; u < NU; u++)
            store_at(p + 16 * u, unit[u]);
        p += 16 * NU;
        if (tail & 8)
            store_at(p, t8);
        if (tail & 4)
            store_at(p + (tail & 8), t4);
        if (tail & 2)
            store_at(p + (tail & 12), (uint16_t)t2);
        if (tail & 1)
            p[tail & 14] = (uint8_t)t1;
    }
    __device__ __forceinline__ void arrived(int tail)   // a use of every register: what was loaded is there
    {
#pragma unroll
        for (int u = 0; u < NU; u++)
            asm volatile("" : "+v"(unit[u])::"memory");
        if (tail & 8)
            asm volatile("" : "+v"(t8)::"memory");
        if (tail & 4)
            asm volatile("" : "+v"(t4)::"memory");
        if (tail & 2)
            asm volatile("" : "+v"(t2)::"memory");
        if (tail & 1)
            asm volatile("" : "+v"(t1)::"memory");
    }
};

// One chain of one head of one sequence, PER positions a lane at a time, in
// order.  In place: position i takes what was at keep[i] if that is > i (= i stays,
// and a list that ascends from 0 has none below), so a tile's stores (positions i)
// can only meet sources of its own or of earlier tiles (those of later ones are at
// keep[j] > j > i).  The tile's loads have
// arrived before any of its stores (the wait and the barrier); the next tile's
// loads need not wait for them.
template <int NU, int PER>
__device__ __forceinline__ void compact_chain(const CompactArgs &a, uint8_t *base, int64_t bstride, int64_t pstride, int tail)
{
    constexpr int TILE = kCompactThreads * PER;
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
        return base + blk * bstride + (int64_t)(pos - bi * a.block_size) * pstride;
    };
    uint8_t *src[PER], *dst[PER];
    bool ok[PER];
    auto places = [&](int i0) {
        int32_t from[PER];
#pragma unroll
        for (int e = 0; e < PER; e++)
            from[e] = keep[min(i0 + e * kCompactThreads + (int)threadIdx.x, n - 1)];
#pragma unroll
        for (int e = 0; e < PER; e++) {
            const int i = i0 + e * kCompactThreads + (int)threadIdx.x;
            ok[e] = i < n && from[e] > i;
            dst[e] = at((uint32_t)i, ok[e]);
            src[e] = at((uint32_t)from[e], ok[e]);
        }
    };
    if (n == 0)
        return;
    places(0);
    for (int i0 = 0; i0 < n; i0 += TILE) {
        Bytes<NU> x[PER];
        uint8_t *to[PER];
        bool on[PER];
#pragma unroll
        for (int e = 0; e < PER; e++) {
            x[e].load(src[e], tail);
            to[e] = dst[e];
            on[e] = ok[e];
        }
        if (n - i0 > TILE)
            places(i0 + TILE);
#pragma unroll
        for (int e = 0; e < PER; e++)
            x[e].arrived(tail);
        __syncthreads();
#pragma unroll
        for (int e = 0; e < PER; e++)
            if (on[e])
                x[e].store(to[e], tail);
    }
}

// WHOLE: caches of records stored whole.  (A kernel of its own: its 80 registers
// would leave the other, of half as many, one workgroup a compute unit instead of
// two, and 56 us instead of 48 for 8 x 32 heads x 8,192 positions.)
template <bool WHOLE>
__global__ __launch_bounds__(kCompactThreads) void compact_positions_kernel(const CompactArgs a)
{
    int c = 0;
    while ((int)blockIdx.z >= a.first[c + 1])
        c++;
    uint8_t *base = a.base[c] + blockIdx.x * a.head_stride[c] + ((int)blockIdx.z - a.first[c]) * a.step[c];
    const int64_t bs = a.block_stride[c], ps = a.pos_stride[c];
    switch (const int width = a.width[c]; width) {   // (uniform) the cache layout's own widths first
    case 4: compact_chain<0, 4>(a, base, bs, ps, 4); break;
    case 8: compact_chain<0, 4>(a, base, bs, ps, 8); break;
    case 16: compact_chain<1, 4>(a, base, bs, ps, 0); break;
    default:
        if constexpr (WHOLE) {
            switch (width >> 4) {
            case 0: compact_chain<0, 4>(a, base, bs, ps, width & 15); break;
            case 1: compact_chain<1, 4>(a, base, bs, ps, width & 15); break;
            case 2: compact_chain<2, 2>(a, base, bs, ps, width & 15); break;
            case 3: compact_chain<3, 2>(a, base, bs, ps, width & 15); break;
            case 4: compact_chain<4, 2>(a, base, bs, ps, 0); break;
            }
        }
    }
}

}  // namespace

const void *copy_blocks_kernel() { return reinterpret_cast<const void *>(&copy_kernel); }
const void *compact_kernel(bool whole)
{
    return whole ? reinterpret_cast<const void *>(&compact_positions_kernel<true>)
                 : reinterpret_cast<const void *>(&compact_positions_kernel<false>);
}

}  // namespace isoq
