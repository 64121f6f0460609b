// Pages of a paged cache: copies of whole cache blocks, and compaction of
// sequences to the positions that are kept (isoq_pages.hip).
#pragma once

#include "isoq_internal.h"

namespace isoq {

constexpr int kCachePlanes = 6;   // K and V records and norms, signs, gamma

struct CopyArgs {
    uint8_t *plane[kCachePlanes];
    int64_t stride[kCachePlanes];   // bytes of a cache block
    int32_t unit[kCachePlanes];     // bytes per access (16, 4 or 1): divides the stride and the plane's address
    const int32_t *pairs;           // [n_pairs][2] source, destination
    int64_t n_blocks;
};
// Grid (pairs, planes, runs of kCopyUnits accesses of a block), 256 threads.
constexpr int kCopyUnits = 2048;
const void *copy_blocks_kernel();

// What moves when a sequence is compacted: a chain is `width` bytes (16, 8, 4,
// 2 or 1) of every position of a head, the byte columns that the cache layout
// keeps together: a record's piece, a norm, or a unit of a record stored whole.
// Chain p of plane c is at
//     base + block block_stride + head head_stride + p step + pos pos_stride.
struct CompactArgs {
    const int32_t *keep;           // [n_seqs][keep_heads][max_keep]
    const int32_t *n_keep;         // [n_seqs]
    const int32_t *block_table;    // [n_seqs][max_blocks]
    int64_t n_blocks;
    int32_t keep_heads, max_keep, max_blocks, block_size;
    FastDiv div_block;
    uint8_t *base[kCachePlanes];
    int64_t block_stride[kCachePlanes], head_stride[kCachePlanes], step[kCachePlanes];
    int32_t pos_stride[kCachePlanes], width[kCachePlanes];
    int32_t first[kCachePlanes + 1];   // plane c's chains are grid z first[c] .. first[c + 1] - 1
};
// Grid (heads, sequences, chains), kCompactThreads threads.
constexpr int kCompactThreads = 1024;
const void *compact_kernel();

}  // namespace isoq
