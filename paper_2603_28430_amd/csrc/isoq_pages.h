// Pages of a paged cache: copies of whole cache blocks, and compaction of
// sequences to the positions that are kept (isoq_pages.hip).
#pragma once

#include "isoq_internal.h"

namespace isoq {

constexpr int kCachePlanes = 6;   // K and V records and norms, signs, gamma

struct CopyArgs {
    uint8_t *plane[kCachePlanes];
    int64_t stride[kCachePlanes];   // bytes of a cache block
    int32_t unit[kCachePlanes];     // bytes per access (16, 4 or 1; a block has one at least)
    int32_t units[kCachePlanes];    // accesses per block
    FastDiv div_units[kCachePlanes];
    const int32_t *pairs;           // [n_pairs][2] source, destination
    int64_t n_pairs, n_blocks;
};
// Grid (workgroups of kCopyUnits accesses of all pairs, planes, the same past
// kCopyGrid), 256 threads.
constexpr int kCopyUnits = 2048, kCopyGrid = 1 << 20;
const void *copy_blocks_kernel();

// What moves when a sequence is compacted: a chain is `width` bytes of every
// position of a head, the byte columns that the cache layout keeps together: a
// record's piece, a norm, or a part of a record stored whole.  Chain p of column
// set c is at
//     base + block block_stride + head head_stride + p step + pos pos_stride.
// A record stored whole is cut into 64 bytes a chain and the rest of it where
// sequences and heads alone fill the card, and into 16, 8, 4, 2 and 1 where they do
// not and more workgroups are wanted.  (us, d = 80, 3 bits, 30 bytes, by fifteen
// chains of 2 bytes / 16, 8, 4, 2 / one: 8 x 32 heads x 12,000 positions 625 / 179 / 68,
// 3 x 8 x 60,000 82 / 41 / 78, one head 68 / 84 / 141; d = 160, 60 bytes: 8 x 32 x 6,553 496
// / 178 / 60, 3 x 8 x 60,000 113 / 58 / 112.)
constexpr int kCompactColumns = 2 * 5 + 4;   // K and V records, their norms, signs, gamma
struct CompactArgs {
    const int32_t *keep;           // [n_seqs][keep_heads][max_keep]
    const int32_t *n_keep;         // [n_seqs]
    const int32_t *block_table;    // [n_seqs][max_blocks]
    int64_t n_blocks;
    int32_t keep_heads, max_keep, max_blocks, block_size;
    FastDiv div_block;
    uint8_t *base[kCompactColumns];
    int64_t block_stride[kCompactColumns], head_stride[kCompactColumns], step[kCompactColumns];
    int32_t pos_stride[kCompactColumns], width[kCompactColumns];
    int32_t first[kCompactColumns + 1];   // set c's chains are grid z first[c] .. first[c + 1] - 1
};
// Grid (heads, sequences, chains), kCompactThreads threads.
constexpr int kCompactThreads = 1024;
// whole: some records are stored whole (widths other than 4, 8 and 16).
const void *compact_kernel(bool whole);

}  // namespace isoq
