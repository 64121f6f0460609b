// Attention over the paged quantized cache on the integer matrix cores (widths
// of the tuned decoding kernels).
//
// A workgroup of four waves has 4, 8 or 12 rows (isoq_attn_m_pick.h); its waves take
// 64 positions in turn.
//
// The logits are those of isoq_scores_m.h: rotated query and codebook as 8-bit
// digits, products of digits summed exactly in int32 by v_mfma_i32_16x16x64_i8,
// the level digits picked four at a time by v_perm_b32.  The sum of values is
// the same product the other way round: with w_t = p_t rho_vt,
//     sum_t w_t c[idx_tj],
// w as a 31-bit integer cut into four digits (in units of 2^-30 of the row's
// largest one in the tile) and the levels as two digits (fp16 queries: a level
// within 2^-16 of the largest) or three (fp32: 2^-24); at 4 bits the digits of
// the eight magnitudes, complemented for the negative ones.
//
// Lane layout.  A tile is 64 positions of a wave and four rows (query heads of
// new tokens that share the key head).  The logits' instruction has the rows'
// digits as A's rows (4 per row) and keys as columns, so lane 16 r + i ends up
// with row r's logits of the positions i, 16 + i, 32 + i, 48 + i.  It turns them
// into w, whose 4 x 4 (position, digit) bytes are transposed in registers and
// go through 1 KB of LDS to become A of the second product: rows again (row,
// digit), k = the tile's 64 positions, lane 16 g + m holding row m's digit for
// the positions 16 i + 4 g + c (word c, byte i).  B's columns are coordinates:
// lane 16 g + n has the coordinates n D/16 .. (n + 1) D/16 - 1 of the same 16
// positions, read from the records (staged in LDS as they are): the index bits
// of four positions are transposed bytewise (v_perm) and then masked, which
// gives selector bytes of four positions without spreading each row's bits.
// Its result has row r's four digit sums in lane 16 r + n: the digits are
// combined by shifts and adds and enter an fp32 sum, one register per
// coordinate and row, which the running maximum of the row rescales.
//
// What bounds it (the kernel's time in a trace; a join of splits takes 4 to 5 us
// more).  With one row a key head (8 sequences x 32 heads x 32,768 positions, d =
// 128, 3 bits: 873 MB) 197 to 205 us, 4.3 TB/s where a large copy moves 4.7, and 216
// to 222 once such calls have followed each other for some ms and the clock has
// fallen: vector
// instructions (87% of issue) no less than memory.  With 4 rows (16 ragged
// sequences x 8 key heads, up to 8,192 positions, 4 bits) 41 us: the decoding's
// vector instructions (about 750 a tile of 64 positions; 52% of issue, a third of
// them the workgroups' preparation) and waits (37%).  With 8 rows (one sequence x 8
// key heads x 131,071) 46 us, 2.4 TB/s: vector (64% of issue) and matrix
// instructions (20%).  d = 256, 2 rows, 4 x 8 heads x 8,190: 21 us.  One sequence of
// 700 positions 11 us: three tiles a wave in series, on eight workgroups.
#pragma once

#include "isoq_attn_device.h"
#include "isoq_scores_m.h"

namespace isoq {
namespace {

// The largest of v and of the lane that a DPP control names, in one instruction:
// left to itself, fmaxf of a moved value is a move, a second maximum that
// quiets NaNs, and the maximum.  (The two wait states between writing a
// register and reading it by DPP are the asm's own.)
#define ISOQ_DPP_MAX(v, ctrl)                                                                      \
    asm("s_nop 1\n\tv_max_f32_dpp %0, %0, %0 " ctrl " row_mask:0xf bank_mask:0xf" : "+v"(v))

// The largest of a 16-lane row, in every lane of it.
__device__ __forceinline__ float row_max16(float v)
{
    ISOQ_DPP_MAX(v, "quad_perm:[1,0,3,2]");
    ISOQ_DPP_MAX(v, "quad_perm:[2,3,0,1]");
    ISOQ_DPP_MAX(v, "row_half_mirror");
    ISOQ_DPP_MAX(v, "row_mirror");
    return v;
}

// Eight coordinates of a query row, as loaded.
struct QueryChunk {
    Raw<true> half;
    Raw<false> whole;
};

template <int D>
__device__ __forceinline__ void attn_load_query(const AttnArgs &a, const AttnSeq &sq, int h, int r, int l, QueryChunk &q)
{
    const int i = r / a.group, g = r - i * a.group;
    const int64_t row = (int64_t)(sq.first + i) * a.n_q_heads + h * a.group + g;
    if (a.q_f16)
        load_row_chunk<true>(static_cast<const char *>(a.q) + row * D * 2 + l * 16, q.half);
    else
        load_row_chunk<false>(static_cast<const char *>(a.q) + row * D * 4 + l * 32, q.whole);
}

// Rotate chunk l of a query row of key head h (scale folded in) into qt[0 .. 7];
// its largest magnitude, an infinity or NaN among them, to mx.
template <int VAR, int D>
__device__ __forceinline__ void attn_rotate(const AttnArgs &a, int h, int l, const QueryChunk &q, float *qt, uint32_t *mx)
{
    constexpr int LPQ = D / kCoordsPerLane, PL = kLanePL<VAR>;
    float x[8], y[8], P[VAR == VAR_BLOCK8 ? 8 : PL];
    if (a.q_f16)
        unpack<true>(q.half, x);
    else
        unpack<false>(q.whole, x);
    const float *par = a.k_params + ((int64_t)(a.k_sets == 1 ? 0 : h) * LPQ + l) * PL;
    if constexpr (VAR == VAR_BLOCK8) {
#pragma unroll
        for (int e = 0; e < 8; e++) {   // row by row: all 64 parameters at once would set the kernel's registers
            load_params<8>(par + 8 * e, P);
            y[e] = P[0] * x[0];
#pragma unroll
            for (int c = 1; c < 8; c++)
                y[e] = fmaf(P[c], x[c], y[e]);
            __builtin_amdgcn_sched_barrier(0);
        }
    } else {
        load_params<PL>(par, P);
        rotate_forward<VAR>(P, x, y);
    }
    uint32_t m = 0;
#pragma unroll
    for (int k = 0; k < 8; k++) {
        const float v = y[k] * a.scale;
        qt[k] = v;
        m = max(m, __float_as_uint(fabsf(v)));   // ordered as the magnitudes; NaN above all
    }
    atomicMax(mx, m);
}

template <int D>
__device__ __forceinline__ void attn_rotate_any(const AttnArgs &a, int h, int l, const QueryChunk &q, float *qt,
                                                uint32_t *mx)
{
    switch (a.variant) {
    case VAR_FULL: attn_rotate<VAR_FULL, D>(a, h, l, q, qt, mx); break;
    case VAR_FAST: attn_rotate<VAR_FAST, D>(a, h, l, q, qt, mx); break;
    case VAR_PLANAR2D: attn_rotate<VAR_PLANAR2D, D>(a, h, l, q, qt, mx); break;
    default: attn_rotate<VAR_BLOCK8, D>(a, h, l, q, qt, mx); break;
    }
}

template <int D, int BITS, int NT>
struct AttnMShape {
    using S = ScoreMShape<D, BITS, 0>;
    static constexpr int WV = 4;                     // waves per workgroup
    static constexpr int ROWS = 4 * NT;              // rows per workgroup
    static constexpr int CL = D / 16;                // coordinates per lane of the second product
    // A record as staged in LDS: a lane's coordinates in groups of up to 8,
    // [group][lane] (one aligned read each: reads that are not aligned to
    // their size took 60 cycles here, aligned ones 10).  Groups of exactly 32
    // or 16 bits that start on whole ones are the record itself; others get a
    // word each.  A row's words + 4: the rows 4 apart that a read's quarters
    // touch lie 16 banks apart.
    static constexpr int NG = (CL + 7) / 8;
    static constexpr int GB = (CL < 8 ? CL : 8) * BITS;   // bits of a full group
    static constexpr bool HALF = GB == 16 && CL % 8 == 0;
    static constexpr int SW = HALF ? 8 * NG : 16 * NG;    // words of a staged record
    static constexpr int RS = SW + 4;
    // word i of a staged record from the record's words
    static __device__ __forceinline__ uint32_t staged(const uint32_t *w, int i)
    {
        if (HALF) {   // groups 2 i and 2 i + 1 (lanes 2 j, 2 j + 1)
            const int g = i / 8, j = i - 8 * g, lo = half(2 * j, g), hi = half(2 * j + 1, g);
            if (hi == lo + 1 && lo % 2 == 0)
                return w[lo / 2];
            return __builtin_amdgcn_perm(w[hi / 2], w[lo / 2], (lo % 2 ? 0x0302u : 0x0100u) | (hi % 2 ? 0x07060000u : 0x05040000u));
        }
        const int g = i / 16, n = i - 16 * g, bit = (n * CL + 8 * g) * BITS, at = bit >> 5, sh = bit & 31;
        const int bits = (CL - 8 * g < 8 ? CL - 8 * g : 8) * BITS;
        if (sh == 0)
            return w[at];
        if (sh + bits <= 32)
            return w[at] >> sh;
        return __builtin_amdgcn_alignbit(w[at + 1], w[at], sh);
    }
    static constexpr int half(int n, int g) { return n * (CL / 8) + g; }   // half-word of lane n's group g
    // LDS words: per row of the workgroup its digit rows, digit sums (8), then
    // the rotated queries; per wave the staged records w's digits and the norms
    static constexpr int row_words() { return 4 * S::ROWW + 8; }
    static constexpr int wave_words() { return 64 * RS + NT * 256 + 128; }
    static constexpr int lds_words()
    {
        // the rotated queries are gone when the waves' parts are written, and
        // everything when the waves' sums are merged (waves x rows x D, m and l)
        const int loop = ROWS * row_words() + (ROWS * D > WV * wave_words() ? ROWS * D : WV * wave_words());
        const int merge = WV * ROWS * (D + 2);
        return loop > merge ? loop : merge;
    }
};

// Selector words of the coordinates 0 .. n - 1 from byte planes: byte i of b[k]
// is byte k of record part i (n * BITS bits each), byte i of sel[c] the index of
// part i's coordinate c (4 bits: in its lower half; see magnitude).
template <int BITS, int N>
__device__ __forceinline__ void plane_selectors(const uint32_t *b, uint32_t *sel)
{
    constexpr uint32_t mask = BITS == 2 ? 0x03030303u : 0x07070707u;
#pragma unroll
    for (int c = 0; c < N; c++) {
        const int bit = c * BITS, k = bit >> 3, sh = bit & 7;
        if (BITS == 4)
            sel[c] = sh ? b[k] >> sh : b[k];
        else if (sh + BITS <= 8)
            sel[c] = (sh ? b[k] >> sh : b[k]) & mask;
        else   // (3 bits) across two bytes
            sel[c] = bit_select(vector_const(sh == 6 ? 0x03030303u : 0x01010101u), b[k] >> sh, b[k + 1] << (8 - sh)) & mask;
    }
}

// A chunk's 3-bit indices, 32 coordinates (three words of the chunk) at a time:
// the four octets' bytes gathered into planes give eight selector words for 25
// instructions, spreading an octet's bits over its own words 8 or 9 for two.
// Word j of a block of 32: coordinates j, 8 + j, 16 + j, 24 + j.
template <int BITS>
constexpr bool attn_by_planes(int chunk, int quad) { return BITS == 3 && 4 * (quad / 8 * 8 + 8) <= chunk; }

template <class S, int BITS, int NS>
__device__ __forceinline__ void attn_selectors(const uint32_t *y, int q0, uint32_t *sel)
{
    if constexpr (BITS == 3) {
        if (attn_by_planes<BITS>(S::CC, q0)) {
            const uint32_t *w = y + q0 / 8 * 3;
            const uint32_t b[3] = {
                __builtin_amdgcn_perm(w[2], __builtin_amdgcn_perm(w[1], w[0], 0x0C060300u), 0x05020100u),
                __builtin_amdgcn_perm(w[2], __builtin_amdgcn_perm(w[1], w[0], 0x0C070401u), 0x06020100u),
                __builtin_amdgcn_perm(w[2], __builtin_amdgcn_perm(w[1], w[0], 0x0C0C0502u), 0x07040100u)};
            uint32_t all[8];
            plane_selectors<3, 8>(b, all);
#pragma unroll
            for (int j = 0; j < NS; j++)
                sel[j] = all[q0 % 8 + j];
            return;
        }
    }
    if constexpr (BITS == 4) {   // a word holds 8 coordinates: its lower and its upper half-bytes
#pragma unroll
        for (int j = 0; j < NS; j++)
            sel[j] = (q0 + j) % 2 ? y[(q0 + j) / 2] >> 4 : y[(q0 + j) / 2];
        return;
    }
    selectors<S, BITS, NS>(y, q0, sel);
}

// 4-bit indices in the lower half of each byte: 0xFF where the index is below 8,
// and the index of the magnitude, 0 .. 7: index 8 + m has magnitude m, 7 - m is
// its mirror image, whose digits are the complements.
__device__ __forceinline__ uint32_t magnitude(uint32_t &sel)
{
    const uint32_t inv = __builtin_amdgcn_perm(0u, 0u, 0x0D0D0D0Du - ((sel >> 3) & 0x01010101u));
    sel = __builtin_amdgcn_bitop3_b32(sel, inv, vector_const(0x07070707u), 0x28);   // (sel ^ inv) & 7
    return inv;
}

// Chunk coordinate of byte b of quad q.
template <class S, int BITS>
__device__ __forceinline__ int attn_coord(int q, int b)
{
    if (attn_by_planes<BITS>(S::CC, q))
        return q / 8 * 32 + 8 * b + q % 8;
    if (BITS == 2 && 4 * (q / 4) + 4 <= S::CC / 4)
        return 16 * (q / 4) + 4 * b + q % 4;
    return 8 * (q / 2) + 2 * b + q % 2;
}

// Selector bytes of the four positions x[0..3] for the coordinates of a group:
// `n` coordinates whose bits start at bit 0 of x; sel[c] byte i = index of
// coordinate c at position i.
template <int BITS, int N>
__device__ __forceinline__ void position_selectors(const uint32_t x[4], uint32_t sel[N])
{
    constexpr int PLANES = (N * BITS + 7) / 8;
    uint32_t b[4];   // byte k of the four positions
    {
        const uint32_t lo = __builtin_amdgcn_perm(x[1], x[0], 0x05010400u), hi = __builtin_amdgcn_perm(x[3], x[2], 0x05010400u);
        b[0] = __builtin_amdgcn_perm(hi, lo, 0x05040100u);
        if constexpr (PLANES > 1)
            b[1] = __builtin_amdgcn_perm(hi, lo, 0x07060302u);
    }
    if constexpr (PLANES > 2) {
        const uint32_t lo = __builtin_amdgcn_perm(x[1], x[0], 0x07030602u), hi = __builtin_amdgcn_perm(x[3], x[2], 0x07030602u);
        b[2] = __builtin_amdgcn_perm(hi, lo, 0x05040100u);
        if constexpr (PLANES > 3)
            b[3] = __builtin_amdgcn_perm(hi, lo, 0x07060302u);
    }
    plane_selectors<BITS, N>(b, sel);
}

// Waves a SIMD that the registers are to allow, where the compiler alone takes a few more than
// leave that number (with none to ten of them spilled).  (us left to the compiler / so, 8
// sequences of 8,192 positions, 8 heads: 12 rows a head, fp16, d = 80, 2 bits 34 / 30, 3 bits 37 /
// 32, d = 96, 2 bits 36 / 32; 8 rows, fp32, d = 128, 3 bits 34 / 32; 2 x 512 tokens, 8 x 4 heads,
// fp32, 3 bits 1,070 / 971.)
constexpr int attn_m_waves(int d, int bits, int nt, int vd)
{
    return nt == 2 ? (vd == 2 && d * bits <= 240 ? 4 : d * bits <= 384 && d <= 128 ? 3 : 1)
                   : (nt == 3 && vd == 2 && d * bits <= 288 && d <= 96 ? 3 : 1);
}

template <int D, int BITS, int NT, int VD, bool PRE>
__global__ __launch_bounds__(256, attn_m_waves(D, BITS, NT, VD)) void attn_m_kernel(const AttnArgs a)
{
    using H = AttnMShape<D, BITS, NT>;
    constexpr int WV = H::WV;
    using S = typename H::S;
    constexpr int64_t RB = (int64_t)D * BITS / 8;
    constexpr int QP = BITS == 4 ? 29 : 30;   // query integers below 2^QP (4 bits: digits of twice them)
    constexpr int CL = H::CL, ROWS = H::ROWS;
    extern __shared__ __align__(16) uint32_t smem[];

    const int hx = (int)(blockIdx.x % (uint32_t)a.n_kv_heads), rt = (int)(blockIdx.x / (uint32_t)a.n_kv_heads);
    const int h = (int)xcd_head((uint32_t)hx, (uint32_t)a.n_kv_heads, a.block_size * RB % 128 != 0);
    const int s = blockIdx.y;
    const int lane = threadIdx.x & 63;
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const AttnSeq sq = attn_seq<PRE>(a, s);
    const int r0 = rt * ROWS, total = sq.rows * a.group;   // rows of the sequence's key head
    if (r0 >= total)   // (block-uniform, as every early return here)
        return;
    const int n = min(ROWS, total - r0);
    const int64_t t0l = (int64_t)blockIdx.z * a.chunk;
    const int t0 = (int)t0l;

    uint32_t *dig = smem;                                            // [ROWS][4][ROWW]
    int *sums = reinterpret_cast<int *>(dig + ROWS * 4 * S::ROWW);   // [ROWS][8]: 4 digit sums, largest magnitude
    uint32_t *mx = reinterpret_cast<uint32_t *>(sums) + 4;
    float *qt = reinterpret_cast<float *>(sums + ROWS * 8);          // [ROWS][D], before the waves' parts
    uint32_t *mine = reinterpret_cast<uint32_t *>(qt) + w * H::wave_words();
    uint32_t *wdig = mine + 64 * H::RS;
    float *norms = reinterpret_cast<float *>(wdig + NT * 256);

    // 0. what does not wait for the lengths: the queries (a chunk of 8 coordinates
    //    per lane), and the block table's entries for the wave's first positions
    //    (later ones are loaded two batches ahead: the records' addresses wait
    //    for them)
    static_assert(ROWS * (D / 8) <= 256, "a chunk of 8 coordinates per lane");
    const int cr = threadIdx.x / (D / 8), cl = threadIdx.x - cr * (D / 8);   // the lane's row and chunk
    QueryChunk query;
    if (cr < n)
        attn_load_query<D>(a, sq, h, r0 + cr, cl, query);
    const int32_t *table = a.block_table + (int64_t)s * a.max_blocks;
    const int tw = t0 + 64 * w + lane;
    auto entry = [&](int b) {   // (positions past the last possible one: that one's)
        return attn_entry<PRE>(a, sq, table, (int)min((int64_t)tw + 64 * WV * (int64_t)b, (int64_t)0x7FFFFFFF));
    };
    AttnEntry next{};
    if (PRE || a.cap > 0)
        next = entry(0);
    __builtin_amdgcn_sched_barrier(0);
    // the positions that the rows attend to: rows come in the tokens' order, so
    // the last one attends to the most
    const int lim_all = sq.limit((r0 + n - 1) / a.group, a.cap), lim_min = sq.limit(r0 / a.group, a.cap);
    if (t0l >= lim_all && blockIdx.z > 0)
        return;   // the join looks at the splits below a row's limit only
    const int tend = (int)min(t0l + a.chunk, (int64_t)lim_all);

    // 1. rotated queries
    for (int i = threadIdx.x; i < ROWS * 8; i += 64 * WV)
        sums[i] = 0;
    __syncthreads();
    if (cr < n)
        attn_rotate_any<D>(a, h, cl, query, qt + cr * D + 8 * cl, mx + 8 * cr);

    // 2. records and norms of the first batch, as in isoq_scores_m.h
    struct Batch {
        uint32_t w[S::RW];
        float rho;
    };
    const uint64_t rstride = (uint64_t)a.n_kv_heads * a.block_size, row0 = (uint64_t)h * a.block_size;
    const uint64_t bstride = rstride * RB;
    auto times = [](uint32_t blk, uint64_t stride, uint32_t add) {   // one multiply unless the stride needs 33 bits
        uint64_t o = (uint64_t)blk * (uint32_t)stride + add;
        if (stride >> 32)
            o += (uint64_t)(blk * (uint32_t)(stride >> 32)) << 32;
        return o;
    };
    const int64_t pstep = (int64_t)a.block_size * S::CP;
    const uint8_t *const k_idx = a.k_idx + row0 * RB, *const v_idx = a.v_idx + row0 * RB;
    const float *const k_rho = a.k_rho + row0, *const v_rho = a.v_rho + row0;
    auto issue = [&](uint64_t at, uint64_t row, const uint8_t *idx, const float *rho, Batch &k) {
        if constexpr (S::LW == 4) {
#pragma unroll
            for (int v = 0; v < S::RW / 4; v++) {
                const u32x4 q4 = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(idx + v * pstep + at));
#pragma unroll
                for (int c = 0; c < 4; c++) {
                    const uint32_t e = q4[c];
                    k.w[4 * v + c] = e;
                }
            }
        } else if constexpr (S::LW == 2) {
            static_assert(S::LW != 2 || S::CP == 8, "one load per piece");
#pragma unroll
            for (int v = 0; v < S::RW / 2; v++) {
                const u32x2 q2 = __builtin_nontemporal_load(reinterpret_cast<const u32x2 *>(idx + v * pstep + at));
                const uint32_t e0 = q2[0], e1 = q2[1];
                k.w[2 * v] = e0;
                k.w[2 * v + 1] = e1;
            }
        } else if constexpr (S::LW == 1) {
#pragma unroll
            for (int v = 0; v < S::RW; v++)
                k.w[v] = reinterpret_cast<const uint32_t *>(idx + at)[v];
        } else {
            // an odd number of half-words, stored whole (isoq_scores_m.h)
            const bool odd = (row0 + row) & 1;
            const uint8_t *pc0 = idx + at;
            const uint32_t *al = reinterpret_cast<const uint32_t *>(pc0 + (odd ? 2 : 0));
            const uint32_t half = *reinterpret_cast<const uint16_t *>(pc0 + (odd ? 0 : RB - 2));
            uint32_t r[S::RW - 1];
#pragma unroll
            for (int v = 0; v < S::RW - 1; v++)
                r[v] = al[v];
            k.w[0] = odd ? (r[0] << 16) | half : r[0];
#pragma unroll
            for (int v = 1; v < S::RW - 1; v++)
                k.w[v] = odd ? __builtin_amdgcn_alignbit(r[v], r[v - 1], 16) : r[v];
            k.w[S::RW - 1] = odd ? r[S::RW - 2] >> 16 : half;
        }
        k.rho = rho[row];
    };
    const int nb = (tend - t0 + 64 * WV - 1) / (64 * WV);   // (0 where no position is left)
    Batch k{}, v{};
    bool valid = false;   // of the lane's position of the batch at hand
    auto fetch = [&](int b) {
        valid = (int64_t)tw + 64 * WV * (int64_t)b < tend && next.blk >= 0 && next.blk < a.n_blocks;
        // an invalid position reads position 0 of the head in block 0 (always
        // present) and gets no weight
        const uint32_t blk = valid ? (uint32_t)next.blk : 0u, pos = valid ? (uint32_t)next.pos : 0u;
        const uint64_t at = times(blk, bstride, 0) + (uint64_t)pos * S::CP;
        const uint64_t row = times(blk, rstride, pos);
        issue(at, row, k_idx, k_rho, k);
        issue(at, row, v_idx, v_rho, v);
        next = entry(b + 1);
    };
    if (nb > 0)
        fetch(0);

    // 3. the queries' digits, as in isoq_scores_m.h
    __syncthreads();
    for (int i = threadIdx.x; i < n * 4 * S::NQ; i += 64 * WV) {
        const int g = i / (4 * S::NQ), cq = i - g * (4 * S::NQ);
        const int c = cq / S::NQ, q = cq - c * S::NQ;
        const int e = head_exponent(__uint_as_float(mx[8 * g]), QP);
        uint32_t word[4] = {0u, 0u, 0u, 0u};
        int sum[4] = {0, 0, 0, 0};
#pragma unroll
        for (int b = 0; b < 4; b++) {
            const int ci = attn_coord<S, BITS>(q, b);
            const int x = ci < S::CC ? to_fixed(qt[g * D + c * S::CC + ci], e) : 0;
            int d[4];
            if constexpr (BITS == 4) {
                digits4(x, d);
#pragma unroll
                for (int j = 0; j < 4; j++)
                    sum[j] += d[j];
            }
            digits4(BITS == 4 ? 2 * x : x, d);
#pragma unroll
            for (int j = 0; j < 4; j++)
                word[j] |= (uint32_t)(d[j] & 255) << (8 * b);
        }
#pragma unroll
        for (int j = 0; j < 4; j++) {
            dig[(g * 4 + j) * S::ROWW + cq] = word[j];
            if constexpr (BITS == 4)
                atomicAdd(sums + 8 * g + j, sum[j]);
        }
    }
    __syncthreads();   // (the waves' parts take the rotated queries' place from here on)

    const int col = lane & 15, kq = lane >> 4;
    uint32_t A[NT][S::NQ];
    i32x4 asum[NT];
    float f1[NT], f2[NT];   // 2^-e (with the quantum) of the digits, in two factors
    float m[NT], l[NT];     // running maximum and (the lane's part of the) sum of row 4 nt + kq,
    float sw[NT];           // (4 bits) and of its weights p rho
    int lim[NT];
    float acc[NT][CL];
#pragma unroll
    for (int nt = 0; nt < NT; nt++) {
        const int ga = 4 * nt + (col >> 2), gr = 4 * nt + kq;
        const uint32_t *row = dig + ((ga < n ? ga : 0) * 4 + (col & 3)) * S::ROWW + kq * S::NQ;
#pragma unroll
        for (int q = 0; q < S::NQ; q += 2) {
            const u32x2 x = *reinterpret_cast<const u32x2 *>(row + q);
            const uint32_t x0 = x[0], x1 = x[1];
            A[nt][q] = ga < n ? x0 : 0u;
            A[nt][q + 1] = ga < n ? x1 : 0u;
        }
        const int gi = gr < n ? gr : 0;
        const int e = head_exponent(__uint_as_float(mx[8 * gi]), QP) - a.k_dig.exp;
        f1[nt] = __builtin_amdgcn_ldexpf(a.k_dig.quantum, -(e / 2));
        f2[nt] = __builtin_amdgcn_ldexpf(1.f, e / 2 - e);
        asum[nt] = i32x4{0, 0, 0, 0};
        if constexpr (BITS == 4)
            asum[nt] = *reinterpret_cast<const i32x4 *>(sums + 8 * gi);
        lim[nt] = gr < n ? sq.limit((r0 + gr) / a.group, a.cap) : 0;
        m[nt] = -INFINITY;
        l[nt] = sw[nt] = 0.f;
#pragma unroll
        for (int c = 0; c < CL; c++)
            acc[nt][c] = 0.f;
    }

    for (int b = 0; b < nb; b++) {
        const int tb = t0 + 64 * WV * b + 64 * w;   // the wave's first position
        const uint64_t ok_mask = __builtin_amdgcn_ballot_w64(valid);
        // positions with a norm that is an infinity or NaN make a NaN of the rows
        // that attend to them (step 6), not of others: their values count as zero
        const bool odd = valid && !(fabsf(k.rho) < INFINITY && fabsf(v.rho) < INFINITY);
        const uint64_t odd_mask = __builtin_amdgcn_ballot_w64(odd);
        // 4. the keys' records, chunk kq of key 16 r + col in y[r]
        uint32_t y[4][S::WC];
#pragma unroll
        for (int i = 0; i < S::WC; i++) {
#pragma unroll
            for (int c = 0; c < 4; c++) {
                const int o = c * S::CB + 32 * i, at = o >> 5, sh = o & 31;
                if (at >= S::RW)
                    y[c][i] = 0u;
                else if (sh == 0)
                    y[c][i] = k.w[at];
                else
                    y[c][i] = __builtin_amdgcn_alignbit(at + 1 < S::RW ? k.w[at + 1] : 0u, k.w[at], sh);
            }
            transpose_rows(y[0][i], y[1][i], y[2][i], y[3][i]);
        }
        // the norms, to the lanes of their positions mod 16
        norms[(lane & 15) * 4 + (lane >> 4)] = k.rho;
        norms[64 + (lane & 15) * 4 + (lane >> 4)] = valid && !odd ? v.rho : 0.f;
        // the values' records as they are, for the second product
#pragma unroll
        for (int i = 0; i < H::SW; i += 4)
            *reinterpret_cast<u32x4 *>(mine + lane * H::RS + i) =
                u32x4{H::staged(v.w, i), H::staged(v.w, i + 1), H::staged(v.w, i + 2), H::staged(v.w, i + 3)};
        __builtin_amdgcn_sched_barrier(0);
        if (b + 1 < nb) {
            fetch(b + 1);
        }
        __builtin_amdgcn_sched_barrier(0);
        if (ok_mask == 0)
            continue;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        const f32x4 krho = *reinterpret_cast<const f32x4 *>(norms + 4 * col);
        const f32x4 vrho = *reinterpret_cast<const f32x4 *>(norms + 64 + 4 * col);

        // 5. logits (in units of ln 2) of the lane's row and its four positions
        float val[NT][4];
#pragma unroll
        for (int st = 0; st < 4; st++) {
            i32x4 d[NT][3];
#pragma unroll
            for (int nt = 0; nt < NT; nt++)
#pragma unroll
                for (int t = 0; t < 3; t++)
                    d[nt][t] = asum[nt];
            auto step = [&](auto nsc, int q0) {
                constexpr int NS = decltype(nsc)::value;
                uint32_t sel[NS], inv[NS], p[NS];
                attn_selectors<S, BITS, NS>(y[st], q0, sel);
                if constexpr (BITS == 4) {
#pragma unroll
                    for (int j = 0; j < NS; j++)
                        inv[j] = magnitude(sel[j]);
                }
#pragma unroll
                for (int t = 0; t < 3; t++) {
#pragma unroll
                    for (int j = 0; j < NS; j++) {
                        p[j] = __builtin_amdgcn_perm(a.k_dig.tab[t][1], a.k_dig.tab[t][0], sel[j]);
                        if constexpr (BITS == 4)
                            p[j] ^= inv[j];
                    }
#pragma unroll
                    for (int nt = 0; nt < NT; nt++)
                        d[nt][t] = digit_mfma<NS>(A[nt] + q0, p, d[nt][t]);
                }
            };
#pragma unroll
            for (int q0 = 0; q0 + 4 <= S::NQ; q0 += 4)
                step(std::integral_constant<int, 4>{}, q0);
            if constexpr (S::NQ % 4 != 0) {
#pragma unroll
                for (int nt = 0; nt < NT; nt++)
                    digit_wait(d[nt]);
                step(std::integral_constant<int, 2>{}, S::NQ - 2);
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int nt = 0; nt < NT; nt++) {
                const i32x4 *x = d[nt];
                const int w01 = (x[0][0] << 8) + x[0][1] + x[1][0];
                const int w2 = x[0][2] + x[1][1] + x[2][0];
                const int w3 = x[0][3] + x[1][2] + x[2][1];
                const float f = fmaf((float)w01, 65536.f, fmaf((float)w2, 256.f, (float)w3));
                val[nt][st] = (f * f1[nt]) * (krho[st] * f2[nt]);
            }
        }
        const bool whole = ok_mask == ~0ull && tb + 64 <= lim_min && n == ROWS;   // (uniform)
        if (!whole) {
#pragma unroll
            for (int st = 0; st < 4; st++) {
                const int kk = 16 * st + col;
                const bool ok = (ok_mask >> kk) & 1;
#pragma unroll
                for (int nt = 0; nt < NT; nt++)
                    val[nt][st] = ok && tb + kk < lim[nt] ? val[nt][st] : -INFINITY;
            }
        }
        // 6. running maximum, weights, and their digits to LDS.  The unit of a row's
        //    weights is 2^-30 of the largest of them: norms at positions that it
        //    does not attend to, or with next to no p, leave it its bits
        float alpha[NT], vunit[NT];
#pragma unroll
        for (int nt = 0; nt < NT; nt++) {
            float top = fmaxf(fmaxf(val[nt][0], val[nt][1]), fmaxf(val[nt][2], val[nt][3]));
            top = fmaxf(m[nt], row_max16(top));
            const float ref = top == -INFINITY ? 0.f : top;
            alpha[nt] = __builtin_amdgcn_exp2f(m[nt] - ref);
            m[nt] = top;
            uint32_t u[4];
            float sum = 0.f, wsum = 0.f, weights[4];
#pragma unroll
            for (int st = 0; st < 4; st++) {
                const float p = __builtin_amdgcn_exp2f(val[nt][st] - ref);
                sum += p;
                weights[st] = p * vrho[st];
            }
            const int ve = head_exponent(row_max16(fmaxf(fmaxf(fabsf(weights[0]), fabsf(weights[1])),
                                                         fmaxf(fabsf(weights[2]), fabsf(weights[3])))), 30);
            vunit[nt] = __builtin_amdgcn_ldexpf(a.v_dig.scale, 8 - ve);   // (sums of digits in units of 256)
#pragma unroll
            for (int st = 0; st < 4; st++) {
                // balanced digits: each byte of x + 128 (in the three lower
                // places), less 128
                const float weight = __builtin_rintf(__builtin_amdgcn_ldexpf(weights[st], ve));
                wsum += weight;
                const int x = (int)weight;
                u[st] = ((uint32_t)x + 0x00808080u) ^ 0x00808080u;
            }
            l[nt] = fmaf(l[nt], alpha[nt], sum);
            if (odd_mask != 0 && tb + __builtin_ctzll(odd_mask) < lim[nt])
                l[nt] = NAN;
            if constexpr (BITS == 4)
                sw[nt] = fmaf(wsum, vunit[nt], sw[nt] * alpha[nt]);
            const uint32_t a01 = __builtin_amdgcn_perm(u[1], u[0], 0x05010400u), a23 = __builtin_amdgcn_perm(u[3], u[2], 0x05010400u);
            const uint32_t b01 = __builtin_amdgcn_perm(u[1], u[0], 0x07030602u), b23 = __builtin_amdgcn_perm(u[3], u[2], 0x07030602u);
            uint32_t *dst = wdig + nt * 256 + lane;   // [digit][row][position mod 16]
            dst[0] = __builtin_amdgcn_perm(a23, a01, 0x05040100u);
            dst[64] = __builtin_amdgcn_perm(a23, a01, 0x07060302u);
            dst[128] = __builtin_amdgcn_perm(b23, b01, 0x05040100u);
            dst[192] = __builtin_amdgcn_perm(b23, b01, 0x07060302u);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        uint32_t W[NT][4];
#pragma unroll
        for (int nt = 0; nt < NT; nt++) {
            // A's row col: row col / 4, digit col mod 4 (lowest first); word c: positions 16 i + 4 kq + c
            const u32x4 x = *reinterpret_cast<const u32x4 *>(wdig + nt * 256 + (col & 3) * 64 + (col >> 2) * 16 + 4 * kq);
#pragma unroll
            for (int c = 0; c < 4; c++) {
                const uint32_t e = x[c];
                W[nt][c] = e;
            }
        }
        // 7. sums of values, up to 8 of the lane's coordinates at a time
        auto group = [&](auto nc, int c0) {
            constexpr int N = decltype(nc)::value;
            uint32_t sel[4][N];
#pragma unroll
            for (int c = 0; c < 4; c++) {
                uint32_t x[4];
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    const int at = (16 * i + 4 * kq + c) * H::RS;   // position 16 i + 4 kq + c
                    if constexpr (H::HALF)
                        x[i] = reinterpret_cast<const uint16_t *>(mine + at)[2 * c0 + col];
                    else
                        x[i] = mine[at + 2 * c0 + col];
                }
                position_selectors<BITS, N>(x, sel[c]);
            }
#pragma unroll
            for (int j = 0; j < N; j++) {
                uint32_t inv[4];
                if constexpr (BITS == 4) {
#pragma unroll
                    for (int c = 0; c < 4; c++)
                        inv[c] = magnitude(sel[c][j]);
                }
                i32x4 d[NT][VD];
#pragma unroll
                for (int t = 0; t < VD; t++) {
                    uint32_t p[4];
#pragma unroll
                    for (int c = 0; c < 4; c++)
                        p[c] = __builtin_amdgcn_perm(a.v_dig.tab[t][1], a.v_dig.tab[t][0], sel[c][j]);
                    if constexpr (BITS == 4) {
#pragma unroll
                        for (int c = 0; c < 4; c++)
                            p[c] ^= inv[c];
                    }
#pragma unroll
                    for (int nt = 0; nt < NT; nt++)
                        d[nt][t] = digit_mfma<4>(W[nt], p, i32x4{0, 0, 0, 0});
                }
#pragma unroll
                for (int nt = 0; nt < NT; nt++) {
                    // d[t][r]: level digit t, weight digit r, both lowest first
                    const i32x4 *x = d[nt];
                    float f;
                    if constexpr (VD == 2) {
                        const int hi = (x[1][3] << 8) + x[1][2] + x[0][3];
                        const int lo = ((x[1][1] + x[0][2]) << 8) + x[1][0] + x[0][1];
                        f = fmaf((float)hi, 65536.f, (float)lo);
                    } else {
                        const int hi = (x[2][3] << 8) + x[2][2] + x[1][3];
                        const int lo = ((x[2][1] + x[1][2] + x[0][3]) << 8) + x[2][0] + x[1][1] + x[0][2];
                        f = fmaf((float)hi, 65536.f, (float)lo) * 256.f;
                    }
                    acc[nt][c0 + j] = fmaf(f, vunit[nt], acc[nt][c0 + j] * alpha[nt]);
                }
            }
        };
#pragma unroll
        for (int c0 = 0; c0 + 8 <= CL; c0 += 8)
            group(std::integral_constant<int, 8>{}, c0);
        if constexpr (CL % 8 != 0)
            group(std::integral_constant<int, CL % 8>{}, CL / 8 * 8);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();   // (the next batch's records and digits take this one's place)
    }

    // 8. the waves' m, l and sums, merged through LDS
#pragma unroll
    for (int nt = 0; nt < NT; nt++) {
        float x = l[nt];
        x += dpp_f<DPP_QUAD_1032>(x);
        x += dpp_f<DPP_QUAD_2301>(x);
        x += dpp_f<DPP_ROW_HALF_MIRROR>(x);
        l[nt] = x + dpp_f<DPP_ROW_MIRROR>(x);
        if (nonfinite(mx[8 * (4 * nt + kq)]) && l[nt] != 0.f)
            l[nt] = NAN;   // an infinity or NaN in the rotated query, which no digits hold, and a position
        if constexpr (BITS == 4) {
            // the levels' half offset (build_value_digits), the same for every
            // coordinate; sw is in units of 256
            float y = sw[nt];
            y += dpp_f<DPP_QUAD_1032>(y);
            y += dpp_f<DPP_QUAD_2301>(y);
            y += dpp_f<DPP_ROW_HALF_MIRROR>(y);
            y += dpp_f<DPP_ROW_MIRROR>(y);
            y *= (VD == 2 ? 128.5f : 32896.5f) / 256.f;
#pragma unroll
            for (int c = 0; c < CL; c++)
                acc[nt][c] += y;
        }
    }
    // (and the parts of the rows' prefix, which lie as the lanes' sums do: a wave adds every
    // WV-th.  64 sequences of 8 x 4 heads with 32 parts a row, d = 128: 4.2 us more, a join
    // 9.8)
    if (PRE && sq.folded > 0) {   // (uniform)
        constexpr int U = CL <= 8 ? 4 : CL <= 16 ? 2 : 1;
#pragma unroll
        for (int nt = 0; nt < NT; nt++) {
            const int rr = r0 + min(4 * nt + kq, n - 1), ii = rr / a.group;
            const int64_t at = ((int64_t)(sq.first + ii) * a.n_q_heads + h * a.group + (rr - ii * a.group)) * a.part_splits;
            for (int k0 = w; k0 < sq.folded; k0 += U * WV) {
                float v[U][CL], vm[U], vl[U];
#pragma unroll
                for (int u = 0; u < U; u++) {
                    const int64_t k = at + min(k0 + u * WV, sq.folded - 1);
                    vm[u] = a.part_ml[2 * k];
                    vl[u] = a.part_ml[2 * k + 1];
#pragma unroll
                    for (int c = 0; c < CL; c++)
                        v[u][c] = a.part[k * D + col * CL + c];
                }
#pragma unroll
                for (int u = 0; u < U; u++) {
                    if (k0 + u * WV >= sq.folded)
                        break;
                    const float top = fmaxf(m[nt], vm[u]), ref = top == -INFINITY ? 0.f : top;
                    const float f = __builtin_amdgcn_exp2f(m[nt] - ref), g = __builtin_amdgcn_exp2f(vm[u] - ref);
                    m[nt] = top;
                    l[nt] = fmaf(g, vl[u], l[nt] * f);
#pragma unroll
                    for (int c = 0; c < CL; c++)
                        acc[nt][c] = fmaf(g, v[u][c], acc[nt][c] * f);
                }
            }
        }
    }
    __syncthreads();
    float *part = reinterpret_cast<float *>(smem);          // [WV][ROWS][D]
    float *ml = part + WV * ROWS * D;                       // [WV][ROWS][2]
#pragma unroll
    for (int nt = 0; nt < NT; nt++) {
        const int r = 4 * nt + kq;
#pragma unroll
        for (int c = 0; c < CL; c++)
            part[(w * ROWS + r) * D + col * CL + c] = acc[nt][c];
        if (col == 0) {
            ml[(w * ROWS + r) * 2] = m[nt];
            ml[(w * ROWS + r) * 2 + 1] = l[nt];
        }
    }
    // the lane's 8 coordinates of a row again
    const int r = (64 * w + lane) / (D / 8), j = (64 * w + lane) - r * (D / 8);
    const int i = (r0 + r) / a.group, g = r0 + r - i * a.group;
    const int64_t row = (int64_t)(sq.first + i) * a.n_q_heads + h * a.group + g;
    float top = -INFINITY, sum = 0.f, y[8];
    auto merge = [&] {
#pragma unroll
        for (int x = 0; x < WV; x++)
            top = fmaxf(top, ml[(x * ROWS + r) * 2]);
        const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll
        for (int c = 0; c < 8; c++)
            y[c] = 0.f;
#pragma unroll 4
        for (int x = 0; x < WV; x++) {
            const float f = __builtin_amdgcn_exp2f(ml[(x * ROWS + r) * 2] - ref);
            sum = fmaf(f, ml[(x * ROWS + r) * 2 + 1], sum);
#pragma unroll
            for (int c = 0; c < 8; c++)
                y[c] = fmaf(f, part[(x * ROWS + r) * D + 8 * j + c], y[c]);
        }
    };
    if (a.part && !(PRE && a.fold > 0)) {
        __syncthreads();
        if (r >= n)
            return;
        merge();
        float *dst = a.part + attn_part(a, row, blockIdx.z) * D + 8 * j;
#pragma unroll
        for (int c = 0; c < 8; c++)
            dst[c] = y[c];
        if (j == 0) {
            float *to = a.part_ml + attn_part(a, row, blockIdx.z) * 2;
            to[0] = top;
            to[1] = sum;
        }
        return;
    }
    // (the rotation's parameters are asked for before the waves wait for each other)
    auto finish = [&](auto var) {
        constexpr int VAR = decltype(var)::value;
        constexpr int PL = VAR == VAR_BLOCK8 ? 8 : kLanePL<VAR>;
        const float *par = a.v_params + ((int64_t)(a.v_sets == 1 ? 0 : h) * (D / 8) + j) * kLanePL<VAR>;
        float P[PL];
        if (r < n)
            load_params<PL>(par, P);
        __syncthreads();
        if (r >= n)
            return;
        merge();
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        float o[8];
#pragma unroll
        for (int c = 0; c < 8; c++)
            y[c] *= inv;
        if constexpr (VAR == VAR_BLOCK8) {   // row by row
#pragma unroll
            for (int c = 0; c < 8; c++)
                o[c] = 0.f;
#pragma unroll
            for (int q = 0; q < 8; q++) {
                if (q > 0)
                    load_params<8>(par + 8 * q, P);
#pragma unroll
                for (int c = 0; c < 8; c++)
                    o[c] = fmaf(P[c], y[q], o[c]);
            }
        } else {
            rotate_inverse<VAR>(P, y, o);
        }
        if (a.q_f16)
            store_row_chunk<true>(static_cast<char *>(a.out) + row * D * 2 + j * 16, o);
        else
            store_row_chunk<false>(static_cast<char *>(a.out) + row * D * 4 + j * 32, o);
        if (j == 0 && a.lse)
            a.lse[row] = attn_lse(top, sum);
    };
    switch (a.variant) {
    case VAR_FULL: finish(std::integral_constant<int, VAR_FULL>{}); break;
    case VAR_FAST: finish(std::integral_constant<int, VAR_FAST>{}); break;
    case VAR_PLANAR2D: finish(std::integral_constant<int, VAR_PLANAR2D>{}); break;
    default: finish(std::integral_constant<int, VAR_BLOCK8>{}); break;
    }
}

}  // namespace
}  // namespace isoq
