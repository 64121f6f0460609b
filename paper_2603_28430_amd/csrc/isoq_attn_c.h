// Attention of many rows (chunks of new tokens) over the paged quantized cache:
// fp16 queries, widths up to 128, on the fp16 matrix cores.
//
// isoq_attn_m.h decodes a tile of 64 positions for 4 to 12 rows; with hundreds of
// rows per key head that decoding is what it spends its time on.  Here a
// workgroup has 128 rows (W = 4 waves) or 256 (W = 8), decodes each tile once into
// LDS, and multiplies in fp16 with fp32 sums:
//   logits   the rotated query in two parts, x = hi + lo with hi = fp16(x) and lo
//            = fp16(x - hi), its row in units of a power of two that brings its
//            largest coordinate to 8 .. 16; the levels as fp16 numbers in units
//            for which they lie closest to them (off by 1e-7, 6e-6, 4e-5 of their
//            root mean square at 2, 3, 4 bits).  What that leaves of them is a
//            third product (kRestNone ..): at 3 bits in e4m3 and with the query in
//            e4m3, which rounds it to 2.6%, at 4 bits, and for codebooks that fp16
//            holds as badly, in fp16.  lse is off by 5e-8 to 8e-8 of its norm, as
//            in fp32 products (4 bits without the third product 2e-6 to 3e-6, with it
//            in e4m3 3e-7 to 8e-7, for 318 us instead of 351).
//   values   the weights w = p rho (in units of a power of two next to the row's
//            largest, which is 2^4 .. 2^15) in fp16, the levels as above; what
//            fp16 leaves of the weights is a second product, in e4m3 and with the
//            levels in e4m3: outputs are off by 2.1e-4 to 2.2e-4 of their norm, where
//            rounding them to fp16 alone takes 2.07e-4; without it 2.9e-4 to 3.2e-4.  What
//            fp16 leaves of the values' levels is not multiplied: at 4 bits, whose 2.2e-4 it
//            is, it is 7e-5 of them at most, a third of that rounding.
// An e4m3 product is half a fp16 product's time: with both corrections in fp16, 2 x
// 512 tokens at 8,192 positions, 3 bits, took 6% longer (with the query's lo in e4m3
// too 6% less, and lse off by 1e-6 to 2e-6; both, and 318 / 351 above, with 128 rows).
//
// What bounds it.  Two equal chunks (2 x 512 tokens at 8,192 positions, 8 x 4 heads)
// take 266 us at 3 bits, 500 TFLOP/s of the definition's operations (4 d a row and
// position), twice that of the matrix cores' own, and 280 to 301 once such calls have
// followed each other for some ms and the clock has fallen; 293 to 352 at 4 bits, 243 to
// 289 at 2, 187 to 192 at d = 64.  (128 rows: 307 to 376, 351 to 440, 274, 200.)  256 rows at
// 131,071 positions, 8 heads, take 267 to 306 (128 rows: 335).  Matrix cores are busy for 53%
// of the cycles (128 rows: 42%), vector instructions issue in 53% (50%), waves wait for 25%
// (28%): a tile of 64 positions takes the two waves of a SIMD 7,500 cycles, of which vector
// instructions issue in 6,350 and matrix products in 4,096 (measured one by one).  Ragged
// chunks of up to 512 tokens are bound by what unequal sequences leave idle as well (38%,
// 43%, 29%), short contexts by 8 us of preparation (the queries' rotation, a chain of loads)
// and 3 of storing the parts, before and after tiles of 3 us each.
//
// 256 rows.  A tile's decoding serves twice the rows, and a SIMD's two waves do
// different things at a time: tiles are decoded one ahead, into the other of two
// buffers, by the first four waves (values) after they have attended to the present
// one, by the next four (keys) before.  (Keys and values read two tiles ahead, a third
// wave to fetch, wave priorities, all waves decoding at once: no faster.)
//
// Layout (v_mfma_f32_32x32x16_f16).  S^T = K Q^T: a wave has 32 rows as columns,
// lane 32 h + n the row n and the positions 8 b + 4 h + i (b, i = 0 .. 3) of each
// 32: a row's maximum and sum are in-lane but for one exchange of halves, and
// the fp16 weights are B of O^T = V^T P^T as they stand, if V^T's positions
// are in the same order: [16 s][h][b][i].  K rows and V^T rows lie in LDS with
// 16 bytes of padding (reads of 16 bytes by 16 rows touch every bank once).
//
// Decoding.  Wave c (of four) spreads chunk c (a quarter of the coordinates) of 64 keys;
// values are decoded four positions at a time (position_selectors), which
// gives V^T's rows directly.  A level's two bytes are two v_perm_b32 for four
// coordinates, two more put them together.  Two waves fetch the records of a later
// tile (K, V) while all compute.
#pragma once

#include "isoq_attn_m.h"

namespace isoq {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

template <int D, int BITS, int REST, int W>
struct AttnCShape {
    using S = ScoreMShape<D, BITS, 0>;
    using H = AttnMShape<D, BITS, 1>;
    static constexpr int ROWS = 32 * W;              // a wave has 32
    static constexpr bool AHEAD = W > 4;             // tiles are decoded one ahead, into the other of two buffers
    static constexpr int KS = S::NQ;                 // 16-coordinate steps of the logits' product (4 chunks of 4 NQ)
    static constexpr int KROW = 32 * KS + 16;        // bytes of a decoded key part
    static constexpr int K8 = (KS + 3) / 4;          // 64-coordinate steps of its correction
    static constexpr int KROWR = REST == kRestBytes ? 64 * K8 + 16 : REST == kRestHalves ? KROW : 0;   // bytes of what fp16 left of a key's levels
    static constexpr int CT = (D + 31) / 32;         // 32-coordinate tiles of the values
    static constexpr int VROW = 2 * 64 + 16;         // bytes of a coordinate's 64 positions
    static constexpr int VROW8 = 64 + 16;            // and in e4m3
    static constexpr int RK = 4 * S::WC + 1;         // words of a key's raw record (odd: lanes are keys)
    static constexpr int RV = H::SW + 1;             // words of a value's raw record
    // LDS bytes: keys, and what fp16 left of them; values in fp16, e4m3 (two
    // buffers of these with AHEAD); raw records (two); of 2 or 4 tiles the norms (K,
    // V), the valid positions, the values' unit and half of their least norm in it,
    // and the first key and value whose norm is an infinity or NaN
    static constexpr int NB = AHEAD ? 2 : 1, NT = AHEAD ? 4 : 2;
    static constexpr int kHalf = 0, kRest = 64 * KROW, kV = kRest + 64 * KROWR, kV8 = kV + 32 * CT * VROW,
                         kBuffer = kV8 + 32 * CT * VROW8;
    static constexpr int kRawK = NB * kBuffer, kRawV = kRawK + 4 * 64 * RK, kRaw = 4 * 64 * (RK + RV),
                         kNorm = kRawK + NB * kRaw, kTile = kNorm + NT * 512;
    static constexpr int loop_bytes() { return kTile + NT * 32; }
    // before the loop the rotated queries, in the keys' order of coordinates (reads of
    // 16 bytes by consecutive rows touch every bank once)
    static constexpr int QS = 16 * KS + 4;
    static constexpr int query_bytes() { return 4 * ROWS * QS; }
    static constexpr int lds_bytes() { return loop_bytes() > query_bytes() ? loop_bytes() : query_bytes(); }
    static_assert(kRest % 16 == 0 && kV % 16 == 0 && kV8 % 16 == 0 && kBuffer % 16 == 0 && kRaw % 16 == 0, "aligned parts");
    static_assert(lds_bytes() <= 160 * 1024, "a compute unit's LDS");

    // place of coordinate e of a row in that order: quad q of chunk c and byte b of it (attn_coord)
    static __device__ __forceinline__ int place(int e)
    {
        const int c = e / S::CC, ci = e - c * S::CC;
        int q, b;
        if (BITS == 3 && 32 * (ci / 32 + 1) <= S::CC) {
            q = ci / 32 * 8 + ci % 8;
            b = ci % 32 / 8;
        } else if (BITS == 2 && 16 * (ci / 16 + 1) <= S::CC) {
            q = ci / 16 * 4 + ci % 4;
            b = ci % 16 / 4;
        } else {
            q = ci / 8 * 2 + ci % 2;
            b = ci % 8 / 2;
        }
        return 4 * (c * S::NQ + q) + b;
    }
};

// The workgroup's n query rows from r0 on, rotated (scale folded in), into qt.  A
// thread keeps its chunk of 8 coordinates, whose parameters and places it has once,
// and asks for four rows at a time.
template <int VAR, class C, int D, int THREADS>
__device__ __forceinline__ void attn_c_queries(const AttnArgs &a, const AttnSeq &sq, int h, int r0, int n, float *qt)
{
    constexpr int NCH = D / 8, PER = THREADS / NCH, PL = kLanePL<VAR>, U = 4;
    const int c = threadIdx.x % NCH, first = threadIdx.x / NCH;
    if (first >= PER)
        return;
    float P[PL];
    load_params<PL>(a.k_params + ((int64_t)(a.k_sets == 1 ? 0 : h) * NCH + c) * PL, P);
    int at[8];
#pragma unroll
    for (int k = 0; k < 8; k++)
        at[k] = C::place(8 * c + k);
    for (int q = first; q < n; q += U * PER) {
        Raw<true> raw[U];
#pragma unroll
        for (int u = 0; u < U; u++) {
            const int r = r0 + min(q + u * PER, n - 1), i = r / a.group;
            const int64_t row = (int64_t)(sq.first + i) * a.n_q_heads + h * a.group + (r - i * a.group);
            load_row_chunk<true>(static_cast<const char *>(a.q) + row * D * 2 + c * 16, raw[u]);
        }
#pragma unroll
        for (int u = 0; u < U; u++) {
            float x[8], y[8];
            unpack<true>(raw[u], x);
            if constexpr (VAR == VAR_BLOCK8) {
#pragma unroll
                for (int e = 0; e < 8; e++) {
                    y[e] = P[8 * e] * x[0];
#pragma unroll
                    for (int k = 1; k < 8; k++)
                        y[e] = fmaf(P[8 * e + k], x[k], y[e]);
                }
            } else {
                rotate_forward<VAR>(P, x, y);
            }
            if (q + u * PER < n) {
                float *dst = qt + (q + u * PER) * C::QS;
#pragma unroll
                for (int k = 0; k < 8; k++)
                    dst[at[k]] = y[k] * a.scale;
            }
        }
    }
}

// Four levels' fp16 values for four selector bytes: tables of the values' low
// and high bytes (4 bits: of the positive levels', whose sign bit is set where
// `inv` says that the index is below 8).
template <int BITS>
__device__ __forceinline__ void level_halves(const uint32_t lo[2], const uint32_t hi[2], uint32_t sel, uint32_t inv,
                                             uint32_t out[2])
{
    const uint32_t l = __builtin_amdgcn_perm(lo[1], lo[0], sel);
    uint32_t h = __builtin_amdgcn_perm(hi[1], hi[0], sel);
    if constexpr (BITS == 4)
        h = __builtin_amdgcn_bitop3_b32(h, inv, vector_const(0x80808080u), 0x78);   // h ^ (inv & 0x80)
    out[0] = __builtin_amdgcn_perm(h, l, 0x05010400u);
    out[1] = __builtin_amdgcn_perm(h, l, 0x07030602u);
}

// Four levels' e4m3 values likewise.
template <int BITS>
__device__ __forceinline__ uint32_t level_bytes(const uint32_t tab[2], uint32_t sel, uint32_t inv)
{
    const uint32_t x = __builtin_amdgcn_perm(tab[1], tab[0], sel);
    return BITS < 4 ? x : __builtin_amdgcn_bitop3_b32(x, inv, vector_const(0x80808080u), 0x78);   // x ^ (inv & 0x80)
}

// C + 2^exp A B^T, 32 x 32 x 64, e4m3
__device__ __forceinline__ f32x16 mfma_bytes(i32x8 a, i32x8 b, f32x16 c, int exp)
{
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, c, 0, 0, 0, 127 + exp, 0, 127);
}

__device__ __forceinline__ i32x8 read_bytes32(const uint8_t *src)
{
    const u32x4 x = *reinterpret_cast<const u32x4 *>(src), y = *reinterpret_cast<const u32x4 *>(src + 16);
    return i32x8{(int)x[0], (int)x[1], (int)x[2], (int)x[3], (int)y[0], (int)y[1], (int)y[2], (int)y[3]};
}

__device__ __forceinline__ f16x8 as_halves(u32x4 v) { return __builtin_bit_cast(f16x8, v); }

// (Up to d = 64 the registers allow three workgroups a compute unit, at 4 bits with
// three of them spilled: 61 us instead of 71 for three ragged chunks of up to 300
// tokens and 6,000 positions, 8 x 2 heads.)
template <int D, int BITS, int REST, int W>
__global__ __launch_bounds__(64 * W, W > 4 ? W / 4 : D <= 64 ? 3 : 2) void attn_c_kernel(const AttnArgs a)
{
    using C = AttnCShape<D, BITS, REST, W>;
    using S = typename C::S;
    using H = typename C::H;
    constexpr int64_t RB = (int64_t)D * BITS / 8;
    extern __shared__ __align__(16) uint32_t smem[];
    uint8_t *const lds = reinterpret_cast<uint8_t *>(smem);

    // (the sequences' first row tiles are not the same places of the grid: where most have no
    // others, as single tokens next to a chunk, every 64th workgroup had work, and they went to
    // one of an XCD's four shader engines, 15 such sequences and one of 512 tokens, 8 x 4 heads,
    // 8,192 positions 1,062 us)
    const uint32_t tiles = gridDim.x / (uint32_t)a.n_kv_heads;
    const int hx = (int)(blockIdx.x % (uint32_t)a.n_kv_heads);
    const int rt = (int)((blockIdx.x / (uint32_t)a.n_kv_heads + blockIdx.y + blockIdx.z) % tiles);
    const int h = (int)xcd_head((uint32_t)hx, (uint32_t)a.n_kv_heads, a.block_size * RB % 128 != 0);
    const int s = blockIdx.y;
    const int lane = threadIdx.x & 63, n32 = lane & 31, half = lane >> 5;
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const AttnSeq sq = attn_seq<false>(a, s);
    const int r0 = rt * C::ROWS, total = sq.rows * a.group;
    if (r0 >= total)   // (block-uniform, as every early return here)
        return;
    const int n = min(C::ROWS, total - r0);
    const int lim_all = sq.limit((r0 + n - 1) / a.group, a.cap);
    const int chunk = attn_chunk(a, sq);
    const int64_t t0l = (int64_t)blockIdx.z * chunk;
    if (t0l >= lim_all && blockIdx.z > 0)
        return;   // the join looks at the splits below a row's limit only
    const int t0 = (int)t0l, tend = (int)min(t0l + chunk, (int64_t)lim_all);
    const int nt = (tend - t0 + 63) / 64;

    // the wave's rows: one per lane of each half
    const int r = 32 * w + n32;
    const bool on = r < n;
    const int tok = (r0 + (on ? r : 0)) / a.group;
    const int lim = on ? sq.limit(tok, a.cap) : 0;
    const int64_t row = (int64_t)(sq.first + tok) * a.n_q_heads + h * a.group + (r0 + (on ? r : 0) - tok * a.group);
    // (rows in the tokens' order) the least of the wave's limits
    const int lim_min = 32 * w + 32 <= n ? sq.limit((r0 + 32 * w) / a.group, a.cap) : 0;
    const int lim_max = 32 * w < n ? sq.limit((r0 + min(32 * w + 31, n - 1)) / a.group, a.cap) : 0;

    // 0. records of the next tile: waves WK (K) and WV (V), a position per lane
    constexpr int WK = W > 4 ? 1 : 0, WV = W > 4 ? 2 : 1;
    const bool fetches = w == WK || w == WV;
    const int32_t *table = a.block_table + (int64_t)s * a.max_blocks;
    const uint64_t rstride = (uint64_t)a.n_kv_heads * a.block_size, row0 = (uint64_t)h * a.block_size;
    const uint64_t bstride = rstride * RB;
    const uint8_t *const idx = (w == WK ? a.k_idx : a.v_idx) + row0 * RB;
    const float *const rhos = (w == WK ? a.k_rho : a.v_rho) + row0;
    const int64_t pstep = (int64_t)a.block_size * S::CP;
    struct Batch {
        uint32_t w[S::RW];
        float rho;
        bool ok;
    } rec{};
    auto block_of = [&](int t) {   // the block-table entry of the lane's position of tile t
        const uint32_t tt = (uint32_t)min((int64_t)t0 + 64 * (int64_t)t + lane, (int64_t)tend - 1);
        return table[fast_div(tt, a.div_block)];
    };
    auto fetch = [&](int t, int32_t blk) {
        const int64_t tl = (int64_t)t0 + 64 * (int64_t)t + lane;
        const uint32_t tt = (uint32_t)min(tl, (int64_t)tend - 1);
        rec.ok = tl < tend && blk >= 0 && blk < a.n_blocks;
        // (an invalid position reads position 0 of the head in block 0, which is always present)
        const uint64_t b = rec.ok ? (uint32_t)blk : 0u;
        const uint32_t pos = rec.ok ? tt - fast_div(tt, a.div_block) * a.block_size : 0u;
        const uint8_t *src = idx + b * bstride + (uint64_t)pos * S::CP;
        const uint64_t crow = b * rstride + pos;
        rec.rho = rhos[crow];
        if constexpr (S::LW == 4) {
#pragma unroll
            for (int v = 0; v < S::RW / 4; v++) {
                const u32x4 q4 = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(src + v * pstep));
#pragma unroll
                for (int c = 0; c < 4; c++) {
                    const uint32_t e = q4[c];
                    rec.w[4 * v + c] = e;
                }
            }
        } else if constexpr (S::LW == 2) {
#pragma unroll
            for (int v = 0; v < S::RW / 2; v++) {
                const u32x2 q2 = __builtin_nontemporal_load(reinterpret_cast<const u32x2 *>(src + v * pstep));
                const uint32_t e0 = q2[0], e1 = q2[1];
                rec.w[2 * v] = e0;
                rec.w[2 * v + 1] = e1;
            }
        } else if constexpr (S::LW == 1) {
#pragma unroll
            for (int v = 0; v < S::RW; v++)
                rec.w[v] = reinterpret_cast<const uint32_t *>(src)[v];
        } else {
            // an odd number of half-words, stored whole (isoq_scores_m.h)
            const bool odd = (row0 + crow) & 1;
            const uint32_t *al = reinterpret_cast<const uint32_t *>(src + (odd ? 2 : 0));
            const uint32_t hw = *reinterpret_cast<const uint16_t *>(src + (odd ? 0 : RB - 2));
            uint32_t x[S::RW - 1];
#pragma unroll
            for (int v = 0; v < S::RW - 1; v++)
                x[v] = al[v];
            rec.w[0] = odd ? (x[0] << 16) | hw : x[0];
#pragma unroll
            for (int v = 1; v < S::RW - 1; v++)
                rec.w[v] = odd ? __builtin_amdgcn_alignbit(x[v], x[v - 1], 16) : x[v];
            rec.w[S::RW - 1] = odd ? x[S::RW - 2] >> 16 : hw;
        }
    };
    // the tiles' unit of values: norms below 2^tile_unit; kept while the tile's
    // largest norm is above 2^(tile_unit - 4)
    int tile_unit = 0;
    auto store_raw = [&](int t) {   // (waves WK and WV) into tile t's places
        float *norm = reinterpret_cast<float *>(lds + C::kNorm + 512 * (t & (C::NT - 1)));
        uint32_t *tile = reinterpret_cast<uint32_t *>(lds + C::kTile + 32 * (t & (C::NT - 1)));
        const int raw = C::kRaw * (t & (C::NB - 1));
        if (w == WK) {
            uint32_t *dst = reinterpret_cast<uint32_t *>(lds + C::kRawK + raw) + lane * C::RK;
#pragma unroll
            for (int c = 0; c < 4; c++)
#pragma unroll
                for (int i = 0; i < S::WC; i++) {
                    const int o = c * S::CB + 32 * i, at = o >> 5, sh = o & 31;
                    dst[c * S::WC + i] = at >= S::RW ? 0u
                                         : sh == 0   ? rec.w[at]
                                                     : __builtin_amdgcn_alignbit(at + 1 < S::RW ? rec.w[at + 1] : 0u, rec.w[at], sh);
                }
            norm[lane] = rec.ok ? rec.rho : 0.f;
            const uint64_t odds = __builtin_amdgcn_ballot_w64(rec.ok && !(fabsf(rec.rho) < INFINITY));
            const uint64_t ok = __builtin_amdgcn_ballot_w64(rec.ok);
            if (lane == 0) {
                tile[0] = (uint32_t)ok;
                tile[1] = (uint32_t)(ok >> 32);
                tile[4] = odds ? __builtin_ctzll(odds) : 0x7FFFFFFF;
            }
        } else {
            uint32_t *dst = reinterpret_cast<uint32_t *>(lds + C::kRawV + raw) + lane * C::RV;
#pragma unroll
            for (int i = 0; i < H::SW; i++)
                dst[i] = H::staged(rec.w, i);
            // (norms that are an infinity or NaN make a NaN of the rows that attend to
            // them in step 4, not of others: the values count as zero)
            const bool odd = rec.ok && !(fabsf(rec.rho) < INFINITY);
            const uint64_t odds = __builtin_amdgcn_ballot_w64(odd);
            if (odd)
                rec.rho = 0.f;
            float top = row_max16(rec.ok ? fabsf(rec.rho) : 0.f), least = row_max16(rec.ok ? -fabsf(rec.rho) : -INFINITY);
#pragma unroll
            for (int half = 0; half < 2; half++)   // over the rows of 16 lanes
#pragma unroll
                for (float *v : {&top, &least}) {
                    const uint32_t b = __float_as_uint(*v);
                    const auto x = half == 0 ? __builtin_amdgcn_permlane16_swap(b, b, false, false)
                                             : __builtin_amdgcn_permlane32_swap(b, b, false, false);
                    *v = fmaxf(__uint_as_float(x[0]), __uint_as_float(x[1]));
                }
            const int e = __builtin_amdgcn_readfirstlane(top > 0.f ? __builtin_amdgcn_frexp_expf(top) : tile_unit);
            if (t == 0 || e > tile_unit || e < tile_unit - 4)
                tile_unit = e;
            norm[64 + lane] = rec.ok ? __builtin_amdgcn_ldexpf(rec.rho, 14 - tile_unit) : 0.f;
            if (lane == 0) {
                tile[2] = (uint32_t)tile_unit;
                tile[5] = odds ? __builtin_ctzll(odds) : 0x7FFFFFFF;
                tile[3] = __float_as_uint(__builtin_amdgcn_ldexpf(-least, 13 - tile_unit));
            }
        }
    };
    int32_t next = 0;
    if (nt > 0 && fetches) {
        fetch(0, block_of(0));
        next = block_of(1);
    }

    // 1. rotated queries, and the wave's rows of them as fp16 pairs in registers
    float *qt = reinterpret_cast<float *>(smem);
    if (4 * S::NQ > S::CC) {   // places past a chunk's coordinates
        constexpr int pad = 4 * S::NQ - S::CC;
        // (the rows' zeros first: a chunk's last places are not the last of its quads)
        for (int i = threadIdx.x; i < C::ROWS * C::QS; i += 64 * W)
            qt[i] = 0.f;
        static_assert(pad >= 0, "");
        __syncthreads();
    }
    switch (a.variant) {   // (uniform)
    case VAR_FULL: attn_c_queries<VAR_FULL, C, D, 64 * W>(a, sq, h, r0, n, qt); break;
    case VAR_FAST: attn_c_queries<VAR_FAST, C, D, 64 * W>(a, sq, h, r0, n, qt); break;
    case VAR_PLANAR2D: attn_c_queries<VAR_PLANAR2D, C, D, 64 * W>(a, sq, h, r0, n, qt); break;
    default: attn_c_queries<VAR_BLOCK8, C, D, 64 * W>(a, sq, h, r0, n, qt); break;
    }
    __syncthreads();
    // the lane's places, 16 st + 8 half + 0 .. 7, and the row's largest magnitude (an
    // infinity or NaN among them) of both lanes'
    const float *mine = qt + r * C::QS;
    f32x4 qv[C::KS][2];
    uint32_t qmax = 0;
#pragma unroll
    for (int st = 0; st < C::KS; st++)
#pragma unroll
        for (int e = 0; e < 2; e++) {
            qv[st][e] = *reinterpret_cast<const f32x4 *>(mine + 16 * st + 8 * half + 4 * e);
#pragma unroll
            for (int k = 0; k < 4; k++)
                qmax = max(qmax, __float_as_uint(fabsf(qv[st][e][k])));
        }
    {
        const auto x = __builtin_amdgcn_permlane32_swap(qmax, qmax, false, false);
        qmax = on ? max(x[0], x[1]) : 0u;
    }
    const int qe = head_exponent(__uint_as_float(qmax), 4);
    const bool counts = on && !nonfinite(qmax);
    auto scaled = [&](float x) { return counts ? __builtin_amdgcn_ldexpf(x, qe) : 0.f; };   // in the row's units
    u32x4 qh[C::KS], ql[C::KS];   // B of 16 places: 8 half + 0 .. 7
    [[maybe_unused]] i32x8 q8[C::K8];   // in e4m3, of 64 places: 32 half + 0 .. 31
#pragma unroll
    for (int st = 0; st < C::KS; st++) {
        f16x8 hi, lo;
#pragma unroll
        for (int e = 0; e < 8; e++) {
            const float v = scaled(qv[st][e / 4][e % 4]);
            hi[e] = (_Float16)v;
            lo[e] = (_Float16)(v - (float)hi[e]);
        }
        qh[st] = __builtin_bit_cast(u32x4, hi);
        ql[st] = __builtin_bit_cast(u32x4, lo);
    }
    if constexpr (REST == kRestBytes) {
#pragma unroll
        for (int st = 0; st < C::K8; st++)
#pragma unroll
            for (int e = 0; e < 8; e++) {
                f32x4 x{0.f, 0.f, 0.f, 0.f};
                if (16 * st + 8 * half < 4 * C::KS)   // (whole groups of 8 quads)
                    x = *reinterpret_cast<const f32x4 *>(mine + 64 * st + 32 * half + 4 * e);
                q8[st][e] = __builtin_amdgcn_cvt_pk_fp8_f32(
                    scaled(x[2]), scaled(x[3]), __builtin_amdgcn_cvt_pk_fp8_f32(scaled(x[0]), scaled(x[1]), 0, false), true);
            }
    }
    // a logit (in units of ln 2) is f1 times sum and norm
    const float f1 = fmaxf(__builtin_amdgcn_ldexpf(a.k_half.scale, -qe), 0x1p-126f);
    __syncthreads();   // (the loop's parts take the queries' place)

    f32x16 acc[C::CT];
#pragma unroll
    for (int c = 0; c < C::CT; c++)
#pragma unroll
        for (int e = 0; e < 16; e++)
            acc[c][e] = 0.f;
    // the row: exponentials are relative to 2^ref, an integer next to the running
    // maximum; acc is in units of 2^(unit - 14), in which the largest weight so far is
    // `most` or up to 2^11 more
    float ref = -INFINITY, l = 0.f, most = 0.f;
    int unit = 0;
    for (int b = 0; b < C::NB; b++) {
        uint8_t *buf = lds + b * C::kBuffer;
        if (D % 32 != 0) {   // coordinates past D: rows of zeros
            for (int i = threadIdx.x; i < (32 * C::CT - D) * C::VROW / 4; i += 64 * W)
                reinterpret_cast<uint32_t *>(buf + C::kV + D * C::VROW)[i] = 0u;
            for (int i = threadIdx.x; i < (32 * C::CT - D) * C::VROW8 / 4; i += 64 * W)
                reinterpret_cast<uint32_t *>(buf + C::kV8 + D * C::VROW8)[i] = 0u;
        }
        if (REST == kRestBytes && C::KS % 4 != 0) {   // places past the keys'
            constexpr int words = (64 * C::K8 - 16 * C::KS) / 4;
            for (int i = threadIdx.x; i < 64 * words; i += 64 * W)
                reinterpret_cast<uint32_t *>(buf + C::kRest + (i / words) * C::KROWR + 16 * C::KS)[i % words] = 0u;
        }
    }

    // 2. decode tile t into its buffer: four waves its keys, a chunk of the
    //    coordinates each, four waves (the same ones, or the next) its values
    const int part4 = w & 3;
    auto decode_keys = [&](int t) {
        const uint32_t *src = reinterpret_cast<const uint32_t *>(lds + C::kRawK + C::kRaw * (t & (C::NB - 1))) + lane * C::RK + part4 * S::WC;
        uint32_t y[S::WC];
#pragma unroll
        for (int i = 0; i < S::WC; i++)
            y[i] = src[i];
        uint8_t *buf = lds + C::kBuffer * (t & (C::NB - 1));
        uint8_t *dst = buf + C::kHalf + lane * C::KROW + part4 * 8 * S::NQ;
        uint8_t *rest = buf + C::kRest + lane * C::KROWR + part4 * (REST == kRestHalves ? 8 : 4) * S::NQ;
        auto part = [&](auto nsc, int q0) {
            constexpr int NS = decltype(nsc)::value;
            uint32_t sel[NS];
            [[maybe_unused]] uint32_t lo[NS];
            attn_selectors<S, BITS, NS>(y, q0, sel);
#pragma unroll
            for (int j = 0; j < NS; j += 2) {
                uint32_t x[4];
                [[maybe_unused]] uint32_t y[4];
#pragma unroll
                for (int k = 0; k < 2; k++) {
                    const uint32_t inv = BITS == 4 ? magnitude(sel[j + k]) : 0u;
                    level_halves<BITS>(a.k_half.tab[0], a.k_half.tab[1], sel[j + k], inv, x + 2 * k);
                    if constexpr (REST == kRestHalves)
                        level_halves<BITS>(a.k_half.tab[4], a.k_half.tab[5], sel[j + k], inv, y + 2 * k);
                    if constexpr (REST == kRestBytes)
                        lo[j + k] = level_bytes<BITS>(a.k_half.tab[3], sel[j + k], inv);
                }
                *reinterpret_cast<u32x4 *>(dst + 8 * (q0 + j)) = u32x4{x[0], x[1], x[2], x[3]};
                if constexpr (REST == kRestHalves)
                    *reinterpret_cast<u32x4 *>(rest + 8 * (q0 + j)) = u32x4{y[0], y[1], y[2], y[3]};
            }
            if constexpr (REST == kRestBytes && S::NQ % 4 == 0) {
                *reinterpret_cast<u32x4 *>(rest + 4 * q0) = u32x4{lo[0], lo[1], lo[2], lo[3]};
            } else if constexpr (REST == kRestBytes) {
#pragma unroll
                for (int j = 0; j < NS; j += 2)
                    *reinterpret_cast<u32x2 *>(rest + 4 * (q0 + j)) = u32x2{lo[j], lo[j + 1]};
            }
        };
#pragma unroll
        for (int q0 = 0; q0 + 4 <= S::NQ; q0 += 4)
            part(std::integral_constant<int, 4>{}, q0);
        if constexpr (S::NQ % 4 != 0)
            part(std::integral_constant<int, 2>{}, S::NQ - 2);
    };
    auto decode_values = [&](int t) {
        // lane word 4 part4 + lane / 16 of the positions 4 p .. 4 p + 3, p = lane mod 16
        const int p = lane & 15, v = 4 * part4 + (lane >> 4);
        const uint32_t *raw = reinterpret_cast<const uint32_t *>(lds + C::kRawV + C::kRaw * (t & (C::NB - 1))) + 4 * p * C::RV;
        uint8_t *buf = lds + C::kBuffer * (t & (C::NB - 1));
        // place of the positions 16 s + 8 b + 4 h in a row: [16 s][h][b]
        uint8_t *dst = buf + C::kV + v * H::CL * C::VROW + 2 * (16 * (p >> 2) + 8 * (p & 1) + 4 * ((p >> 1) & 1));
        // in e4m3, of the positions 32 k + 8 b + 4 h: [h][k][b]
        uint8_t *dst8 = buf + C::kV8 + v * H::CL * C::VROW8 + 32 * (p & 1) + 16 * (p >> 3) + 4 * ((p >> 1) & 3);
        auto part = [&](auto nc, int c0) {
            constexpr int N = decltype(nc)::value;
            uint32_t x[4], sel[N];
#pragma unroll
            for (int i = 0; i < 4; i++) {
                if constexpr (H::HALF)
                    x[i] = reinterpret_cast<const uint16_t *>(raw + i * C::RV)[2 * c0 + v];
                else
                    x[i] = raw[i * C::RV + 2 * c0 + v];
            }
            position_selectors<BITS, N>(x, sel);
#pragma unroll
            for (int c = 0; c < N; c++) {
                const uint32_t inv = BITS == 4 ? magnitude(sel[c]) : 0u;
                uint32_t o[2];
                level_halves<BITS>(a.v_half.tab[0], a.v_half.tab[1], sel[c], inv, o);
                *reinterpret_cast<u32x2 *>(dst + (c0 + c) * C::VROW) = u32x2{o[0], o[1]};
                *reinterpret_cast<uint32_t *>(dst8 + (c0 + c) * C::VROW8) = level_bytes<BITS>(a.v_half.tab[2], sel[c], inv);
            }
        };
#pragma unroll
        for (int c0 = 0; c0 + 8 <= H::CL; c0 += 8)
            part(std::integral_constant<int, 8>{}, c0);
        if constexpr (H::CL % 8 != 0)
            part(std::integral_constant<int, H::CL % 8>{}, H::CL / 8 * 8);
    };
    auto attend = [&](int t) {
        const int tb = t0 + 64 * t;
        const uint8_t *buf = lds + C::kBuffer * (t & (C::NB - 1));
        const uint32_t *tile = reinterpret_cast<const uint32_t *>(lds + C::kTile + 32 * (t & (C::NT - 1)));
        if (tb < lim_max) {   // (wave-uniform)
            // 3. S^T of the wave's rows and the tile's positions; a step's keys
            //    are read while the one before multiplies
            f32x16 st[2];
#pragma unroll
            for (int k = 0; k < 2; k++)
#pragma unroll
                for (int e = 0; e < 16; e++)
                    st[k][e] = 0.f;
            const uint8_t *key = buf + C::kHalf + n32 * C::KROW + 16 * half;
            const uint8_t *rest = buf + C::kRest + n32 * C::KROWR + (REST == kRestHalves ? 16 : 32) * half;
            u32x4 kh[2][2];
            [[maybe_unused]] u32x4 kr[2][2];
            auto read_keys = [&](int ks) {
#pragma unroll
                for (int k = 0; k < 2; k++) {
                    kh[ks & 1][k] = *reinterpret_cast<const u32x4 *>(key + 32 * k * C::KROW + 32 * ks);
                    if constexpr (REST == kRestHalves)
                        kr[ks & 1][k] = *reinterpret_cast<const u32x4 *>(rest + 32 * k * C::KROW + 32 * ks);
                }
            };
            if constexpr (REST == kRestBytes) {
                i32x8 lo[2];
                lo[0] = read_bytes32(rest);
#pragma unroll
                for (int i = 0; i < 2 * C::K8; i++) {   // step i / 2, positions 32 (i mod 2) ..
                    if (i + 1 < 2 * C::K8)
                        lo[(i + 1) & 1] = read_bytes32(rest + 32 * ((i + 1) & 1) * C::KROWR + 64 * ((i + 1) / 2));
                    else
                        read_keys(0);
                    __builtin_amdgcn_sched_barrier(0);
                    st[i & 1] = mfma_bytes(lo[i & 1], q8[i / 2], st[i & 1], -kLevelRest);
                    __builtin_amdgcn_sched_barrier(0);
                }
            } else {
                read_keys(0);
            }
#pragma unroll
            for (int ks = 0; ks < C::KS; ks++) {
                if (ks + 1 < C::KS)
                    read_keys(ks + 1);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int k = 0; k < 2; k++)
                    st[k] = __builtin_amdgcn_mfma_f32_32x32x16_f16(as_halves(kh[ks & 1][k]), as_halves(ql[ks]), st[k], 0, 0, 0);
#pragma unroll
                for (int k = 0; k < 2 && REST == kRestHalves; k++)
                    st[k] = __builtin_amdgcn_mfma_f32_32x32x16_f16(as_halves(kr[ks & 1][k]), as_halves(qh[ks]), st[k], 0, 0, 0);
#pragma unroll
                for (int k = 0; k < 2; k++)
                    st[k] = __builtin_amdgcn_mfma_f32_32x32x16_f16(as_halves(kh[ks & 1][k]), as_halves(qh[ks]), st[k], 0, 0, 0);
                __builtin_amdgcn_sched_barrier(0);
            }
            // 4. running maximum (in units of 1 / f1) and weights, in the tile's unit.
            //    Exponentials are 2^(logit - ref), ref an integer, so that rescalings
            //    are exact.  Where the row's largest weight so far would lie below 2^4
            //    or above 2^15 there, the row gets a unit of its own that brings it to
            //    2^13 .. 2^14, so norms at positions that the row does not attend to, or
            //    with next to no weight, cost it no bits, and a unit that falls cannot
            //    overflow its sums.  Rare: a tile that raises ref has a weight of half
            //    of its least norm at least.  (8 prompts of 1,024 tokens whose first
            //    position takes most of half of the rows' weight: 264 us with a value
            //    as large as the others or 1/50 of them, 291 with 1/500, where such
            //    rows keep a unit of their own; 2^4 holds the weight that makes the
            //    row to 2^-14 with its rest in e4m3.)
            const float *norm = reinterpret_cast<const float *>(lds + C::kNorm + 512 * (t & (C::NT - 1))) + 4 * half;
            const u32x4 about = *reinterpret_cast<const u32x4 *>(tile);
            const uint32_t ok0 = about[0], ok1 = about[1];
            const int tu = (int)about[2], half_least = (int)about[3];
            const bool whole = (ok0 & ok1) == ~0u && tb + 64 <= lim_min;
#pragma unroll
            for (int k = 0; k < 2; k++)
#pragma unroll
                for (int b = 0; b < 4; b++) {
                    const f32x4 x = *reinterpret_cast<const f32x4 *>(norm + 32 * k + 8 * b);
#pragma unroll
                    for (int i = 0; i < 4; i++)
                        st[k][4 * b + i] *= x[i];
                }
            if (!whole) {
                // the lane's positions are 32 k + 8 b + i, 4 half further
                const int left = lim - tb - 4 * half;
                const uint32_t mask[2] = {ok0 >> (4 * half), ok1 >> (4 * half)};
#pragma unroll
                for (int k = 0; k < 2; k++)
#pragma unroll
                    for (int e = 0; e < 16; e++) {
                        const int pos = 8 * (e / 4) + e % 4;
                        if (!(mask[k] & (1u << pos)) || left <= 32 * k + pos)
                            st[k][e] = -INFINITY;
                    }
            }
            float top = -INFINITY;
#pragma unroll
            for (int k = 0; k < 2; k++)
#pragma unroll
                for (int e = 0; e < 16; e++)
                    top = fmaxf(top, st[k][e]);
            auto both = [](float v) {   // the larger of the row's two lanes'
                const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
                return fmaxf(__uint_as_float(x[0]), __uint_as_float(x[1]));
            };
            const float was = ref;
            ref = fmaxf(ref, __builtin_ceilf(both(top) * f1));
            const float base = ref == -INFINITY ? 0.f : ref;
            const int fall = (int)fmaxf(was - base, -1000.f);   // (there was nothing: -1000)
            int move = most > 0.f ? fall + unit - tu : 0;   // of acc (or it is zero)
            float held = ref > -INFINITY ? most : 0x1p4f;
            if (move != 0 || ref > was)   // (fall and the unit's change may cancel: l and unit follow all the same)
                held = 0.f;
            float up = -base, down = 1.f;
            if (__builtin_amdgcn_ballot_w64(held < 0x1p4f) != 0) {
                l = __builtin_amdgcn_ldexpf(l, fall);
                const float before = __builtin_amdgcn_ldexpf(most, min(move, 100));
                float large = ref > was ? __int_as_float(half_least) : 0.f;
                auto off = [&] { return fmaxf(before, large) > 0x1p15f || fmaxf(before, large) < 0x1p4f; };
                int shift = 0;   // of the tile's weights
                if (__builtin_amdgcn_ballot_w64(off() && ref > -INFINITY) != 0) {
                    large = 0.f;
#pragma unroll
                    for (int k = 0; k < 2; k++)
#pragma unroll
                        for (int b = 0; b < 4; b++) {
                            const f32x4 x = *reinterpret_cast<const f32x4 *>(norm + 64 + 32 * k + 8 * b);
#pragma unroll
                            for (int i = 0; i < 4; i++)
                                large = fmaxf(large, fabsf(__builtin_amdgcn_exp2f(fmaf(st[k][4 * b + i], f1, -base)) * x[i]));
                        }
                    large = both(large);
                    // (sums that would move by more than 2^100 keep their unit: the tile's weights are nothing next to them)
                    if (off() && fmaxf(before, large) > 0.f)
                        shift = move > 100 ? fall - move : min(14 - __builtin_amdgcn_frexp_expf(fmaxf(before, large)), 100);
                }
                unit = tu - shift;
                move += shift;
                most = fmaxf(__builtin_amdgcn_ldexpf(most, move), __builtin_amdgcn_ldexpf(large, shift));
                const float scale = __builtin_amdgcn_ldexpf(1.f, min(move, 126));
#pragma unroll
                for (int c = 0; c < C::CT; c++)
#pragma unroll
                    for (int e = 0; e < 16; e++)
                        acc[c][e] *= scale;
                // (past 2^-60 the weights are zero in fp16 and e4m3 either way, and l keeps its small ones)
                shift = max(shift, -60);
                up += (float)shift;
                down = __builtin_amdgcn_ldexpf(1.f, -shift);
            }
            float sum = 0.f;
            u32x4 p[4];   // positions 16 s .. 16 s + 15 (B's order)
            i32x8 pr;     // of all 64, what fp16 left
#pragma unroll
            for (int k = 0; k < 2; k++)
#pragma unroll
                for (int b = 0; b < 4; b++) {
                    const f32x4 x = *reinterpret_cast<const f32x4 *>(norm + 64 + 32 * k + 8 * b);
                    float y[4];
#pragma unroll
                    for (int i = 0; i < 4; i++) {
                        const float e = __builtin_amdgcn_exp2f(fmaf(st[k][4 * b + i], f1, up));
                        sum += e;
                        y[i] = e * x[i];
                    }
#pragma unroll
                    for (int i = 0; i < 2; i++) {
                        const int at = 2 * (b % 2) + i;
                        uint32_t o;
                        asm("v_cvt_pk_f16_f32 %0, %1, %2" : "=v"(o) : "v"(y[2 * i]), "v"(y[2 * i + 1]));
                        p[2 * k + b / 2][at] = o;
                        const f16x2 r = __builtin_bit_cast(f16x2, o);
                        y[2 * i] -= (float)r.x;
                        y[2 * i + 1] -= (float)r.y;
                    }
                    pr[4 * k + b] = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false), true);
                }
            l = fmaf(sum, down, l);
            if (min((int)tile[4], (int)tile[5]) < lim - tb)
                l = NAN;
            // 5. O^T += V^T P^T, likewise
            const uint8_t *val = buf + C::kV + n32 * C::VROW + 16 * half;
            const uint8_t *val8 = buf + C::kV8 + n32 * C::VROW8 + 32 * half;
            u32x4 vv[2][C::CT];
            i32x8 v8[2];
            v8[0] = read_bytes32(val8);
            auto read_values = [&](int k) {
#pragma unroll
                for (int c = 0; c < C::CT; c++)
                    vv[k & 1][c] = *reinterpret_cast<const u32x4 *>(val + 32 * c * C::VROW + 32 * k);
            };
#pragma unroll
            for (int c = 0; c < C::CT; c++) {
                if (c + 1 < C::CT)
                    v8[(c + 1) & 1] = read_bytes32(val8 + 32 * (c + 1) * C::VROW8);
                else
                    read_values(0);
                __builtin_amdgcn_sched_barrier(0);
                acc[c] = mfma_bytes(v8[c & 1], pr, acc[c], 0);
                __builtin_amdgcn_sched_barrier(0);
            }
#pragma unroll
            for (int k = 0; k < 4; k++) {
                if (k + 1 < 4)
                    read_values(k + 1);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int c = 0; c < C::CT; c++)
                    acc[c] = __builtin_amdgcn_mfma_f32_32x32x16_f16(as_halves(vv[k & 1][c]), as_halves(p[k]), acc[c], 0, 0, 0);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    };
    if constexpr (!C::AHEAD) {
        if (nt > 0 && fetches)
            store_raw(0);
        __syncthreads();
        for (int t = 0; t < nt; t++) {
            decode_keys(t);
            decode_values(t);
            if (t + 1 < nt && fetches) {   // (waves WK and WV fetch the next tile's records while all compute)
                fetch(t + 1, next);
                next = block_of(t + 2);
            }
            __syncthreads();
            attend(t);
            if (t + 1 < nt && fetches)
                store_raw(t + 1);
            __syncthreads();
        }
    } else if (nt > 0) {
        // the first four waves decode the next tile's keys before they attend to this
        // one, the next four its values after it: of the two waves of a SIMD one has
        // vector instructions while the other has matrix products
        if (fetches) {
            store_raw(0);
            if (nt > 1)
                fetch(1, next);
            next = block_of(2);
        }
        __syncthreads();
        if (w < 4)
            decode_values(0);
        else
            decode_keys(0);
        if (nt > 1 && fetches)
            store_raw(1);
        __syncthreads();
        for (int t = 0; t < nt; t++) {
            if (t + 2 < nt && fetches) {
                fetch(t + 2, next);
                next = block_of(t + 3);
            }
            if (w >= 4 && t + 1 < nt)
                decode_keys(t + 1);
            attend(t);
            if (w < 4 && t + 1 < nt)
                decode_values(t + 1);
            if (t + 2 < nt && fetches)
                store_raw(t + 2);
            __syncthreads();
        }
    }

    // 6. the row's part, for the join; or the row itself: a lane has four
    //    consecutive coordinates at a time, a slot of the 4-D and 2-D rotations
    {
        const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(l), __float_as_uint(l), false, false);
        l = __uint_as_float(x[0]) + __uint_as_float(x[1]);
    }
    if (nonfinite(qmax) && l != 0.f)
        l = NAN;   // an infinity or NaN in the rotated query (counted as zero till here), and a position
    if (!on)
        return;
    const float vs = __builtin_amdgcn_ldexpf(a.v_half.scale, unit - 14);
    if (!a.part) {   // (one split; 8-D slots are two lanes', and go through the join)
        const float inv = l == 0.f ? 0.f : vs / l;
        auto finish = [&](auto var) {
            constexpr int VAR = decltype(var)::value;
#pragma unroll
            for (int c = 0; c < C::CT; c++)
#pragma unroll
                for (int b = 0; b < 4; b++)
                    if (D % 32 == 0 || 32 * c + 8 * b < D) {
                        const float y[4] = {acc[c][4 * b] * inv, acc[c][4 * b + 1] * inv, acc[c][4 * b + 2] * inv,
                                            acc[c][4 * b + 3] * inv};
                        attn_emit<VAR, 4>(a, row, h, 8 * c + 2 * b + half, y);
                    }
        };
        switch (a.variant) {   // (uniform)
        case VAR_FULL: finish(std::integral_constant<int, VAR_FULL>{}); break;
        case VAR_FAST: finish(std::integral_constant<int, VAR_FAST>{}); break;
        case VAR_PLANAR2D: finish(std::integral_constant<int, VAR_PLANAR2D>{}); break;
        }
        if (half == 0 && a.lse)
            a.lse[row] = attn_lse(ref, l);
        return;
    }
    float *dst = a.part + attn_part(a, row, blockIdx.z) * D + 4 * half;
#pragma unroll
    for (int c = 0; c < C::CT; c++)
#pragma unroll
        for (int b = 0; b < 4; b++)
            if (D % 32 == 0 || 32 * c + 8 * b < D)
                *reinterpret_cast<f32x4 *>(dst + 32 * c + 8 * b) =
                    f32x4{acc[c][4 * b] * vs, acc[c][4 * b + 1] * vs, acc[c][4 * b + 2] * vs, acc[c][4 * b + 3] * vs};
    if (half == 0) {
        float *ml = a.part_ml + attn_part(a, row, blockIdx.z) * 2;
        ml[0] = ref;
        ml[1] = l;
    }
}

}  // namespace
}  // namespace isoq
