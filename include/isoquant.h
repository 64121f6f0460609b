/*
 * isoquant.h -- C ABI of the IsoQuant stage-1 quantize/dequantize library for
 * AMD Instinct MI355X (gfx950).
 *
 * IsoQuant (arXiv 2603.28430) compresses a d-dimensional vector x in four
 * steps (Algorithm 1): split off the norm rho = ||x|| (Sec. 3); rotate the
 * direction block by block, with 4-D quaternion blocks v -> q_L v conj(q_R)
 * (IsoQuant-Full, Sec. 5.2), v -> q_L v (IsoQuant-Fast, Sec. 5.3), 2-D
 * planar rotations (Sec. 5.4) or 8-D grouped blocks (Table 3's block-size
 * axis, Haar(SO(8)) blocks as in Sec. 5.7); quantize every rotated coordinate with one
 * shared b-bit Lloyd-Max codebook; then dequantize, rotate back and multiply
 * by rho.
 *
 * Conventions shared by every call:
 *   - Status codes are returned, never exceptions.  Arguments are validated
 *     before any device work; a call that returns an error launched nothing.
 *   - Rows are contiguous, row-major [n][d].  Coordinate 4i of a row is the
 *     real part of quaternion block i; the 2-D case pairs (2j, 2j+1); 8-D
 *     block i holds coordinates 8i .. 8i+7.
 *   - Device buffers are owned by the caller and must live on the device that
 *     was current at isoq_params_init.  Row buffers (fp16/fp32) must be
 *     16-byte aligned, index records and norm arrays 4-byte aligned.
 *   - `stream` is a hipStream_t (NULL = the null stream).  Calls are
 *     asynchronous on it and never synchronise the device.  n = 0 is a valid
 *     no-op.  Output buffers must not overlap inputs, except that the
 *     reconstruction may be written in place over the input of
 *     isoq_roundtrip (x_hat == x exactly).
 *   - A parameter handle is immutable after init; concurrent calls that share
 *     it are safe.  Only init and destroy allocate or free device memory.
 *   - Supported shapes in this version: bits in {2, 3, 4}, fp16 or fp32 rows
 *     (arithmetic is fp32 in every case); d from 1 to 1024 for quantize,
 *     dequantize and round trip (tuned kernels for d in {64, 128, 256, 512},
 *     packed-row kernels for fp16 rows at other multiples of 16 up to 504, a
 *     generic kernel family for every other width), d in {64, 128, 256, 512}
 *     for the KV-cache append (and, fp16 rows only, 80, 96, 160 and 192), d in
 *     {64, 80, 96, 128, 160, 192, 256, 512} for the attention-score call
 *     without the sketch and for attention (any d from 1 to 1024 by
 *     width-generic kernels), d in {64, 128, 256, 512} and (fp16 rows, or any
 *     query type for the scores) 80, 96, 160 and 192 for the stage-2 sketch
 *     and the calls that use it (Full, Fast and 2-D handles; every other call
 *     takes all four variants).
 *   - Widths that are not a multiple of the block size (4; 2-D: 2; 8-D: 8)
 *     follow Sec. 5.1: the last block is zero padded, all pw rotated
 *     coordinates are quantized and stored (pw = 4 ceil(d/4); 2-D:
 *     2 ceil(d/2); 8-D: 8 ceil(d/8)), and the padded coordinates are dropped
 *     after the inverse rotation.
 *   - Rows must be finite.  The squared norm is accumulated in fp32, so an
 *     fp32 row must have 1e-18 <= ||x|| <= 1e18 or be exactly zero (every fp16
 *     row qualifies); a zero row gives rho = 0, x_hat = 0 and every index
 *     2^(bits-1) - 1.
 */
#ifndef ISOQUANT_H
#define ISOQUANT_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum isoq_status {
    ISOQ_OK = 0,
    ISOQ_E_INVALID = 1,     /* bad enum value, n < 0, rows_per_set < 1, bad codebook  */
    ISOQ_E_UNSUPPORTED = 2, /* valid request outside the shapes listed above           */
    ISOQ_E_NULL = 3,        /* required pointer is NULL                                */
    ISOQ_E_ALIGN = 4,       /* pointer misaligned                                      */
    ISOQ_E_HIP = 5,         /* HIP runtime error (launch failure, no device, ...)      */
    ISOQ_E_NOMEM = 6,       /* device or host allocation failed                        */
    ISOQ_E_DEVICE = 7       /* called with a device other than the handle's            */
} isoq_status;

/* variants (Sec. 5.2, 5.3, 5.4; ISOQ_BLOCK8: 8-D grouped blocks, Table 3 and
 * Sec. 5.7) */
enum { ISOQ_FULL = 0, ISOQ_FAST = 1, ISOQ_PLANAR2D = 2, ISOQ_BLOCK8 = 3 };
/* row element types */
enum { ISOQ_F32 = 0, ISOQ_F16 = 1 };

typedef struct isoq_params isoq_params;

/*
 * isoq_params_init -- build the rotation parameters and the codebook of one
 * quantizer and copy them to the current device.
 *
 *   variant   ISOQ_FULL, ISOQ_FAST, ISOQ_PLANAR2D or ISOQ_BLOCK8.
 *   d, bits   vector width and bits per coordinate.
 *   n_sets    number of independent rotation sets (e.g. one per attention
 *             head); row r of a later call uses set (r / rows_per_set) mod
 *             n_sets.  The codebook is shared by all sets.
 *   rot_host  NULL, or host array of raw draws (Sec. 5.5: unconstrained
 *             vectors normalised on the fly), n_sets * isoq_raw_params_per_set
 *             doubles: Full, per set and block i, u_L[4] then u_R[4]; Fast,
 *             u_L[4] per block; 2-D, one angle theta (radians) per coordinate
 *             pair; 8-D, a raw 8x8 matrix G per block of 8 coordinates
 *             (row-major).  Quaternions are normalised here (u / ||u||); a zero
 *             u is ISOQ_E_INVALID.  An 8-D block rotates by the orthogonal
 *             factor Q of G = QR with a positive diagonal in R (Haar on O(8)
 *             for Gaussian G), with column 0 negated when det Q = -1 (so Q is
 *             in SO(8)); G with dependent columns is ISOQ_E_INVALID.
 *             NULL: draw them from `seed` (Haar sampling, Sec. 5.5): u ~ N(0,I4)
 *             and theta ~ U[0, 2 pi) from Philox4x32-10 with key = seed and
 *             counter (block, set, stream, 0), stream 0 for u_L, 1 for u_R, 2 for
 *             theta (8-D: G ~ N(0,1) entries 4q .. 4q+3 from counter
 *             (block, set, 4, q), q = 0..15); Box-Muller maps the four 32-bit words (w0..w3) to
 *             (z0, z1) = sqrt(-2 ln U1) (cos 2 pi U2, sin 2 pi U2) with
 *             U1 = (w0 + 1/2) / 2^32, U2 = w1 / 2^32, likewise (z2, z3) from
 *             (w2, w3); theta = 2 pi w0 / 2^32.
 *   codebook_host  NULL, or host array of 2^bits levels, strictly increasing
 *             and symmetric about 0 (|c_k + c_{K-1-k}| <= 1e-6 max|c|; they are
 *             then symmetrised exactly).  NULL: Lloyd-Max levels for N(0, 1/d)
 *             after 200 Lloyd iterations from levels evenly spaced on
 *             [-3/sqrt(d), 3/sqrt(d)].  Decision thresholds are the midpoints
 *             of adjacent levels.  The kernels take the sign of a rotated
 *             value y (y > 0) and compare |y| with the positive thresholds
 *             (|y| > t), so a value exactly on a threshold goes to the level
 *             of smaller magnitude: the lower level for y > 0, the upper one
 *             for y < 0 (0 itself goes to level 2^(bits-1) - 1).
 *   out       receives the handle (set to NULL on error).
 * Host arrays are only read during the call; the caller keeps ownership.
 */
isoq_status isoq_params_init(isoq_params **out, int variant, int d, int bits, int n_sets,
                             const double *rot_host, const double *codebook_host, uint64_t seed);

/* Free the handle and its device memory (NULL is accepted).  Must not race
 * with calls still running on the GPU that use the handle: synchronise their
 * streams first. */
isoq_status isoq_params_destroy(isoq_params *p);

/*
 * isoq_params_export -- copy out the values the device uses (fp32).  Any
 * output may be NULL.
 *   rot_out        n_sets * isoq_export_params_per_set floats: Full, per
 *                  block q_L[4] then q_R[4] (unit); Fast q_L[4]; 2-D
 *                  (cos theta, sin theta) per pair; 8-D the block's
 *                  orthogonal Q (64 floats, row-major).  These are the
 *                  parameter counts of Table 1 (8 g4, 4 g4, 2 g2 per set;
 *                  8-D, not in Table 1: 64 g8).
 *   levels_out     2^bits levels, ascending.
 *   thresholds_out 2^bits - 1 decision thresholds, ascending.
 */
isoq_status isoq_params_export(const isoq_params *p, float *rot_out, float *levels_out,
                               float *thresholds_out);

/* Read back the shape of a handle (any output may be NULL). */
isoq_status isoq_params_info(const isoq_params *p, int *variant, int *d, int *bits, int *n_sets);

/*
 * isoq_quantize -- encoder half of Algorithm 1: norm split, blockwise rotation,
 * scalar quantization.
 *   x          device, [n][d] rows of `dtype`.
 *   idx_packed device, [n][isoq_record_bytes(variant, d, bits)] bytes: per row
 *              one record of the pw rotated coordinates in which coordinate j
 *              occupies bits [j*bits, (j+1)*bits), bit m being bit (m mod 8) of
 *              byte m/8 (least significant first); bits past pw*bits are 0.
 *   norms      device, [n] fp32 rho = ||x||_2.
 * Index of a coordinate y: number of thresholds t_k with y > t_k applied to the
 * direction x / max(rho, 1e-12).
 */
isoq_status isoq_quantize(const isoq_params *p, int dtype, const void *x, int64_t n,
                          int64_t rows_per_set, uint8_t *idx_packed, float *norms, void *stream);

/*
 * isoq_dequantize -- decoder half of Algorithm 1: level lookup, inverse block
 * rotation, multiplication by rho.  Inputs as produced by isoq_quantize; output
 * x_hat device [n][d] rows of `dtype` (fp16 is rounded to nearest even).
 */
isoq_status isoq_dequantize(const isoq_params *p, int dtype, const uint8_t *idx_packed,
                            const float *norms, int64_t n, int64_t rows_per_set, void *x_hat,
                            void *stream);

/*
 * isoq_roundtrip -- the fused stage-1 path x -> x_hat of Algorithm 1 with no
 * index traffic to memory.  Bitwise equal to isoq_quantize followed by
 * isoq_dequantize on the same handle, rows_per_set and dtype.
 */
isoq_status isoq_roundtrip(const isoq_params *p, int dtype, const void *x, int64_t n,
                           int64_t rows_per_set, void *x_hat, void *stream);

/*
 * isoq_kv_append -- quantize-on-append into a paged K/V cache, for
 * autoregressive decoding (the fused KV-cache compression the paper names as
 * its next step, Sec. 10): the new key and value rows are encoded as by
 * isoq_quantize (Algorithm 1's encoder) and their index records and norms are
 * written straight into the cache slots of their tokens.  Any d in 1..1024:
 * d in {64, 128, 256, 512}, and fp16 rows at 80, 96, 160 and 192, take one
 * launch for both tensors; other widths, and fp32 rows at those four, one
 * launch of the width-generic encoder per tensor.
 *
 *   pk, pv      handles of the K and V quantizers.  They must agree in variant,
 *               d and bits; each has n_sets == 1 or n_sets == n_heads, and the
 *               row of (token t, head h) uses set h (resp. set 0).  pv may be
 *               pk.  pv, v_new, v_idx and v_rho all NULL: keys only.
 *   dtype       ISOQ_F16 or ISOQ_F32, the element type of k_new and v_new.
 *   k_new, v_new  device, [n_tokens][n_heads][d] rows (16-byte aligned).
 *   slot_mapping  device, int64 [n_tokens] (8-byte aligned): cache slot of
 *               token t; a slot < 0 or >= n_blocks * block_size skips the token
 *               (padding), its rows are not written.
 *   k_idx, v_idx  device, n_blocks * n_heads * block_size * R bytes (R =
 *               isoq_packed_bytes; 4-byte aligned): slot s is position s mod
 *               block_size of cache block s / block_size, and (block b, head
 *               h) owns the block_size * R bytes from (b n_heads + h)
 *               block_size R on.  Inside that region the records are stored
 *               piece-major: record byte k of position p lies at byte
 *               (floor(k / P) block_size + p) P + k mod P, with P = 16 if 16
 *               divides R, else 8 if 8 divides R, else P = R (records stored
 *               whole, position after position).  Pieces of consecutive
 *               positions are adjacent, which the logit kernel reads in one
 *               coalesced load.  Record bytes as in isoq_quantize.
 *   k_rho, v_rho  device, fp32 [n_blocks][n_heads][block_size].
 * Limits: n_tokens * n_heads < 2^31, n_blocks * block_size < 2^31, n_heads and
 * block_size >= 1, and for the one-launch shapes at most 65,535 launch blocks
 * of tokens (n_tokens up to 8,388,480 at d = 64, 4,194,240 at d = 128,
 * 2,097,120 at d = 256, 1,048,560 at d = 512; fp16 rows: 6,291,360 at d = 80,
 * 5,242,800 at d = 96, 3,145,680 at d = 160, 2,621,400 at d = 192); beyond
 * that ISOQ_E_UNSUPPORTED.  Distinct tokens must map to distinct slots (a repeated slot
 * is written by both rows in an unspecified order).  Slots not named are left
 * untouched.  n_tokens = 0 is a no-op.
 */
isoq_status isoq_kv_append(const isoq_params *pk, const isoq_params *pv, int dtype,
                           const void *k_new, const void *v_new, const int64_t *slot_mapping,
                           int64_t n_tokens, int n_heads, uint8_t *k_idx, float *k_rho,
                           uint8_t *v_idx, float *v_rho, int64_t n_blocks, int block_size,
                           void *stream);

/*
 * isoq_kv_scores -- attention logits of decoding queries against the keys of
 * a paged cache written by isoq_kv_append, without dequantizing the keys.  A
 * key's reconstruction is rho T^{-1}(c[idx]) and T is orthogonal (Prop. 1), so
 * <q, k_hat> = rho <T q, c[idx]>: each query is rotated once and the logits
 * are sums over the packed index records.  Any d in 1..1024: at d in {64, 80,
 * 96, 128, 160, 192, 256, 512} by lookup tables or matrix products; at other
 * widths a width-generic kernel sums (T q_pad)_j c[idx_j] over the record's
 * zero-padded coordinates (q_pad: q with zeros past d), one workgroup per
 * query head.
 *
 *   pk          the K quantizer (n_sets == 1 or n_sets == n_kv_heads; key head h
 *               uses set h, resp. 0).
 *   dtype       ISOQ_F16 or ISOQ_F32, the element type of q.
 *   q           device, [n_seqs][n_q_heads][d] (16-byte aligned).  Query head hq
 *               reads key head hq / (n_q_heads / n_kv_heads) (grouped-query
 *               attention; n_q_heads must be a multiple of n_kv_heads).
 *   k_idx, k_rho  the cache, laid out as in isoq_kv_append (k_idx 16-byte
 *               aligned), n_blocks cache blocks of block_size positions.
 *   block_table device, int32 [n_seqs][max_blocks_per_seq]: cache block of the
 *               sequence's positions [j * block_size, (j+1) * block_size).
 *   seq_lens    device, int32 [n_seqs]: positions of each sequence.
 *   scores      device, fp32 [n_seqs][n_q_heads][max_len]:
 *               scores[s][hq][t] = scale * <q[s][hq], k_hat(s, t)> for
 *               t < min(seq_lens[s], max_len, max_blocks_per_seq * block_size).
 *               Other positions, and positions whose block id lies outside
 *               [0, n_blocks), are not written.
 * Limits: n_seqs <= 65535, max_blocks_per_seq * block_size < 2^31, and at the
 * tuned widths at most 160 KB for group * (d/F * 2^(F bits) + d) * 4 bytes with
 * F = 2 for 2 and 3 bits, F = 1 for 4 bits (ISOQ_E_UNSUPPORTED otherwise; e.g.
 * at d = 128, 3 bits, 16.9 KB per query head): what the lookup tables of a
 * group would take in LDS.
 * Arithmetic: the query is rotated in fp32.  One query head per key head: sums
 * of table lookups in fp32.  Two or more (and single heads at d = 512, 3 and 4
 * bits): fixed-point digits on the integer matrix cores, the codebook levels
 * within 2^-23 of themselves (most Lloyd-Max levels within 2^-24), the rotated
 * query's coordinates within 2^-31 of its largest, the sums exact and rounded
 * to fp32 once; closer to an exact sum than the tables on ordinary keys.  A
 * query with an infinity or NaN gives what an IEEE sum over its rotated
 * coordinates gives, for any group: infinite or NaN logits.
 */
isoq_status isoq_kv_scores(const isoq_params *pk, int dtype, const void *q, int n_seqs,
                           int n_q_heads, int n_kv_heads, const uint8_t *k_idx, const float *k_rho,
                           int64_t n_blocks, int block_size, const int32_t *block_table,
                           int max_blocks_per_seq, const int32_t *seq_lens, float scale,
                           float *scores, int64_t max_len, void *stream);

/*
 * Stage-2 residual sketch (Sec. 8: the stage-1 residual r = x - x_hat is
 * projected by a quantized Johnson-Lindenstrauss transform and corrects inner
 * products without bias).  A sketch handle holds a Gaussian projection S
 * [m][d]; a row is stored as its stage-1 record and rho plus the m sign bits
 * z_i = [(S r)_i > 0] and gamma = ||r||, and <q, x> is estimated by
 *     <q, x_hat> + sqrt(pi/2) / m * gamma * <S q, 2 z - 1>.
 *
 * isoq_sketch_init -- build the sketch of quantizer p on the current device.
 *   m       sketch bits per row: 64 or 128 at d = 64, 80, 96, 128, 160 and
 *           192; 64 at d = 256 and 512 (the projection, m d fp16, is staged in
 *           LDS).  Other d, other m, or an 8-D handle: ISOQ_E_UNSUPPORTED.
 *   S_host  NULL, or host array [m][d] of doubles (row-major).  NULL: S is
 *           drawn from `seed`: S[i][4g .. 4g+3] is the Box-Muller quadruple of
 *           Philox4x32-10 with key = seed and counter (g, i, 3, 0) (the
 *           mapping of isoq_params_init).
 * The sketch is bound to p's rotation (it stores S T^{-1} for every set); use
 * it only with the handle it was built from.  Only init and destroy allocate.
 */
typedef struct isoq_sketch isoq_sketch;
isoq_status isoq_sketch_init(isoq_sketch **out, const isoq_params *p, int m, const double *S_host,
                             uint64_t seed);
isoq_status isoq_sketch_destroy(isoq_sketch *sk);
/* m and the projection S as used (fp32, [m][d]); any output may be NULL. */
isoq_status isoq_sketch_export(const isoq_sketch *sk, int *m, float *S_out);

/*
 * isoq_quantize_qjl -- isoq_quantize plus the stage-2 sketch of every row.
 *   idx_packed, norms  as isoq_quantize (bitwise the same records and norms).
 *   signs   device, [n][m/8] bytes (4-byte aligned): bit i of a row's record
 *           (bit i mod 8 of byte i / 8) is z_i.  The projection runs in fp16
 *           with fp32 accumulation, so a sign whose exact projection lies
 *           within about 2^-9 sum_j |S'_ij| |e_j| rho of zero may differ from
 *           an exact computation (S' = S T^{-1}, e the normalised rotated error).
 *   gamma   device, [n] fp32 ||x - x_hat||.
 * Needs one rotation set per block of rows: n_sets == 1, or rows_per_set a
 * multiple of 64 rows at d = 128 (32 at d = 256); ISOQ_E_UNSUPPORTED otherwise.
 * At d = 80, 96, 160 and 192: fp16 rows and n_sets == 1 only.
 */
isoq_status isoq_quantize_qjl(const isoq_params *p, const isoq_sketch *sk, int dtype, const void *x,
                              int64_t n, int64_t rows_per_set, uint8_t *idx_packed, float *norms,
                              uint8_t *signs, float *gamma, void *stream);

/*
 * isoq_kv_append_qjl -- quantize-on-append of key rows with the stage-2
 * residual sketch (Sec. 8): each new key row is encoded as by
 * isoq_quantize_qjl (records, norms, m sign bits and gamma, bit for bit the
 * same) and all four go straight into the cache slot of its token, in one
 * launch.  Values need no sketch: append them with isoq_kv_append.
 *
 *   pk, sk      the K quantizer and its sketch (same variant, d, sets and
 *               device); pk->n_sets == 1 or n_heads (head h uses set h).
 *   dtype, k_new, slot_mapping, n_tokens, n_heads, k_idx, k_rho, n_blocks,
 *   block_size  as in isoq_kv_append.
 *   k_signs     device, [n_blocks][n_heads][block_size][m/8] bytes (4-byte
 *               aligned), the sign sketch of each slot, bit i of byte i/8 =
 *               [(S (x - x_hat))_i > 0].
 *   k_gamma     device, fp32 [n_blocks][n_heads][block_size], ||x - x_hat||.
 * Skipped slots (< 0 or >= n_blocks * block_size) are not written; other
 * slots not named are untouched.  Limits as in isoq_kv_append; the widths and
 * sketch sizes are those of isoq_sketch_init.
 */
isoq_status isoq_kv_append_qjl(const isoq_params *pk, const isoq_sketch *sk, int dtype, const void *k_new,
                               const int64_t *slot_mapping, int64_t n_tokens, int n_heads, uint8_t *k_idx,
                               float *k_rho, uint8_t *k_signs, float *k_gamma, int64_t n_blocks, int block_size,
                               void *stream);

/*
 * isoq_kv_scores_qjl -- isoq_kv_scores with the stage-2 residual correction:
 *   scores[s][hq][t] = scale * (rho <T q, c[idx]> + sqrt(pi/2) / m * gamma
 *                               * <S q, 2 z - 1>)
 * for keys stored with their sketch: k_signs device [n_blocks][n_kv_heads]
 * [block_size][m/8] bytes and k_gamma device fp32 [n_blocks][n_kv_heads]
 * [block_size] (4-byte aligned), in the layout of k_idx / k_rho (sign
 * records as written by isoq_quantize_qjl).  sk is the keys' sketch (built
 * from pk).  Other arguments and limits as isoq_kv_scores; S q is computed
 * in fp32.
 */
isoq_status isoq_kv_scores_qjl(const isoq_params *pk, const isoq_sketch *sk, int dtype, const void *q,
                               int n_seqs, int n_q_heads, int n_kv_heads, const uint8_t *k_idx,
                               const float *k_rho, const uint8_t *k_signs, const float *k_gamma,
                               int64_t n_blocks, int block_size, const int32_t *block_table,
                               int max_blocks_per_seq, const int32_t *seq_lens, float scale, float *scores,
                               int64_t max_len, void *stream);

/*
 * isoq_kv_scores_filled -- isoq_kv_scores (sk, k_signs and k_gamma NULL) or
 * isoq_kv_scores_qjl that also writes -inf to every position of
 * scores[s][hq][0 .. max_len) which those leave unwritten, so that a softmax
 * over max_len ignores them and the buffer needs no initialisation.
 * n_blocks and max_blocks_per_seq may be 0 (every position is then -inf);
 * max_len at most 67,107,840.
 */
isoq_status isoq_kv_scores_filled(const isoq_params *pk, const isoq_sketch *sk, int dtype, const void *q,
                                  int n_seqs, int n_q_heads, int n_kv_heads, const uint8_t *k_idx,
                                  const float *k_rho, const uint8_t *k_signs, const float *k_gamma,
                                  int64_t n_blocks, int block_size, const int32_t *block_table,
                                  int max_blocks_per_seq, const int32_t *seq_lens, float scale, float *scores,
                                  int64_t max_len, void *stream);

/*
 * isoq_kv_attn -- attention of new tokens over a paged cache of quantized keys
 * and values written by isoq_kv_append, without decompressing either: decoding
 * steps (one new token a sequence), drafted tokens and chunks of a prompt
 * (several, causal).  For token i of a sequence's n new tokens, query head hq
 * and key head h = hq / (n_q_heads / n_kv_heads):
 *     s_t = scale * <q, k_hat(t)>,  out = sum_t softmax(s)_t v_hat(t),
 *     lse = ln sum_t exp(s_t)
 * over the positions t < seq_lens[s] - (n - 1 - i): the new tokens are the
 * sequence's last positions (append them first), and each attends to those up
 * to its own.  Positions past max_len or max_blocks_per_seq * block_size, and
 * positions whose block id lies outside [0, n_blocks), are left out, whatever
 * the cache holds there.  A token with no position left: out = 0, lse = -inf.
 *
 *   pk, pv      the K and V quantizers, of one variant, d and bits (any d in
 *               1..1024); n_sets 1 or n_kv_heads each.
 *   dtype       ISOQ_F16 or ISOQ_F32: the element type of q and out.
 *   q, out      device, [n_tokens][n_q_heads][d] (16-byte aligned).
 *   q_start     device, int32 [n_seqs + 1], ascending: sequence s has the tokens
 *               q_start[s] .. q_start[s+1] - 1.  max_q_len: the most tokens that a
 *               sequence has (known to the host).  The call is planned as if all
 *               had as many: a loose bound costs time, and so do single tokens
 *               next to a long chunk, which two calls take less for (15 and one
 *               of 512 at 8,192 positions, 8 x 4 heads, d = 128: 41 and 155 us, 382
 *               in one call).  Rows of no sequence are left
 *               as they were, in out and lse; so are a sequence's tokens from
 *               max_q_len on.  NULL: one token a sequence, n_tokens == n_seqs and
 *               max_q_len == 1.
 *   k_idx, k_rho, v_idx, v_rho, n_blocks, block_size, block_table,
 *   max_blocks_per_seq, seq_lens  as in isoq_kv_scores (the records 16-byte
 *               aligned).
 *   max_len     positions of the longest sequence at most, as far as the host
 *               knows (max_blocks_per_seq * block_size if it does not): a closer
 *               bound cuts long caches into better splits (16 sequences of 8,192
 *               positions, 8 x 4 heads, in a table of 131,072: 40 us with it, 86
 *               without).
 *   scale       up to 2.35e38 in magnitude: it is used in units of ln 2, as a float
 *               (larger ones, infinities and NaN are ISOQ_E_INVALID).
 *   lse         device, fp32 [n_tokens][n_q_heads], or NULL.
 *   workspace   device, at least isoq_kv_attn_workspace(...) bytes for the same
 *               arguments (16-byte aligned; may be NULL where that is 0).  Its
 *               contents matter only while the call runs on its stream: calls
 *               on different streams, or captured graphs that may run at the
 *               same time, need one each.  A smaller one is ISOQ_E_INVALID.
 * Limits: n_seqs <= 65535, n_tokens * n_q_heads < 2^31, max_q_len * n_q_heads <=
 * 2^23, max_blocks_per_seq * block_size <= 2^31 - 1024.
 * Arithmetic: logits, softmax statistics and sums in fp32 or in integers of 32
 * bits (see the kernels for what is rounded).  Weights and value levels are digits
 * (30 bits, and 16, of fp32 queries 24), but for fp16 queries with 32 rows and more a key
 * head (its query heads times max_q_len) at d = 64, 80, 96 and 128: there they are fp16 with
 * a correction, and out is off by 2.1e-4 to 2.2e-4 of its norm where its own rounding to
 * fp16 takes 2.07e-4.  A row's result is as exact as its
 * own weights and norms allow, whatever norms stand at other positions.  A query
 * with an infinity or NaN gives NaN in its row of out and lse if it attends to
 * any position, and so does a norm of k_rho or v_rho that is one in the rows that
 * attend to its position, not in others.  The result
 * does not depend on the order in which workgroups run.
 */
isoq_status isoq_kv_attn(const isoq_params *pk, const isoq_params *pv, int dtype, const void *q,
                         const int32_t *q_start, int64_t n_tokens, int max_q_len, int n_seqs, int n_q_heads,
                         int n_kv_heads, const uint8_t *k_idx, const float *k_rho, const uint8_t *v_idx,
                         const float *v_rho, int64_t n_blocks, int block_size, const int32_t *block_table,
                         int max_blocks_per_seq, const int32_t *seq_lens, int64_t max_len, float scale, void *out,
                         float *lse, void *workspace, size_t workspace_bytes, void *stream);
/* Bytes of workspace for isoq_kv_attn with these arguments (0 for invalid ones). */
size_t isoq_kv_attn_workspace(const isoq_params *pk, const isoq_params *pv, int dtype, int64_t n_tokens, int max_q_len,
                              int n_seqs, int n_q_heads, int n_kv_heads, int block_size, int max_blocks_per_seq,
                              int64_t max_len);

/*
 * isoq_kv_attn_cross -- attention to states of another length, as a decoder's to
 * its encoder's: isoq_kv_attn, but for one thing: every token of a sequence
 * attends to all of its seq_lens[s] positions.  The states' keys and values are
 * quantized once (isoq_kv_append at slots of their own) and read by every step;
 * tokens that share states (the beams of one input) may be one sequence of several
 * tokens.  Arguments, limits, arithmetic and workspace (isoq_kv_attn_workspace) as
 * isoq_kv_attn.
 */
isoq_status isoq_kv_attn_cross(const isoq_params *pk, const isoq_params *pv, int dtype, const void *q,
                               const int32_t *q_start, int64_t n_tokens, int max_q_len, int n_seqs, int n_q_heads,
                               int n_kv_heads, const uint8_t *k_idx, const float *k_rho, const uint8_t *v_idx,
                               const float *v_rho, int64_t n_blocks, int block_size, const int32_t *block_table,
                               int max_blocks_per_seq, const int32_t *seq_lens, int64_t max_len, float scale, void *out,
                               float *lse, void *workspace, size_t workspace_bytes, void *stream);

/*
 * isoq_kv_attn_prefix -- isoq_kv_attn for sequences that share long beginnings (an
 * instruction, a document): a prefix's positions are in the cache once and are
 * attended to by the rows of all its sequences together, the sequences' own
 * positions follow them.  A token attends to all positions of its prefix and, as
 * in isoq_kv_attn, to its sequence's own up to itself.
 *
 *   block_table, seq_lens, max_len  the sequences' own positions (their new tokens
 *               are the last of those).
 *               Rotary positions count the prefix's too: what isoq_kv_plan gives, which
 *               counts from 0 here, and prefix_lens[p].
 *   prefix_start  device, int32 [n_prefixes + 1], ascending: prefix p is shared by
 *               the sequences prefix_start[p] .. prefix_start[p + 1] - 1, which stand
 *               side by side.  Sequences of none have only their own positions.
 *               NULL: n_prefixes is 1 (or 0) and all sequences share it.
 *   prefix_table, prefix_lens  device, int32 [n_prefixes][max_prefix_blocks] and
 *               [n_prefixes]: the prefixes' blocks and lengths, as block_table and
 *               seq_lens (the same cache and block_size).
 *   max_prefix_tokens  tokens of all sequences of one prefix at most, 1 or more (n_tokens
 *               if the host does not know); a prefix's tokens from there on are left as
 *               they were in out and lse.  max_prefix_len: positions of the longest prefix
 *               at most (max_prefix_blocks * block_size if it does not know).  Where that,
 *               n_prefixes, max_prefix_blocks or n_blocks is 0 the call is isoq_kv_attn's.
 *   workspace   at least isoq_kv_attn_prefix_workspace(...) bytes.
 * n_prefixes <= 65535; where it, max_prefix_blocks and max_prefix_len are not 0, max_prefix_tokens
 * (or n_tokens, if fewer) * n_q_heads <= 2^23.
 * Everything else as isoq_kv_attn, the rows of a prefix being those of all its sequences
 * together: single tokens behind one that many share are as exact as a chunk's rows, and
 * how many share it may change their last bits.
 */
isoq_status isoq_kv_attn_prefix(const isoq_params *pk, const isoq_params *pv, int dtype, const void *q,
                                const int32_t *q_start, int64_t n_tokens, int max_q_len, int n_seqs, int n_q_heads,
                                int n_kv_heads, const uint8_t *k_idx, const float *k_rho, const uint8_t *v_idx,
                                const float *v_rho, int64_t n_blocks, int block_size, const int32_t *block_table,
                                int max_blocks_per_seq, const int32_t *seq_lens, int64_t max_len,
                                const int32_t *prefix_table, int max_prefix_blocks, const int32_t *prefix_lens,
                                int64_t max_prefix_len, const int32_t *prefix_start, int n_prefixes,
                                int64_t max_prefix_tokens, float scale, void *out, float *lse, void *workspace,
                                size_t workspace_bytes, void *stream);
size_t isoq_kv_attn_prefix_workspace(const isoq_params *pk, const isoq_params *pv, int dtype, int64_t n_tokens,
                                     int max_q_len, int n_seqs, int n_q_heads, int n_kv_heads, int block_size,
                                     int max_blocks_per_seq, int64_t max_len, int n_prefixes, int64_t max_prefix_tokens,
                                     int max_prefix_blocks, int64_t max_prefix_len);

/*
 * isoq_kv_copy_blocks -- copy whole cache blocks inside a paged cache (forking
 * a sequence whose last block is shared, copy on write; moving blocks): for
 * every pair (source, destination) of block_pairs, the records and norms of
 * all heads, and with sk the signs and gammas, of block `source` go to block
 * `destination`, in one launch.
 *
 *   pk          the K quantizer, whose record size V shares (v_idx and v_rho, or
 *               both NULL: keys only).
 *   sk, k_signs, k_gamma  the keys' sketch and its arrays, or all NULL.
 *   block_pairs device, int32 [n_pairs][2].  A pair with a block outside [0,
 *               n_blocks), or of equal blocks, is skipped.  A destination must
 *               not be a source or destination of another pair (its contents are
 *               then unspecified; nothing else is touched).
 *   k_idx .. k_gamma, n_blocks, block_size  the cache, laid out as in
 *               isoq_kv_append (records 16-byte aligned).
 * Limits: n_pairs < 2^24, n_blocks * block_size < 2^31, and a block of one array is
 * at most 2^31 bytes.  n_pairs = 0 is a no-op.
 */
isoq_status isoq_kv_copy_blocks(const isoq_params *pk, const isoq_sketch *sk, const int32_t *block_pairs,
                                int64_t n_pairs, int n_heads, uint8_t *k_idx, float *k_rho, uint8_t *v_idx,
                                float *v_rho, uint8_t *k_signs, float *k_gamma, int64_t n_blocks, int block_size,
                                void *stream);

/*
 * isoq_kv_compact -- keep some positions of sequences and drop the others, in
 * place: afterwards position i < n_keep[s] of sequence s holds, for head h,
 * what position keep[s][h][i] held (records, norms, signs, gammas), in one
 * launch.  n_keep is then the sequences' lengths, and a sequence's blocks from
 * ceil(n_keep / block_size) on are free.
 *
 *   keep        device, int32 [n_seqs][keep_heads][max_keep], each list strictly
 *               ascending, from 0 or more; keep_heads is n_heads, or 1: one list
 *               for all heads.
 *   n_keep      device, int32 [n_seqs], entries of each list that count (cut to
 *               [0, max_keep]).
 *   block_table, max_blocks_per_seq  as in isoq_kv_scores.  The blocks of a
 *               sequence that is compacted must not be another's too, nor
 *               stand in its row twice (copy a shared block first).  An
 *               entry whose source or destination has no block in [0,
 *               n_blocks), or lies outside the table, is skipped.
 *   pk, sk, k_idx .. k_gamma, n_heads, n_blocks, block_size  as in
 *               isoq_kv_copy_blocks.
 * Positions from n_keep[s] on keep their contents.  In a list that does not ascend
 * strictly from 0 or more, entries with keep[s][h][i] < i are skipped too.
 * Limits: n_seqs <= 65535, n_heads < 2^22, max_keep <= 2^31 - 8192,
 * max_blocks_per_seq * block_size < 2^31.
 */
isoq_status isoq_kv_compact(const isoq_params *pk, const isoq_sketch *sk, const int32_t *keep, int keep_heads,
                            int max_keep, const int32_t *n_keep, int n_seqs, const int32_t *block_table,
                            int max_blocks_per_seq, int n_heads, uint8_t *k_idx, float *k_rho, uint8_t *v_idx,
                            float *v_rho, uint8_t *k_signs, float *k_gamma, int64_t n_blocks, int block_size,
                            void *stream);

/*
 * isoq_kv_plan -- the block tables and slots of a step's tokens, from the
 * sequences' lengths before and after it, on the GPU: what isoq_kv_append
 * (slot_mapping), isoq_qk_norm_rope (positions) and isoq_kv_attn (q_start,
 * seq_lens, block_table) take.  Nothing is read back, so that lengths may be
 * ones that only the GPU knows (n_keep of isoq_kv_compact, drafts that were
 * accepted), and a step can be captured into a graph.
 *
 *   lens, new_lens  device, int32 [n_seqs]: positions of each sequence before and
 *               after the step (cut to 0 .. max_blocks_per_seq * block_size).  A
 *               sequence that grows has new_lens - lens new tokens; one that
 *               shrinks (drafts taken back, the end of a sequence: 0) has none.
 *   block_table device, int32 [n_seqs][max_blocks_per_seq], in and out: the
 *               first ceil(length / block_size) entries of a row are the blocks
 *               that the sequence owns; further ones are ignored and, but for
 *               those that it takes, left as they were.
 *   free_blocks, n_free, max_free  device, int32 [max_free], in and out, and int32
 *               [1]: the first *n_free entries are free blocks (cut to 0 ..
 *               max_free).  Blocks that sequences release go behind them (past
 *               max_free: they are lost), in the order of the sequences and their
 *               positions; then the sequences that grow take blocks from the end.
 *               A sequence is refused if it and those before it want more than there
 *               are: it keeps its length and blocks, and its tokens get no slot.
 *   seq_lens    device, int32 [n_seqs]: the lengths now (may be lens itself; not
 *               new_lens).  seq_lens[s] != new_lens[s]: refused (or cut).
 *   q_start     device, int32 [n_seqs + 1]: sequence s has the tokens q_start[s] ..
 *               q_start[s + 1] - 1, those of refused sequences among them.
 *   slot_mapping, positions  device, int64 and int32 [n_tokens]: each token's slot
 *               (-1 for none: isoq_kv_append skips it) and position in its sequence
 *               (behind a prefix, isoq_kv_attn_prefix, its rotary position is that and
 *               the prefix's length).  n_tokens may
 *               be more than there are (a captured step of a fixed size): tokens
 *               past the last have slot -1 and position 0.  If it is fewer, those
 *               past n_tokens are left out, though lengths and blocks count them.
 *   n_free_out  device, int32 [1]: free blocks left (may be n_free itself).
 * Other buffers must not overlap.  Limits: n_seqs <= 65535, (max_blocks_per_seq + 1) *
 * block_size < 2^31, max_free, n_tokens and the new tokens of a step < 2^31 (q_start
 * stays at 2^31 - 1 past them).
 */
isoq_status isoq_kv_plan(const int32_t *lens, const int32_t *new_lens, int n_seqs, int32_t *block_table,
                         int max_blocks_per_seq, int block_size, int32_t *free_blocks, int64_t max_free,
                         const int32_t *n_free, int32_t *seq_lens, int32_t *q_start, int64_t *slot_mapping,
                         int32_t *positions, int64_t n_tokens, int32_t *n_free_out, void *stream);

/*
 * Rotary positions.  A handle holds the angles by which the pairs of a head are
 * turned: pair i of a row at position p by p * freqs[i] radians, and the pair's
 * length is multiplied by `amplitude`.  The first rot_dim coordinates are
 * rotated, the rest is passed on.
 *
 * isoq_rope_init -- build a handle on the current device.
 *   d           width of a head, 1 .. 1024.
 *   rot_dim     coordinates that are rotated: even, 0 .. d.
 *   layout      ISOQ_ROPE_PAIRS: pair i is coordinates (2 i, 2 i + 1);
 *               ISOQ_ROPE_HALVES: (i, rot_dim / 2 + i).
 *   freqs       host, rot_dim / 2 doubles (isoq_rope_freqs, or others).
 *   amplitude   finite (1 leaves lengths as they are).
 * isoq_rope_freqs -- host only: base^(-2 i / rot_dim) for i < rot_dim / 2, slowed
 * down for contexts that are `factor` times longer than the `original` positions:
 * a pair that turns at most `low` times in those by `factor`, one that turns at
 * least `high` times not at all, between them blended linearly in the number of
 * turns.  factor 1: as they are; original 0: every pair by factor.
 */
enum { ISOQ_ROPE_PAIRS = 0, ISOQ_ROPE_HALVES = 1 };
typedef struct isoq_rope isoq_rope;
isoq_status isoq_rope_init(isoq_rope **out, int d, int rot_dim, int layout, const double *freqs, double amplitude);
isoq_status isoq_rope_destroy(isoq_rope *r);
isoq_status isoq_rope_freqs(int rot_dim, double base, double factor, double original, double low, double high,
                            double *out);

/*
 * isoq_qk_norm_rope -- norms and rotary positions of new tokens' queries and keys
 * in one pass: each row (a head of a token) becomes
 *     y = weight * x / sqrt(mean(x^2) + eps)     (where there is a weight)
 * and its rotated pairs are turned by the angles of the token's position.  q_out
 * is what isoq_kv_attn takes, k_out what isoq_kv_append takes.
 *
 *   dtype       ISOQ_F16 or ISOQ_F32, the element type of q, k, q_out and k_out.
 *   q, k        device, token t's heads at q + t * q_stride (k + t * k_stride)
 *               elements, one after another: a part of a projection's output that
 *               holds queries, keys and values may be passed as it is.  Aligned to
 *               their elements; 16 bytes, with strides and widths that are
 *               multiples of as much, are faster.  n_q_heads or n_kv_heads may be 0.
 *   positions   device, int32 [n_tokens], any value (negative ones turn back).
 *               Angles are exact to 2^-31 of a turn at every position, for frequencies
 *               of up to a turn (2 pi) a position; for k turns, to k + 1 times that.
 *   q_weight, k_weight  device, fp32 [d], or NULL: no norm.
 *   q_out, k_out  device, [n_tokens][heads][d] (16-byte aligned); may be q (k)
 *               itself where its stride is n_q_heads * d (n_kv_heads * d).
 * Arithmetic: fp32, rounded once (fp16: to nearest even); a normed row whose squares add up
 * past fp32's largest number (fp32 values from 5e17 on can) is 0.  Limits: n_tokens *
 * (n_q_heads + n_kv_heads) < 2^31, heads <= 65535.
 */
isoq_status isoq_qk_norm_rope(const isoq_rope *r, int dtype, const void *q, int64_t q_stride, int n_q_heads,
                              const void *k, int64_t k_stride, int n_kv_heads, const int32_t *positions,
                              int64_t n_tokens, const float *q_weight, const float *k_weight, float eps, void *q_out,
                              void *k_out, void *stream);

/* Sizes: bytes of one packed index record, ceil(pw * bits / 8) with the
 * padded width pw = 4 g4 (Full, Fast) or 2 g2 (2-D); isoq_packed_bytes is
 * ceil(d * bits / 8), the same number whenever d is a multiple of 4.  Raw
 * draws per set for rot_host (Full 8 g4, Fast 4 g4, 2-D g2); exported
 * parameters per set (Full 8 g4, Fast 4 g4, 2-D 2 g2), with g4 = ceil(d/4),
 * g2 = ceil(d/2).  Return 0 for invalid arguments. */
size_t isoq_record_bytes(int variant, int d, int bits);
size_t isoq_packed_bytes(int d, int bits);
size_t isoq_raw_params_per_set(int variant, int d);
size_t isoq_export_params_per_set(int variant, int d);

/*
 * Host-only helpers (no device needed), the same computations init performs:
 *   isoq_codebook_lloyd   2^bits Lloyd-Max levels for N(0, 1/d) after `iters`
 *                         iterations (see isoq_params_init), as doubles.
 *   isoq_rotation_draws   the seeded raw draws init uses when rot_host is NULL,
 *                         n_sets * isoq_raw_params_per_set doubles.
 */
isoq_status isoq_codebook_lloyd(int bits, int d, int iters, double *levels_out);
isoq_status isoq_rotation_draws(int variant, int d, int n_sets, uint64_t seed, double *out);

/* Static text for a status code. */
const char *isoq_status_string(isoq_status s);

/* The HIP call and error text behind the last ISOQ_E_HIP (or a hipMalloc
 * ISOQ_E_NOMEM) returned on the calling thread; "" if none.  Valid until the
 * next call on the same thread. */
const char *isoq_last_hip_error(void);

#ifdef __cplusplus
}
#endif

#endif /* ISOQUANT_H */
