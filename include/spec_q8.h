/*
 * spec_q8.h -- operators of a decode step held in 8 bits, and the draw from a filtered distribution, for
 * callers that run a decoder layer themselves: rows to 8 bits (plain, behind a residual addition and RMSNorm,
 * behind SwiGLU), the product of such rows with 8-bit weights, a paged 8-bit KV cache with the attention that
 * reads it, and temperature / top-k / top-p / min-p sampling, whose filtered rows spec_verify_step takes.
 *
 * Conventions as in spec_verify.h: device pointers, work queued on the given stream and not synchronised,
 * nothing allocated, negative spec_status on failure, host-checkable arguments checked before any launch.
 * Every call may be recorded into a HIP graph.  Buffers that overlap are an error unless said otherwise.
 *
 * 8-bit numbers are OCP e4m3 (largest 448, no infinity, NaN 0x7f/0xff), rounded to nearest even.  What they
 * stand for is the number times the scale of its block:
 *
 *   rows     q [M][Kp] with Kp = cols rounded up to a multiple of 128, zero beyond cols;
 *            scales fp32 [Kp/128][M], one for each row and 128 columns: amax / 448, at least 2^-126.  A block
 *            that holds a NaN or an infinity stands for NaN throughout.
 *   weights  [n_out][n_in] in the tile order of spec_q8_pack_weight; scales fp32 [ceil(n_out/128)][Kp/128], one
 *            for each 128 x 128 block.
 *   cache    see spec_kv8_cache.
 */
#ifndef SPEC_Q8_H
#define SPEC_Q8_H

#include <stddef.h>
#include <stdint.h>

#include "spec_verify.h"

#ifdef __cplusplus
extern "C" {
#endif

#define SPEC_Q8_BLOCK 128            /* columns that share a scale */
#define SPEC_Q8_MAX_COLS 65536       /* widest row of spec_q8_add_rmsnorm */
#define SPEC_KV8_PAGE 32             /* positions of a cache page */
#define SPEC_FILTER_MAX_VOCAB 262144

/* Types are SPEC_DTYPE_FP32 or SPEC_DTYPE_BF16.  q, packed matrices and the product's y 16-byte aligned; everything else as its element
 * type asks.  Columns, n_out and n_in: at most 2^30 (SPEC_ERR_SHAPE beyond).  rows = 0 does nothing. */

/* q, scales = the rows of x [rows][cols], ld elements apart (ld >= cols). */
int spec_q8_quantize(const void* x, int32_t x_dtype, int64_t ld, int32_t rows, int32_t cols, void* q, float* scales,
                     void* stream);

/* h = x + delta (delta NULL: h = x); x_out = h rounded to x's type (x_out may be x, or NULL: not written);
 * q, scales = h / sqrt(mean(h^2) + eps) * gain, taken from the fp32 sum.  x, x_out, delta: [rows][cols], contiguous.
 * cols <= SPEC_Q8_MAX_COLS. */
int spec_q8_add_rmsnorm(const void* x, int32_t x_dtype, const void* delta, int32_t delta_dtype, const float* gain,
                        float eps, int32_t rows, int32_t cols, void* x_out, void* q, float* scales, void* stream);

/* q, scales = silu(gate) * up of gate_up [rows][2 d_ffn]: d_ffn gate columns, then d_ffn up columns. */
int spec_q8_swiglu(const void* gate_up, int32_t dtype, int32_t rows, int32_t d_ffn, void* q, float* scales, void* stream);

/* Bytes of a packed [n_out][n_in] matrix of 8-bit numbers: n_out rounded up to 16, n_in to 128 (0: no such matrix). */
size_t spec_q8_packed_weight_bytes(int32_t n_out, int32_t n_in);

/* Row-major e4m3 [n_out][n_in] -> the order the product reads.  Tile (kb, j) holds out features 16j..16j+15 and in
 * features 128kb..128kb+127 in 2048 bytes; element (h, g, n, e) of [2][4][16][16] is
 * W[16j + n][128kb + 64h + 16g + e], so that a wavefront fetches the operand of one 16x16x128 matrix instruction
 * with two 16-byte loads per lane.  Tiles are ordered [kb][j].  Beyond n_out and n_in: zero. */
int spec_q8_pack_weight(const void* src, void* dst_packed, int32_t n_out, int32_t n_in, void* stream);

/* y [M][N] (contiguous) = sum over blocks kb of scales[kb][m] * w_scales[n/128][kb] * (q's block . w's block):
 * the sums over blocks in fp32, y rounded once to y_dtype.  q: [M][Kp], M <= 1048560; K is the row length before padding.  The
 * two scales of a block are multiplied first: their product is meant to be a normal fp32 number.
 * Within a block: for fp32 y products are exact and their sum is fp32.  For bf16 y it is one fp8 matrix instruction, at twice the rate, which cuts
 * off each of eight neighbouring products at 2^-13 of the largest of them; all in all that is less than 2^-10 of the sum of the magnitudes
 * of the products (the numbers that are multiplied were rounded by up to 2^-4).  Callers whose sums cancel and who want what is left ask for fp32. */
int spec_q8_gemm(const void* q, const float* scales, const void* w_packed, const float* w_scales, void* y, int32_t y_dtype,
                 int32_t M, int32_t N, int32_t K, void* stream);

/* A paged cache of one layer.  A page holds 32 positions of every kv head:
 *   data    [n_pages][n_kv_heads][2][32 * head_dim] e4m3: keys, then values.  Key (t, d) of a page is byte
 *           [t/16][d/16][t%16][d%16], value (t, d) is byte [d/32][(t%16)/4][d%16][(d%32)/16][t/16][t%4]: the orders in
 *           which the two matrix products of the attention take them, 16 bytes per lane.
 *   scales  fp32 [n_pages][n_kv_heads][2], one for a page's keys of a head and one for its values.  spec_kv8_append
 *           makes them powers of two, so that a scale that has to grow costs the older positions of a page nothing
 *           but what falls below the smallest e4m3 number; spec_kv8_attention takes any positive scale.
 *   table   int32 [batch][blocks_per_seq]: the page of positions 32i .. 32i+31 of a sequence.
 * Positions whose page number is outside [0, n_pages) are neither written nor attended to.  No two sequences may name
 * the same page where spec_kv8_append writes.  data 16-byte aligned; head_dim 64 or 128. */
typedef struct {
    void* data;
    float* scales;
    const int32_t* table;
    int32_t n_pages, n_kv_heads, head_dim, batch, blocks_per_seq;
} spec_kv8_cache;

/* The windows of a step: sequence b has rows row0[b] .. row0[b+1]-1 (device int32[batch+1], ascending from 0, at most
 * `rows` in all, at most max_window in one sequence) at positions kv_len[b] + 0, 1, ... (device int32[batch], read and
 * not changed: the caller advances it by what it keeps).
 *
 * qkv: bf16 [rows][(n_q_heads + 2 n_kv_heads) * head_dim]: query heads, key heads, value heads.  cos_sin: fp32
 * [max_pos][head_dim/2][2], dimension i paired with i + head_dim/2; NULL: no rotation.  q_out: bf16
 * [rows][n_q_heads * head_dim], the rotated queries (NULL only without a rotation: they are then left in qkv).
 * Keys (rotated, in fp32) and values are rounded to 8 bits once.  A page's scale is set by its new positions where
 * it holds no older one (position < kv_len), else it never shrinks; when it grows, the older positions are rounded
 * again.  A NaN or an infinity is stored as NaN and does not touch the scale.
 * A row whose position is negative, beyond the table or beyond max_pos is not written, and its q_out row is zero.  qkv and
 * q_out 16-byte aligned, cos_sin 8-byte. */
int spec_kv8_append(const spec_kv8_cache* cache, const void* qkv, int32_t n_q_heads, const int32_t* row0,
                    const int32_t* kv_len, int32_t rows, int32_t max_window, const float* cos_sin, int32_t max_pos,
                    void* q_out, void* stream);

/* out bf16 [rows][n_q_heads * head_dim] = softmax(scale * q . k) v, row j of a window over positions 0 .. kv_len[b] + j.
 * q: bf16, rows ld_q elements apart (a multiple of 8, and q 16-byte aligned).  A row that sees no position (a negative
 * kv_len, no valid page) is zero.  A position that a row does not see adds nothing to it, whatever the cache holds there.  Scores, weights
 * and sums are fp32, the weights that meet the values fp16 (eleven bits, of which out keeps eight); a value scale below 2^-80
 * counts as 2^-80.  Rows of no sequence are not written.  out 16-byte aligned.  max_len: the largest kv_len + window that the
 * caller expects; it decides only how the work is split (0: the table's capacity).  workspace: device scratch for the
 * parts of long sequences, 16-byte aligned; with less than spec_kv8_workspace_bytes fewer parts are made (NULL: none). */
size_t spec_kv8_workspace_bytes(int32_t rows, int32_t n_q_heads, int32_t head_dim);
int spec_kv8_attention(const spec_kv8_cache* cache, const void* q, int64_t ld_q, int32_t n_q_heads, const int32_t* row0,
                       const int32_t* kv_len, int32_t rows, int32_t max_window, int32_t max_len, float scale, void* out,
                       void* workspace, size_t workspace_bytes, void* stream);

/* Filtered draws.  Row r of logits ([rows][vocab], ld elements apart): with m the largest logit, token i has the mass
 *     w_i = floor(2^44 exp((l_i - m) / temperature[r]))
 * -- whole numbers, so that every sum below is exact and no result depends on the order of a sum.  Tokens are ranked by
 * falling logit, equal ones by rising id.  A token is kept if it has mass and
 *     top_k:  its rank is below top_k[r]                                                    (top_k[r] <= 0: all)
 *     top_p:  the mass ranked before it is below top_p[r] times the mass that top_k leaves   (top_p[r] >= 1: all)
 *     min_p:  its mass is at least min_p[r] times the largest                                (min_p[r] <= 0: all)
 * (the first token always is).  temperature[r] <= 0 (or NaN) keeps the first token alone, one between 0 and 2^-126 counts as 2^-126, an
 * infinite one as fp32's largest number, a difference of logits that fp32 does not hold as infinite; a NaN in top_p or min_p keeps all.  The token drawn is the first id whose
 * inclusive prefix sum of kept masses exceeds floor(uniforms[r] * kept mass).  Excluded logits may be -inf; a row
 * with a NaN, a +inf or no finite logit gives token -1, n_kept 0, logprob NaN and a filtered row of -inf. */
typedef struct {
    const void* logits;          /* device dtype[rows][vocab] */
    int32_t dtype, rows, vocab;  /* vocab <= SPEC_FILTER_MAX_VOCAB */
    int64_t ld;                  /* elements from a row to the next, >= vocab */
    const float* uniforms;       /* device fp32[rows] in [0, 1) */
    const float* temperature;    /* device fp32[rows]; NULL: 1 */
    const int32_t* top_k;        /* device int32[rows], or NULL */
    const float* top_p;          /* device fp32[rows], or NULL */
    const float* min_p;          /* device fp32[rows], or NULL */
} spec_filter_args;

typedef struct {
    int32_t* tokens;             /* device int32[rows] */
    float* logprob;              /* device fp32[rows], or NULL: log of the drawn token's share of the kept mass */
    int32_t* n_kept;             /* device int32[rows], or NULL */
    float* logits_out;           /* device fp32[rows][vocab], or NULL: the logits, -inf where not kept */
} spec_filter_out;

/* workspace: device scratch, 16-byte aligned, through which calls without top_k share a row out among workgroups; with less than
 * spec_filter_workspace_bytes (0 where that would not pay) a row is one workgroup's (NULL: none).  Calls that overlap in time need
 * their own. */
size_t spec_filter_workspace_bytes(int32_t rows, int32_t vocab);
int spec_filter_sample(const spec_filter_args* args, const spec_filter_out* out, void* workspace, size_t workspace_bytes,
                       void* stream);

#ifdef __cplusplus
}
#endif
#endif
