/*
 * spec_prompt.h -- whole prompts through a bf16 decoder: the operators of a layer over packed rows of several sequences, on the
 * weights that spec_pack_weight lays out and into the cache of a spec_verify.h handle, which then decodes from there.
 * Normalised rows, products with bias, activation and residual, rotary embedding with the cache's new keys and
 * values, causal attention.
 *
 * Conventions as in spec_verify.h: device pointers, work queued on the given stream and not synchronised,
 * nothing allocated, negative spec_status on failure, host-checkable arguments checked before any launch.
 * Every call may be recorded into a HIP graph.  Buffers that overlap are an error unless said otherwise.
 *
 * Packed rows: sequence b has rows row0[b] .. row0[b+1]-1 of a tensor (device int32[batch+1], ascending from 0 or more; what lies
 * outside [0, rows) counts as cut off, a pair that descends as no rows).  Rows of no sequence are neither read nor written.  Where
 * numbers that do not ascend make sequences overlap, nothing outside the tensors is touched, but which rows are computed, and with which results,
 * is not defined.
 */
#ifndef SPEC_PROMPT_H
#define SPEC_PROMPT_H

#include <stddef.h>
#include <stdint.h>

#include "spec_verify.h"

#ifdef __cplusplus
extern "C" {
#endif

#define SPEC_PROMPT_MAX_COLS 65536       /* widest row of spec_prompt_rmsnorm */
#define SPEC_PROMPT_MAX_ROWS (1 << 20)   /* of spec_prompt_rmsnorm and spec_prompt_gemm, at most */
#define SPEC_PROMPT_MAX_LD (1 << 22)     /* elements from a row to the next, at most */
#define SPEC_PROMPT_MAX_SEQS 65536

/* y bf16 [rows][cols] (contiguous) = x / sqrt(mean(x^2) + eps) * gain.  x: SPEC_DTYPE_FP32 or SPEC_DTYPE_BF16, rows ld elements apart
 * (ld >= cols); gain fp32[cols].  Sums are fp32, also of rows whose squares are not.  cols <= SPEC_PROMPT_MAX_COLS.  Pointers as aligned
 * as their elements. */
int spec_prompt_rmsnorm(const void* x, int32_t x_dtype, int64_t ld, const float* gain, float eps, int32_t rows, int32_t cols, void* y,
                        void* stream);

/* y [M][N] = residual + act(x W^T + bias), in fp32, rounded once to y_dtype (SPEC_DTYPE_FP32 or SPEC_DTYPE_BF16).
 * x: bf16 [M][K], rows ld_x elements apart (a multiple of 8), 16-byte aligned.  w_packed: W [N][K] as spec_pack_weight lays it out, so K is
 * a multiple of 32.  y: rows ld_y elements apart.  Sums are fp32; M = 0 does nothing.
 * SPEC_ACT_SWIGLU: W has 2 N rows, gate rows and then up rows, packed with interleave_halves (N is a multiple of 16);
 * y = silu(gate) * up. */
#define SPEC_ACT_NONE 0
#define SPEC_ACT_RELU 1     /* max(v, 0) */
#define SPEC_ACT_GELU 2     /* v * (1 + erf(v / sqrt(2))) / 2, off by 5e-7 |v| at most */
#define SPEC_ACT_SILU 3     /* v / (1 + exp(-v)); off by (2^-20 + |v| 2^-23) of itself, or 1e-30, at most */
#define SPEC_ACT_SWIGLU 4
typedef struct {
    const float* bias;         /* device fp32[N] (SPEC_ACT_SWIGLU: [2 N], gate then up), or NULL */
    const void* residual;      /* device [M][N], or NULL; may be y, with its type and ld */
    int64_t ld_residual;
    int32_t residual_dtype;
    int32_t activation;        /* SPEC_ACT_* */
} spec_prompt_epilogue;
/* epilogue NULL: none of it.  workspace: device scratch, 16-byte aligned, through which few rows share K out among workgroups; with less
 * than spec_prompt_gemm_workspace_bytes (0 where that would not pay) they do so less, or not (NULL: none).  Calls that overlap in time need
 * their own. */
size_t spec_prompt_gemm_workspace_bytes(int32_t M, int32_t N, int32_t K, int32_t activation);
/* The most of that over all numbers of rows up to M (many rows need none where few do): for a workspace that calls of different M use. */
size_t spec_prompt_gemm_workspace_bytes_up_to(int32_t M, int32_t N, int32_t K, int32_t activation);
int spec_prompt_gemm(const void* x, int64_t ld_x, const void* w_packed, const spec_prompt_epilogue* epilogue, void* y, int32_t y_dtype,
                     int64_t ld_y, int32_t M, int32_t N, int32_t K, void* workspace, size_t workspace_bytes, void* stream);

/* The rotary embedding of a layer's queries and keys, and its keys and values into the handle's cache (bf16 models).
 * qkv: bf16 [rows][(n_q_heads + 2 n_kv_heads) * head_dim] of the handle's model: query heads, key heads, value heads; rows ld_qkv elements apart.
 * Row row0[b] + j is at position pos0[b] + j (pos0 NULL: j) of slot seq_slot[b] (device int32[batch] both).
 * rotated: bf16 [rows][(n_q_heads + n_kv_heads) * head_dim], rows ld_rotated elements apart: the queries and keys, rotated in fp32 and rounded
 * once; the same keys, and the values, go to the cache.  rotated may be qkv with its ld (one row: any): they are then rotated in place.
 * kv_len is neither read nor changed: the caller sets it once all layers are in.  A sequence whose slot is outside [0, max_batch), or
 * whose positions leave [0, max_kv_len), is not written to the cache, its rotated rows are zero and spec_verify_poll reports
 * it (SPEC_ERR_INVALID_ARG, SPEC_ERR_KV_OVERFLOW).  A paged cache takes the pages that it lacks up to the last new position; where the
 * pool runs dry the rest is not written (SPEC_ERR_KV_OVERFLOW).  A slot may be named twice if the positions differ.  batch: at most the
 * model's max_batch.
 * Base addresses 16-byte aligned, lds multiples of 8. */
struct spec_handle;
int spec_prompt_append(spec_handle* h, int32_t layer, const void* qkv, int64_t ld_qkv, void* rotated, int64_t ld_rotated,
                       const int32_t* row0, const int32_t* seq_slot, const int32_t* pos0, int32_t batch, int32_t rows, void* stream);

/* Causal attention over packed sequences: out[i] = sum over t of softmax_t(scale * q_i . k_t) v_t, where row j of a sequence's len_q query rows
 * sees its key rows 0 .. len_k - len_q + j (len_k = len_q: a whole prompt; len_q = 1: a single token behind len_k - 1 older ones).  A row
 * that sees nothing is zero.  A position that a row does not see adds nothing to it, whatever lies there.  Older keys and values are packed rows that
 * the caller has kept: those in a handle's cache lie in another order (spec_verify_step and spec_kv_export read them).
 * All bf16; rows ld elements apart (multiples of 8; addresses 16-byte aligned).  q, out [q_rows][n_q_heads * head_dim], k, v
 * [k_rows][n_kv_heads * head_dim]; n_q_heads is a multiple of n_kv_heads and query head h reads kv head h / (n_q_heads / n_kv_heads); head_dim 64 or
 * 128.  Scores, softmax and sums are fp32; the weights are rounded to bf16 where they meet the values, which leaves the result some 0.0020 of its size
 * off where rounding it alone leaves 0.0016 (root mean square).
 * max_q_len, max_k_len: the longest sequences that the caller expects (0: unknown).  They and the workspace (device scratch, 16-byte
 * aligned; NULL or too little: none) decide only how the work is split.  Calls that overlap in time need a workspace of their own. */
typedef struct {
    const void *q, *k, *v;
    int64_t ld_q, ld_k, ld_v, ld_out;
    const int32_t* q_row0;     /* device int32[batch+1] */
    const int32_t* k_row0;     /* device int32[batch+1], or NULL: q_row0 (k_rows is then q_rows) */
    int32_t n_q_heads, n_kv_heads, head_dim;
    int32_t batch, q_rows, k_rows;
    int32_t max_q_len, max_k_len;
    float scale;               /* |scale| log2(e) a finite float */
    void* out;
} spec_prompt_attn_args;
size_t spec_prompt_attention_workspace_bytes(int32_t q_rows, int32_t batch, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim);
/* At least that for any numbers of rows and sequences up to these; 2^20 (head_dim + 2) bytes at most. */
size_t spec_prompt_attention_workspace_bytes_up_to(int32_t q_rows, int32_t batch, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim);
int spec_prompt_attention(const spec_prompt_attn_args* args, void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif
