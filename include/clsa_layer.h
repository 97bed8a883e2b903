/*
 * clsa_layer.h -- what a decoder layer runs around its cache (NVIDIA B200, sm_100a).
 *
 * Part of the library that clsa.h declares: the conventions stated there (pointers, ownership, errors, streams, dtypes,
 * paged caches) hold here too. Four operators:
 *
 *   clsa_add_norm        the residual's addition and an RMS norm of the sum, the result in bf16 and/or in 8 bits with scales
 *   clsa_norm_rope_axes  clsa_norm_rope with positions on several axes (time, height, width, ..)
 *   clsa_dense_attn      attention of the newest tokens over every cached token, or over the last `window` ones (bf16 caches)
 *   clsa_dense_attn8     the same over the 8-bit caches of clsa_cache8.h
 */
#ifndef CLSA_LAYER_H_
#define CLSA_LAYER_H_

#include "clsa_cache8.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- attention over a whole cache, or its last tokens ------------------------------------------------------------ */

/* Bytes of workspace that clsa_dense_attn and clsa_dense_attn8 may need for these params (any window). 256-byte aligned; its first 256
 * bytes (the status word) zero before the first use, the rest needs no clearing. It may be one with the workspace of the calls of
 * clsa_cache8.h (give it the larger size, all of it zero before its first use) and of clsa_topk, but not with that of the other calls of
 * clsa.h, nor be shared by calls that overlap on the GPU. Reads the scalar fields of p only. *bytes is HOST memory. */
CLSA_API clsa_status clsa_dense_workspace_bytes(const clsa_params* p, size_t* bytes);

/* For each sequence b, query t (of T = q_per_seq) and query head h with KV head g = h / (Hq/Hkv),
 *   O = sum_s softmax_s(sm_scale * Q[b][t][h] . K[s][g]) V[s][g]   over the visible positions s:
 *     window == 0, causal == 0   all s < seq_len[b]. Here seq_len[b] may be anything from 0 on: the queries need not be in the cache
 *                                (cross attention to states of another length, empty places of a batch)
 *     causal == 1                s <= seq_len[b] - T + t
 *     window  > 0                s >  seq_len[b] - T + t - window  as well: the query's own position and the window - 1 before it
 *   q   bf16 [B][T][Hq][D], 16-byte aligned;  out  bf16 [B][T][Hq][D], 16-byte aligned, rounded from fp32. Weights meet V in 16 bits (two
 *       bf16) for up to 32 query columns (T * Hq/Hkv) of a KV head, in one bf16 for more: off by up to 2^-16 and 2^-8 of each
 *   lse fp32 [B][T][Hq] or NULL: log-sum-exp of the scaled logits (natural log); with it, results over two parts of a context join
 * A query that sees nothing yields zeros and lse = -inf. What lies in cache rows that a query does not see (rows behind the sequence,
 * in front of its window, other pages' rows) never reaches its result, NaN and infinities included. A NaN or an infinite logit among
 * the visible ones gives NaN, a logit of -inf has weight 0; an element of V that is not finite makes those outputs that see it not finite.
 * Sums over V are divided by the weights' sum at their end: V's magnitudes times the rows seen stay below 2^119.
 * T <= 32 and T * Hq/Hkv <= 512; groups up to 16; D == 128. p->num_cache_rows, the extent of the row space, is required: a row
 * outside it, or of a page outside it, counts as not visible and flags CLSA_DEV_BAD_INDEX. A sequence with seq_len > max_seq_len or < T
 * (< 0 where window == 0 and causal == 0) counts as empty and flags CLSA_DEV_BAD_SEQLEN. idx_dim, top_k and the indexer's cache are not
 * used. Results are the same from call to call.
 * Up to 32 query tokens share one pass over the cache: made for decoding and drafted tokens, not for prefill chunks. */
CLSA_API clsa_status clsa_dense_attn(const clsa_params* p, int32_t window, const void* q, void* out, float* lse, void* workspace,
                                     size_t workspace_bytes, clsa_stream stream);

/* clsa_dense_attn over an 8-bit cache (its K and V; a sequence begins on a multiple of 16 rows, as every scale block makes it: flagged
 * CLSA_DEV_BAD_SCALE_BLOCK and counted as empty otherwise). Logits may have any size that is a float, for queries of magnitudes below
 * 2^118 / sm_scale; a query's elements below 2^-31 of its head's largest round to f16's last place. Weights meet V in f16: off by up to 2^-11
 * of each, and by up to 2^-36 of the largest weight times its V's scale. Scale bytes are fetched by the aligned words of 4 that they lie in: up to
 * 3 bytes in front of the first one are read (and not used), none behind the last. */
CLSA_API clsa_status clsa_dense_attn8(const clsa_params* p, const clsa_cache8* c, int32_t window, const void* q, void* out, float* lse,
                                      void* workspace, size_t workspace_bytes, clsa_stream stream);

/* ---- residual addition and RMS norm ------------------------------------------------------------------------------- */

/* Rows of a matrix: element (r, i) at data[r * stride + i] in the array's own elements. data 16-byte aligned (scales: 1), rows
 * beginning on multiples of 16 bytes (scales: 1). stride >= the row's length, or 0 for an input row that every row shares. */
typedef struct {
  void* data;
  int64_t stride;
} clsa_rows;

/* What clsa_add_norm computes for each row:
 *   s = x + residual                                      (fp32)
 *   y = s * (mean_i s_i^2 + eps)^(-1/2) * weight          (fp32, of the unrounded s; weight NULL = ones)
 * and, with scale_group > 0, per group of scale_group consecutive elements
 *   e = the smallest exponent in -100 .. 120 with max |y| <= 448 * 2^e over the group's finite elements (-100 if all are zero),
 *   code = y * 2^-e as e4m3, rounded to nearest even, saturating (an infinity becomes +-448, a NaN stays one), scale byte e + 127:
 * the format of clsa_cache8.h, of y itself (no rounding to bf16 in between). */
typedef struct {
  int32_t dim;         /* elements of a row: a multiple of 16, 16 .. 16384 */
  float eps;           /* >= 0, finite */
  const void* weight;  /* bf16 [dim] or NULL, 16-byte aligned */
  int32_t scale_group; /* 0 (no codes), 32, 64, 128 (dividing dim) or dim */
} clsa_add_norm_spec;

/* num_rows rows in one launch:
 *   x, residual  bf16; residual NULL: s = x
 *   sum_out      bf16, s rounded to nearest even; NULL: not wanted. May be x or residual itself (same data and stride)
 *   y_out        bf16, y rounded to nearest even; NULL: not wanted. May be x or residual itself, where sum_out is not
 *   codes_out    e4m3 [num_rows][dim], scales_out  bytes [num_rows][dim / scale_group]: both, with scale_group > 0, or neither
 * Beyond that no output shares memory with another argument: such calls are refused (rows of different distances in bytes count as all that lies
 * between the first and the last of them).
 * At least one of y_out and codes_out is given. num_rows 0 .. 2^30; 0 does nothing. Squares are summed in fp32: magnitudes above about
 * 1e17 overflow the norm. */
CLSA_API clsa_status clsa_add_norm(const clsa_add_norm_spec* spec, int32_t num_rows, const clsa_rows* x, const clsa_rows* residual,
                                   const clsa_rows* sum_out, const clsa_rows* y_out, const clsa_rows* codes_out,
                                   const clsa_rows* scales_out, clsa_stream stream);

/* ---- positions on several axes -------------------------------------------------------------------------------------- */

#define CLSA_MAX_AXES 4

/* Which axis' position turns pair i of a head (HOST memory, read during the call): its angle is position[axis_of_pair[i]] * inv_freq[i].
 * Runs of pairs per axis and axes in turn are both described so. */
typedef struct {
  int32_t num_axes;          /* 1 .. CLSA_MAX_AXES */
  uint8_t axis_of_pair[128]; /* [rot_dim / 2], each < num_axes */
} clsa_rope_axes;

/* clsa_norm_rope with num_axes positions per token, each a signed 32-bit number: position of token i on axis a at
 * positions[a * axis_stride + i] (axis_stride >= num_tokens, or 0: one position serves every axis). A token whose position on axis 0 is
 * negative is skipped, its outputs left as they were; the other axes' positions may be negative. Everything else as there (spec, heads,
 * overlaps, num_tokens); spec->rot_dim > 0. With equal positions on all axes the results are those of clsa_norm_rope, bit for bit. */
CLSA_API clsa_status clsa_norm_rope_axes(const clsa_norm_rope_spec* spec, const clsa_rope_axes* axes, int32_t num_tokens,
                                         const int32_t* positions, int64_t axis_stride, const clsa_heads* q, const clsa_heads* q_out,
                                         const clsa_heads* k, const clsa_heads* k_out, clsa_stream stream);

#ifdef __cplusplus
}
#endif
#endif /* CLSA_LAYER_H_ */
