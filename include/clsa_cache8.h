/*
 * clsa_cache8.h -- caches held in 8 bits: what fills them and what reads them (NVIDIA B200, sm_100a).
 *
 * Part of the library that clsa.h declares: the conventions stated there (pointers, ownership, errors, streams, dtypes,
 * visibility, the index contract, paged caches) hold here too. Four operators:
 *
 *   clsa_norm_rope       RMS norm of each query and key head and the position rotation, in one pass (bf16 -> bf16)
 *   clsa_cache8_append   the newest tokens' K (optionally normed and rotated in the same pass), V and K_idx rows into the
 *                        8-bit caches
 *   clsa_index_scores8   Eq. 3's scores over 8-bit indexer keys (then clsa_topk, as it is)
 *   clsa_sparse_attn8    Eq. 4 for one layer over the selected rows of the 8-bit K and V caches
 *
 * The format. A cache holds e4m3 codes (1 sign, 4 exponent, 3 mantissa bits, largest finite value 448) and, for each block of
 * `scale_block` consecutive cache rows and each KV head, one scale byte x that stands for the power of two 2^(x - 127)
 * (the e8m0 format); the value of an element is code * 2^(x - 127). K and V have scales of their own; K_idx has one per block.
 * Scale bytes lie in 27 .. 247 (2^-100 .. 2^120); a byte outside is read as the nearest of these. Scales are powers of two so
 * that a block whose largest magnitude grows is re-coded by moving exponents (exact except where a code becomes subnormal),
 * and so that applying a scale never rounds.
 */
#ifndef CLSA_CACHE8_H_
#define CLSA_CACHE8_H_

#include "clsa.h"

#ifdef __cplusplus
extern "C" {
#endif

#define CLSA_DEV_BAD_SCALE_BLOCK 64u /* clsa_cache8_append, clsa_index_scores8: seq_start[b] is not a multiple of scale_block: that
                                        sequence was not appended to, its scores mean nothing */

/* Heads of a run of tokens: element (token, head, d) at data[token * token_stride + head * head_stride + d], bf16. Slices of
 * a projection's output rows are described as they are. data 16-byte aligned, strides (in elements) multiples of 8,
 * head_stride >= the head dimension. token_stride >= 0: 0 reads one row for every token (inputs only). */
typedef struct {
  void* data;
  int32_t num_heads; /* 1 .. 1024 */
  int64_t token_stride;
  int64_t head_stride;
} clsa_heads;

/* What clsa_norm_rope computes for each head x[0 .. D) of a token at position `pos`:
 *   y = norm ? x * (mean_d x_d^2 + eps)^(-1/2) * weight : x                    (fp32; weight NULL = ones)
 *   z: for each i < rot_dim / 2 the pair (y_a, y_b) turned by the angle pos * inv_freq[i], both parts times rot_scale,
 *      z_a = (y_a cos - y_b sin) rot_scale,  z_b = (y_b cos + y_a sin) rot_scale,
 *      (a, b) = (i, i + rot_dim / 2), or (2i, 2i + 1) with interleaved; dimensions from rot_dim on are y's.
 * Angles are formed and reduced in 64 bits (pos * inv_freq exceeds what fp32 resolves at long contexts). */
typedef struct {
  int32_t head_dim;      /* D: 64, 128 or 256 */
  int32_t norm;          /* 0 or 1 */
  float eps;             /* >= 0, finite */
  int32_t rot_dim;       /* 0 (no rotation) .. head_dim, a multiple of 16 */
  int32_t interleaved;   /* 0 or 1 */
  float rot_scale;       /* finite; 1 unless the model scales its rotations */
  const float* inv_freq; /* fp32 [rot_dim / 2]; may be NULL when rot_dim == 0 */
  const void* q_weight;  /* bf16 [head_dim] or NULL, 16-byte aligned */
  const void* k_weight;  /* bf16 [head_dim] or NULL, 16-byte aligned */
} clsa_norm_rope_spec;

/* Norm and rotation of the query and key heads of num_tokens tokens in one launch, rounded once to bf16.
 *   positions  int32 [num_tokens], < 2^31; a token with a negative position is skipped, its outputs left as they were
 *              (padding). NULL when rot_dim == 0 and no token is to be skipped.
 *   q, q_out   the queries and where their results go, same num_heads (both NULL: no queries)
 *   k, k_out   the keys, likewise
 * An output may be its own input (same data and strides); other overlaps are not allowed. num_tokens 0 .. 2^30; 0 is a
 * call that does nothing (its pointers may be NULL then). Squares are summed in fp32: magnitudes above about 1e18 overflow the
 * norm, and with eps == 0 a row of magnitudes below about 1e-19 underflows it. */
CLSA_API clsa_status clsa_norm_rope(const clsa_norm_rope_spec* spec, int32_t num_tokens, const int32_t* positions,
                                    const clsa_heads* q, const clsa_heads* q_out, const clsa_heads* k,
                                    const clsa_heads* k_out, clsa_stream stream);

/* An 8-bit cache. Rows are those of clsa_params (seq_start / seq_len or a block table); a sequence begins on a scale block (in a
 * contiguous cache every seq_start is a multiple of scale_block); p->num_cache_rows, the extent of the
 * row space, is required by every call below, and a row at or beyond it is treated like an index outside its sequence.
 * p's own bf16 cache pointers and strides are not used. */
typedef struct {
  void* k;       /* e4m3 [rows][Hkv][D], element (r,g,d) at byte r*kv_token_stride + g*kv_head_stride + d; 16-byte aligned */
  void* v;       /* e4m3, same layout and strides */
  void* k_scale; /* bytes, scale of (row r, head g) at g*scale_head_stride + r / scale_block */
  void* v_scale;
  int64_t kv_token_stride;   /* bytes, multiple of 16; num_cache_rows * kv_token_stride < 2^36 (64 GiB) */
  int64_t kv_head_stride;    /* bytes, multiple of 16 */
  int64_t scale_head_stride; /* >= ceil(num_cache_rows / scale_block) */
  void* idx_k;       /* e4m3 [rows][d_idx], element (r,j) at byte r*idx_token_stride + j; 16-byte aligned */
  void* idx_k_scale; /* bytes [ceil(num_cache_rows / scale_block)] */
  int64_t idx_token_stride; /* bytes, multiple of 16 */
  int32_t scale_block;      /* rows per scale: 16, 32, 64 or 128. With a block table it must divide block_size */
} clsa_cache8;

/* Bytes of workspace that the three calls below may need for these params. 256-byte aligned and all zero before its first
 * use; the calls leave their counters at zero. It may be shared by these calls for other params and caches too (give it the
 * largest size) and by clsa_topk, but not by the other calls of clsa.h (their scratch lies elsewhere in it), nor by calls
 * that overlap on the GPU. Reads the scalar fields of p and c only. *bytes is HOST memory. */
CLSA_API clsa_status clsa_cache8_workspace_bytes(const clsa_params* p, const clsa_cache8* c, size_t* bytes);

/* The newest T = q_per_seq tokens of every sequence into the caches: token t of sequence b goes to position
 * s = seq_len[b] - T + t (seq_len already counts them). Per block of scale_block rows and head:
 *   e = the smallest exponent in -100 .. 120 with max |x| <= 448 * 2^e over the block's new rows (finite elements), and not
 *       below the block's present exponent if it holds older rows of the sequence,
 *   code = x * 2^-e rounded to nearest even, saturating (an infinity becomes +-448, a NaN stays one),
 *   and the older rows of a block whose exponent grew are re-coded: code * 2^(e_old - e) rounded to nearest even.
 * Rows behind the sequence's last token are left as they were.
 *   spec      NULL, or the norm and rotation that K's rows go through first (with k_weight, at position s, in fp32: no
 *             intermediate rounding); spec->head_dim must equal p->head_dim
 *   k_new, v_new  bf16 heads of the B * T new tokens in order (b, t), num_heads == num_kv_heads (both NULL: K_idx only)
 *   idx_k_new     likewise, num_heads == 1, idx_dim elements (NULL: K and V only)
 * A block that a call appends to must belong to one sequence (full blocks may be shared). A sequence that does not begin on a
 * scale block is skipped and flagged (CLSA_DEV_BAD_SCALE_BLOCK). A sequence with seq_len < T or
 * > max_seq_len is skipped and flagged (CLSA_DEV_BAD_SEQLEN), a block outside num_cache_rows too (CLSA_DEV_BAD_INDEX). */
CLSA_API clsa_status clsa_cache8_append(const clsa_params* p, const clsa_cache8* c, const clsa_norm_rope_spec* spec,
                                        const clsa_heads* k_new, const clsa_heads* v_new, const clsa_heads* idx_k_new,
                                        void* workspace, size_t workspace_bytes, clsa_stream stream);

/* scores[b][t][s] = sum_j q_idx[b][t][j] * K_idx[s][j] for every visible s: clsa_index_scores over an 8-bit cache (its
 * arguments, its results for the values that the codes stand for). Codes are exact in the 16-bit operands of the
 * matrix instructions, so are bf16 queries down to 2^-31 of their row's largest magnitude; sums are fp32. T up to 32 streams
 * the keys once; larger T expands them to bf16 in the workspace (halved, and exact: 2^128 is no bf16) and runs the tensor-core
 * GEMM of clsa_index_scores over them, doubling its sums. A row outside num_cache_rows counts as a row of zeros and flags CLSA_DEV_BAD_INDEX. */
CLSA_API clsa_status clsa_index_scores8(const clsa_params* p, const clsa_cache8* c, const void* q_idx, float* scores,
                                        int64_t score_stride, void* workspace, size_t workspace_bytes, clsa_stream stream);

/* clsa_sparse_attn over an 8-bit cache: its arguments and results (bf16 outputs, optional fp32 log-sum-exp, zeros and -inf for
 * a query with count 0). T >= 1. p->sm_scale finite and > 0 as there. Logits may have any size that is a float, for queries of
 * magnitudes below 2^118 / sm_scale (beyond that a query counts as less than it is).
 *   hints  NULL, or as for clsa_sparse_attn_hinted with shared_gpu == 0 (CLSA_ERR_UNSUPPORTED otherwise)
 * Results do not depend on hints beyond rounding, and are the same from call to call. */
CLSA_API clsa_status clsa_sparse_attn8(const clsa_params* p, const clsa_cache8* c, const void* q, const int32_t* idx,
                                       const int32_t* count, void* out, float* lse, const clsa_attn_hints* hints,
                                       void* workspace, size_t workspace_bytes, clsa_stream stream);

#ifdef __cplusplus
}
#endif
#endif /* CLSA_CACHE8_H_ */
