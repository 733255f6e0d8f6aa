/*
 * vsd_decode.h -- C ABI of libvsd's decoding side: drafting from an 8-bit LM
 * head under a decoding policy.
 *
 *   vsd_quantize_fp8       a matrix in e4m3 with a scale for each block of 128 columns
 *   vsd_lmhead_logits_fp8  draft logits from such matrices (beside vsd_lmhead_logits)
 *   vsd_sample_filtered    one token a row from what temperature, top-k, top-p and
 *                          min-p leave of a distribution (beside vsd_sample_paths),
 *                          and the logits with what they leave out at -inf
 *
 * The draft's distribution q may be as coarse as the drafting likes: verification
 * (Eq. 1 of arxiv 2602.05774) is lossless against the q that the tokens were drawn
 * from.  Under a policy both models' rows are filtered, and the filtered rows go to
 * vsd_verify_paths, vsd_estep_mstep and the tree calls, to which a logit of -inf is
 * a token without mass; at the policy's T their softmax is the renormalised kept
 * distribution.  (A correction may be a token that the draft's policy leaves out: its
 * logq_corr is -inf, the gradient, which has no log q in it, is finite, and the loss is
 * infinite in vsd_tree_estep_mstep, while vsd_estep_mstep counts -2^20 for it.)
 * vsd_lmhead_backward takes the logits of an 8-bit head as it takes those of the bf16
 * one (a gradient straight through the rounding of the weight).
 *
 * The conventions of vsd.h hold: device pointers owned by the caller, work enqueued
 * on `stream`, argument checks before anything is enqueued, data errors in the
 * status word of the workspace (vsd_device_status).  Calls sharing a workspace are
 * ordered on one stream.
 */
#ifndef VSD_DECODE_H_
#define VSD_DECODE_H_

#include "vsd.h"

#ifdef __cplusplus
extern "C" {
#endif

/* A row's T, top_k, top_p or min_p is out of its range (vsd_device_status). */
#define VSD_STATUS_BAD_PARAM 16

/* Quantizes x [R][H] of `dtype` to e4m3 with a scale for each block of block_rows
 * (1 or 128) rows and 128 columns; blocks at the lower and right edge are smaller.
 *   scale[i][j] = the least power of two s with amax / s <= 448, amax the block's
 *                 largest magnitude; 1 if that is 0; at least 2^-126
 *   q[r][h]     = x[r][h] / s rounded once, to nearest even (the quotient is exact)
 *   q      device, [R][H] e4m3;  scale  device, float [ceil(R / block_rows)][ceil(H / 128)]
 * A block that holds a NaN or an infinity has the scale NaN and NaN in every q.
 * H a multiple of 16, x and q 16-byte aligned; 1 <= R <= 16777216, H <= 1048576.
 * x, q and scale may not overlap. */
vsd_status vsd_quantize_fp8(const void* x, vsd_dtype dtype, int32_t R, int32_t H,
                            int32_t block_rows, void* q, float* scale, void* stream);

/* The draft LM head on 8-bit operands:
 *   logits[r][v] = sum_j hidden_scale[r][j] weight_scale[v / 128][j]
 *                        sum_{128 j <= h < 128 (j + 1)} hidden[r][h] weight[v][h]
 *   hidden  device, e4m3 [R][H];  hidden_scale  device, float [R][ceil(H / 128)]
 *   weight  device, e4m3 [V][H];  weight_scale  device, float [ceil(V / 128)][ceil(H / 128)]
 *   logits  device, bf16 [R][V], written
 *   ws      device workspace of at least 256 bytes, its first word the status word,
 *           cleared here
 * Any finite scales, not only powers of two; the product of two may be past a float's
 * range, or below it, where a block's scaled sum is not.  Products are exact; a block's
 * 128 are summed on the tensor cores, the blocks in fp32, and the sum is rounded once to
 * bf16.  H a multiple of 16, hidden and weight 16-byte aligned, logits 2-byte;
 * 1 <= R <= 16777216, 1 <= V <= 1048576, H <= 1048576.  logits may not overlap an
 * input.  A device wait that runs out sets the timeout bit of the status word. */
vsd_status vsd_lmhead_logits_fp8(const void* hidden, const float* hidden_scale,
                                 const void* weight, const float* weight_scale, int32_t R,
                                 int32_t V, int32_t H, void* logits, void* ws, size_t ws_bytes,
                                 void* stream);

/* A decoding policy.  The values hold for every row; an array [R] (device) holds for
 * its parameter instead of the value, where it is not NULL.
 *   T      0 (greedy: the most likely token alone) or 2^-64 .. 2^64
 *   top_k  <= 0: off
 *   top_p  >= 1: off; <= 0: the most likely token alone
 *   min_p  <= 0: off; >= 1: as 1
 * NaN, or a T out of its range, is refused (VSD_ERR_INVALID_ARG), in an array by
 * VSD_STATUS_BAD_PARAM for its row. */
typedef struct {
    float T;
    int32_t top_k;
    float top_p, min_p;
    const float* row_T;
    const int32_t* row_top_k;
    const float* row_top_p;
    const float* row_min_p;
} vsd_policy;

/* Outputs (device, caller-owned); a NULL member is not written. */
typedef struct {
    int32_t* tokens;   /* [R] the token drawn; needs u                                  */
    float* logq_tok;   /* [R] its log probability among the kept ones; needs u          */
    int32_t* kept;     /* [R] how many tokens are kept                                  */
    void* filtered;    /* [R][V] of the logits' dtype: the logit of a kept token, -inf
                          for the others; may be the logits themselves                  */
} vsd_filtered_outputs;

/* Bytes of device workspace (0 if a size is invalid). */
size_t vsd_sample_filtered_workspace_bytes(int32_t R, int32_t V);

/* One token a row from the filtered distribution of logits [R][V].
 * Tokens are ordered by falling logit, the lower id first among equals (-0 is 0);
 * those at -inf are never kept.  With e_i = exp((x_i - x_max) / T) in that order, kept
 * are the first n = min(k, n_p, n_m):
 *   k    top_k, or all that are not at -inf
 *   n_p  the least n with e_1 + .. + e_n >= top_p (e_1 + .. + e_k)
 *   n_m  the number with e_i >= min_p (decided on the logits, to within 2^-39 of min_p,
 *        however small)
 * Drawn is the first token v, in the vocabulary's order, with
 * sum of e over the kept tokens up to v  >  u[r] (sum of e over all kept);
 * u >= 1 draws the last kept token, u < 0 (or NaN) the first.
 * Sums are of whole numbers: each e is within 2^-41 of itself and one unit of
 * 2^-(62 - s), s = max(12, ceil(log2 V)) (2^-45 at 128256 tokens, 2^-42 at 2^20).  So no
 * result depends on an order of summation, equal calls give equal bits, and decisions by
 * sums are those of real arithmetic but within 2^-41 of the sum and V units of a border.
 * A row with NaN or +inf, or all at -inf, sets VSD_STATUS_BAD_ROW; such a row, and one
 * whose parameters are refused, has token -1, logq_tok NaN, kept 0, and is all -inf in
 * `filtered`.
 *   u   [R], or NULL: nothing is drawn (tokens and logq_tok have to be NULL then)
 *   ws  256-byte aligned; its first word is the status word, cleared here
 * 1 <= R <= 16777216, 1 <= V <= 1048576; rows at any alignment of their type.  Outputs
 * may not overlap inputs or one another, but `filtered` may be the logits. */
vsd_status vsd_sample_filtered(const void* logits, vsd_dtype dtype, int32_t R, int32_t V,
                               const vsd_policy* policy, const float* u,
                               vsd_filtered_outputs* out, void* ws, size_t ws_bytes,
                               void* stream);

#ifdef __cplusplus
}
#endif

#endif /* VSD_DECODE_H_ */
