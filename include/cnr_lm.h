/*
 * cnr_lm.h -- operators for language models next to the checkpoint path of cnr.h: a token embedding is a
 * table like those, and so is the matrix whose product with the hidden states gives the logits (often the same
 * one); the program that tracks and checkpoints them multiplies with them, in training and in serving.
 *
 *   cnr_quantize_blocks   a matrix to 8-bit floating point with a scale for each block of 128, and its
 *                         transpose for the backward pass
 *   cnr_block_product     the product of two such matrices: a layer's output, its gradients, the logits
 *   cnr_count_tokens      tokens of prompts and of decoding steps entered into each sequence's set and counts
 *   cnr_adjust_logits     penalties for repeated tokens, biases and a grammar's masks on logits
 *
 * The general rules of cnr.h hold: device pointers owned by the caller unless a comment says "host", work
 * is only enqueued on `stream`, nothing is allocated, conditions found on the device never fault and are
 * reported by cnr_poll_errors.  Infinities and NaN are ordinary inputs here.  A size of zero is an empty
 * matrix or list: the call writes what is left to write and succeeds.
 *
 * Blocked matrices: a matrix X of n_rows x dim is held as
 *   codes   uint8 [n_rows][cnr_block_row_bytes(dim)]: e4m3 values (sign, 4 bits of exponent with bias 7, 3
 *           of mantissa; 0x7f and 0xff are NaN, no infinities, largest 448); bytes at columns >= dim are 0;
 *           16-byte aligned base
 *   scale   [ceil(dim / 128)][cnr_block_scale_stride(n_rows, kind)]: entry [j][i] belongs to columns
 *           [128 j, 128 (j + 1)) of row i (CNR_BLOCK_ROW) or of rows [128 i, 128 (i + 1)) (CNR_BLOCK_TILE);
 *           entries that belong to no row are not read for a result and may hold anything;
 *           uint8 b from 1 to 254 standing for 2^(b - 127) (CNR_SCALE_E8M0) or float (CNR_SCALE_F32; finite, one
 *           below 2^-126 counts as 0); 16-byte aligned base
 * and stands for scale * code.
 */
#ifndef CNR_LM_H
#define CNR_LM_H

#include "cnr.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { CNR_FLOAT_F32 = 0, CNR_FLOAT_BF16 = 1, CNR_FLOAT_F16 = 2 } cnr_float_type;
typedef enum { CNR_SCALE_E8M0 = 0, CNR_SCALE_F32 = 1 } cnr_scale_type;
typedef enum {
    CNR_BLOCK_ROW = 0, /* 1 x 128: activations and gradients */
    CNR_BLOCK_TILE = 1 /* 128 x 128: weights */
} cnr_block_kind;

#define CNR_BLOCK 128u
#define CNR_LM_MAX_SIZE 2147483647u /* rows, columns, tokens of a vocabulary, slots, masks: CNR_E_TOO_LARGE beyond */

/* Sizes (pure host arithmetic). */
size_t cnr_block_row_bytes(uint64_t dim);                            /* dim rounded up to a multiple of 128 */
size_t cnr_block_scale_stride(uint64_t n_rows, cnr_block_kind kind); /* n_rows rounded up to a multiple of 128,
                                                                        divided by 128 for CNR_BLOCK_TILE */
size_t cnr_block_scale_count(uint64_t n_rows, uint64_t dim, cnr_block_kind kind);

/* Quantizes X = x[0 .. n_rows)[0 .. dim).  With amax the largest |x| of a block's finite values,
 *   CNR_SCALE_E8M0   scale = 2^e, e the least integer >= -126 with amax <= 448 * 2^e
 *   CNR_SCALE_F32    scale = max(amax / 448 rounded to float, 2^-126)
 * and 1 where amax is 0; each code is the e4m3 value nearest to the quotient x / scale, of two equally near
 * ones the one with an even mantissa; infinities and NaN become NaN.
 *   x          float, bfloat16 or IEEE half as `type` says, aligned to its element
 *   stride     elements from one row to the next, >= dim
 *   codes, scale      X as a blocked matrix, both or neither NULL
 *   codes_t, scale_t  the transpose of X, dim x n_rows, as a blocked matrix of the same kind, both or neither
 *              NULL: for CNR_BLOCK_TILE the same codes and scales transposed; for CNR_BLOCK_ROW its blocks are
 *              128 rows of one column of X
 * x is read once, whichever are asked for.  CNR_E_TOO_LARGE from 2^24 tiles of 128 x 128 on. */
cnr_status cnr_quantize_blocks(cnr_ctx *ctx, const void *x, cnr_float_type type, uint64_t n_rows, uint64_t dim,
                               uint64_t stride, cnr_block_kind kind, cnr_scale_type scale_type, uint8_t *codes,
                               void *scale, uint8_t *codes_t, void *scale_t, void *stream);

/* out[i][j] = sum over t < k of A[i][t] * B[j][t], added to out[i][j] where accumulate is not 0; A is a
 * blocked matrix of m x k, B of n x k, both with scales of scale_type.  Results are rounded once, to out's type.
 * For float outputs the products are added up in fp32.  For the 16-bit types the 8-bit matrix instructions add them up,
 * which of each eight products drop what lies 2^-14 or more below the largest: beyond its rounding a result is off by up to 2^-10 of
 * the sum of its products' magnitudes (measured: 1e-5 for normal codes, 1.4e-4 for codes of evenly spread exponents, 4.3e-4 where one of each eight is
 * 2^14 times the others).  That is below half a step of the type unless products cancel; then a result can lose all its digits: take
 * a float output where that matters.  For float outputs scale * code passes through bfloat16, which holds it
 * exactly from 2^-126 on (smaller values lose bits below 2^-133).  A result is infinite or NaN only where codes are NaN or fp32 cannot
 * hold a block's sum or the total; tiles of a float output in which one is, or in which scale * code reaches 2^128, take several
 * times as long.  The result does not depend on other work on the GPU.
 * CNR_E_TOO_LARGE from 2^24 tiles of 128 x 128 outputs on, and from m > 2^19 with k >= 2^24 - 128 on.
 *   out_stride  elements from one row of out to the next, >= n; out is aligned to its element
 *   workspace   NULL, or cnr_block_product_workspace_bytes(ctx, m, n, k) bytes, 16-byte aligned, contents
 *               irrelevant: with it, products with few outputs and a large k are split over the whole GPU
 * Backward of Y = X W^T with X of tokens x k, W of n x k in tiles:  dX = dY W is the product of dY and W's
 * transpose (codes_t of W), dW = dY^T X that of the transposes of dY and X. */
size_t cnr_block_product_workspace_bytes(const cnr_ctx *ctx, uint64_t m, uint64_t n, uint64_t k);
cnr_status cnr_block_product(cnr_ctx *ctx, const uint8_t *a_codes, const void *a_scale, cnr_block_kind a_kind,
                             uint64_t m, const uint8_t *b_codes, const void *b_scale, cnr_block_kind b_kind,
                             uint64_t n, uint64_t k, cnr_scale_type scale_type, void *out, cnr_float_type out_type,
                             uint64_t out_stride, int accumulate, void *workspace, void *stream);

/* Tokens of n sequences entered into the state of their slots.  For every token t of sequence i with
 * 0 <= t < vocab: bit t of seen[slot] is set and, for tokens that the model wrote (prompt 0, counts not NULL),
 * counts[slot][t] goes up by one, where slot = slots[i] (i when slots is NULL).  Other tokens (padding) are skipped and counted as
 * cnr_mark_touched counts look-ups outside the table; sequences whose slot is not below n_slots are skipped
 * and raise CNR_FLAG_ROW_ID if they have tokens.
 *   seen      uint32 [n_slots][cnr_bitmap_words(vocab)], laid out as a tracking bitmap; 4-byte aligned
 *   counts    uint32 [n_slots][vocab], or NULL: no counts are kept
 *   tokens    int32 or int64 [n_tokens] as `type` says
 *   offsets   uint64 [n + 1], ascending: sequence i has tokens [offsets[i], offsets[i + 1]), as far as they
 *             lie below n_tokens; NULL: n_tokens == n, one token each (a decoding step)
 *   slots     int32 [n] or NULL; sequences may share a slot, which then has the tokens of all
 *   prompt    not 0: the tokens are seen but not counted
 *   restart   not 0: the slots of the call, their counts too, are emptied first */
cnr_status cnr_count_tokens(cnr_ctx *ctx, uint32_t *seen, uint32_t *counts, uint64_t n_slots, uint64_t vocab,
                            const void *tokens, uint64_t n_tokens, cnr_index_type type, const uint64_t *offsets,
                            const int32_t *slots, uint64_t n, int prompt, int restart, void *stream);

/* What cnr_adjust_logits applies to row i (sequence i); a host struct, read during the call.
 *   seen, counts, n_slots  the state kept by cnr_count_tokens, or seen NULL: no penalties; counts NULL: only
 *                 the repetition penalty.  Counts are looked up for seen tokens only
 *   slots         int32 [n]: row i's slot, or NULL: slot i; a row whose slot is not below n_slots gets no
 *                 penalties and raises CNR_FLAG_ROW_ID, a negative one no penalties
 *   repetition, frequency, presence   float [n], or NULL: 1, 0, 0
 *   bias_offsets  uint64 [n + 1], or NULL: no biases; row i's biases are entries [bias_offsets[i],
 *                 bias_offsets[i + 1]) of bias_tokens and bias_values, as far as they lie below n_bias
 *   bias_tokens   int32 [n_bias], strictly ascending within a row; entries outside the vocabulary are skipped
 *   bias_values   float [n_bias]
 *   masks         uint32 [n_masks][cnr_bitmap_words(vocab)], or NULL: everything is allowed; set bits
 *                 are the tokens that the grammar allows; bits at positions >= vocab are ignored
 *   mask_of       int32 [n]: row i's mask, or NULL: mask i; negative: everything is allowed; one that is
 *                 not below n_masks allows everything and raises CNR_FLAG_ROW_ID */
typedef struct {
    const uint32_t *seen, *counts;
    uint64_t n_slots;
    const int32_t *slots;
    const float *repetition, *frequency, *presence;
    const uint64_t *bias_offsets;
    const int32_t *bias_tokens;
    const float *bias_values;
    uint64_t n_bias;
    const uint32_t *masks;
    uint64_t n_masks;
    const int32_t *mask_of;
} cnr_adjustments;

/* out[i][t] = -infinity where row i's mask does not allow t, whatever the logit is (a row whose mask allows
 * nothing is -infinity throughout), else, in fp32 with one rounding each and one to out's type,
 *   v = logits[i][t]
 *   v = v > 0 ? v / repetition : v * repetition    where t was seen
 *   v = v - frequency * count                      where t was seen
 *   v = v - presence                               where t was seen and count > 0
 *   v = v + bias
 * logits and out are float, bfloat16 or half [n][vocab] as `type` says, with rows stride and out_stride >= vocab
 * elements apart, aligned to their element; out may be logits itself, with the same stride. */
cnr_status cnr_adjust_logits(cnr_ctx *ctx, const void *logits, uint64_t stride, void *out, uint64_t out_stride,
                             cnr_float_type type, uint64_t n, uint64_t vocab, const cnr_adjustments *adjustments /* host */,
                             void *stream);

#ifdef __cplusplus
}
#endif
#endif
