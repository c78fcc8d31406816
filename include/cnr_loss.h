/*
 * cnr_loss.h -- losses over the vocabulary, next to the operators of cnr_lm.h: what trains the table that gives the logits, and
 * what a teacher or a server tells of them.
 *
 *   cnr_vocabulary_loss   softmax cross entropy, or distillation from a teacher's top logits, over a vocabulary whose
 *                         logits are never all in memory; cnr_vocabulary_loss_backward: its gradients
 *   cnr_top_logits        the largest logits of each row, and the logarithm of the sum of all exponentials
 *
 * The general rules of cnr.h and cnr_lm.h hold: device pointers owned by the caller unless a comment says "host", work is only enqueued on `stream`, nothing
 * is allocated, infinities and NaN are ordinary inputs, sizes of zero succeed.  Results, states that are written and workspaces overlap neither the operands nor each other.
 */
#ifndef CNR_LOSS_H
#define CNR_LOSS_H

#include "cnr_lm.h"

#ifdef __cplusplus
extern "C" {
#endif

/* The logits z[i][v] = sum over t < dim of hidden[i][t] * weight[v][t], of which a vocabulary's losses are made; a host struct, read during the call.
 *   hidden, weight  float, bfloat16 or half [n][dim] and [vocab][dim] as `type` says, aligned to their element, rows
 *                   hidden_stride and weight_stride >= dim elements apart.  Products and sums are fp32's.  Rows of 16 bits of a multiple of 8
 *                   elements, 16 bytes aligned, are read where they are by more than 16 rows; others are laid out in the workspace first.  Floats of
 *                   more than 64 rows are multiplied in three parts of 8 bits: six of nine products, off by 2^-21 of the product at most and 2^-24 on average, and by 2^-131
 *                   of either factor, which is more only next to a float below 2^-110 */
typedef struct {
    const void *hidden;
    uint64_t hidden_stride;
    const void *weight;
    uint64_t weight_stride;
    cnr_float_type type;
    uint64_t n, vocab, dim;
} cnr_vocabulary;

/* What the rows ought to be followed by; a host struct, read during the call.
 *   tokens       int32 or int64 [n][top] as token_type says, rows token_stride >= top apart.  Negative ones are padding; those >= vocab are skipped too and
 *                counted as cnr_mark_touched counts look-ups outside the table
 *   logits       NULL: top is 1 and each token the row's target; or a teacher's logits of the tokens, [n][top] as logit_type says, rows
 *                logit_stride >= top apart, in any order; a token may come more than once
 *   temperature  > 0, from 2^-126 to 3e38; divides the teacher's logits and the row's own.  Not read where logits is NULL */
typedef struct {
    const void *tokens;
    cnr_index_type token_type;
    uint64_t token_stride, top;
    const void *logits;
    cnr_float_type logit_type;
    uint64_t logit_stride;
    float temperature;
} cnr_targets;

#define CNR_LOSS_MAX_TOP 1024u             /* entries of a row: CNR_E_TOO_LARGE beyond, as of the others */
#define CNR_LOSS_MAX_ROWS 1048576u
#define CNR_LOSS_MAX_VOCABULARY 134217728u
#define CNR_LOSS_MAX_DIM 1048576u

/* loss[i], float [n], with lse = log sum over v of exp(z[i][v] / T):
 *   target t         lse - z[i][t], by the same sums of products, so never below 0   (T is 1)
 *   teacher          sum over j of q_j (log q_j - z[i][tokens[j]] / T + lse),  q the softmax of the teacher's logits / T over the row's tokens
 * A row without a token (a padded target, no token within the vocabulary, a teacher whose logits are all -infinity) is left out: its loss is 0, it has no
 * gradient, and its hidden state may hold anything.  A row with a NaN or an infinite z that is not -infinity has a loss of NaN.  |z / T| is to be below 2^127.
 *   state        float [cnr_loss_state_floats(n, top)], kept for the backward pass; may be NULL for targets that no backward pass follows
 *   workspace    cnr_loss_workspace_bytes(n, vocab, dim, type, 0, type) bytes at least (which serve fewer rows as well), 256-byte aligned,
 *                contents irrelevant; where vocab is 0, NULL
 * Nothing depends on other work on the GPU, sums are joined in order. */
size_t cnr_loss_state_floats(uint64_t n, uint64_t top);
size_t cnr_loss_workspace_bytes(uint64_t n, uint64_t vocab, uint64_t dim, cnr_float_type type, int training, cnr_float_type dweight_type);
cnr_status cnr_vocabulary_loss(cnr_ctx *ctx, const cnr_vocabulary *vocabulary /* host */, const cnr_targets *targets /* host */, float *loss, float *state,
                               void *workspace, size_t workspace_bytes, void *stream);

/* Gradients of sum over i of dloss[i] * loss[i], by the state of the forward pass over the same vocabulary and targets, unchanged since:
 *   dz[i][v] = dloss[i] / T * (exp(z[i][v] / T - lse) - sum of the q_j with tokens[j] = v)
 *   dhidden  NULL, or [n][dim] of `type`: dz weight
 *   dweight  NULL, or [vocab][dim] of dweight_type, `type` or float: dz^T hidden, added to what is there where accumulate is not 0
 * Logits are computed again, a piece of the vocabulary at a time.  Between the products dz is rounded to `type` once; where n is at most 64 or dweight is float it is two
 * numbers of `type` (off by 2^-17 of it for bfloat16, 2^-23 for half; dhidden of more than 64 rows takes the first); three bfloat16 for floats, and for bfloat16 up to n = 128 where
 * dweight is float.  Few rows (up to 16, up to 64 of floats) keep it in fp32, but for bfloat16 and half next to a weight of 3 * 2^24 elements or more that is read where it is.
 * Halves are scaled by the power of two that takes the largest |dloss / T| to 2^13 to 2^14, so that small gradients are not lost.  Each result is rounded once, after its sum in
 * fp32.  A row with dloss 0 adds nothing, whatever it holds; a dloss that is infinite or NaN makes gradients infinite or NaN.
 *   workspace    cnr_loss_workspace_bytes(n, vocab, dim, type, 1, dweight_type) bytes at least (dweight_type: `type` where dweight is NULL) */
cnr_status cnr_vocabulary_loss_backward(cnr_ctx *ctx, const cnr_vocabulary *vocabulary /* host */, const cnr_targets *targets /* host */, const float *state,
                                        const float *dloss, void *dhidden, uint64_t dhidden_stride, void *dweight, cnr_float_type dweight_type,
                                        uint64_t dweight_stride, int accumulate, void *workspace, size_t workspace_bytes, void *stream);

/* The `top` largest of each row of logits, largest first, of equal ones the lower token first; NaN counts as larger than infinity, -0 as 0.
 *   logits   float, bfloat16 or half [n][vocab] as `type` says, rows stride >= vocab elements apart, aligned to their element
 *   tokens   int32 [n][top], or NULL; -1 beyond the vocabulary's size
 *   values   of `type` [n][top], or NULL: the logits of these tokens, bit for bit; -infinity beyond the vocabulary's size
 *   lse      float [n], or NULL: log sum over v of exp(logits[i][v]), summed in fp32; a value minus it is the token's log probability
 * CNR_E_TOO_LARGE beyond CNR_LOSS_MAX_TOP and from n = 2^22 on. */
cnr_status cnr_top_logits(cnr_ctx *ctx, const void *logits, uint64_t stride, cnr_float_type type, uint64_t n, uint64_t vocab, uint64_t top, int32_t *tokens,
                          void *values, float *lse, void *stream);

#ifdef __cplusplus
}
#endif
#endif
