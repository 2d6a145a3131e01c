/*
 * tahq -- the loss at the end of the last pipeline stage on AMD MI355X (gfx950): softmax cross entropy of hidden states against the
 * weight of a large vocabulary, and its gradients.  Logits are never stored as a whole, neither forward nor backward.
 *
 * For a token with hidden state x and target t, over all rows w_v of the vocabulary's weight:
 *   l_v = x . w_v           lse = log sum_v exp(l_v)          loss = lse - l_t
 *   gradients, with p_v = exp(l_v - lse) and g the gradient of the token's loss:
 *   grad x = g sum_v (p_v - [v = t]) w_v                      grad w_v = sum over tokens g (p_v - [v = t]) x
 * A token whose target is cfg->ignore does not count: its loss and lse are 0, it adds nothing to any gradient and its own is 0, whatever its
 * hidden state holds, NaN included.  A target outside 0 .. vocab - 1 that is not `ignore` makes the token's loss NaN, and its gradients.
 *
 * Products of bf16 are exact and summed in fp32; softmax statistics and losses are fp32.  Products of fp32 are fp32's or, for many tokens
 * and rows of the vocabulary, those of sums of three bf16: off by 2^-24 of their size, or, below magnitudes of 2^-100, by 2^-126 of the other
 * number's; logits of infinite numbers are what fp32's products make of them either way.  (A gradient that an infinite hidden state or weight
 * is a factor in, mostly 0 times it, may be NaN where fp32's is infinite.)  Logits of -infinity and masks of any lowest number have p = 0; one
 * of +infinity, or NaN, makes NaN of the token's loss and lse.  In the backward pass logits are computed again, a piece of the vocabulary at a
 * time, and p_v - [v = t] (times g with LOSS_NONE, otherwise g comes last) is rounded to cfg->dtype for the matrix cores, as a hidden state or
 * weight would be.
 *
 * Tensors are contiguous and row-major: hidden states [rows, cols], weight [vocab, cols].  Conventions as in tahq.h; targets and
 * grad_loss need no more alignment than their elements'.
 */
#ifndef TAHQ_LOSS_H
#define TAHQ_LOSS_H

#include "tahq.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { TAHQ_LOSS_NONE = 0, TAHQ_LOSS_SUM = 1, TAHQ_LOSS_MEAN = 2 };

typedef struct {
    uint32_t struct_size;     /* = sizeof(tahq_loss_config)                                              */
    uint32_t rows;            /* tokens, 1 .. 2^31-1                                                     */
    uint32_t cols;            /* channels, 1 .. TAHQ_LOSS_MAX_COLS                                       */
    uint32_t vocab;           /* rows of the weight, 1 .. 2^31-1                                         */
    uint32_t dtype;           /* tahq_dtype of hidden states, weight and the hidden states' gradient     */
    uint32_t weight_dtype;    /* tahq_dtype of the weight's gradient                                     */
    uint32_t reduction;       /* TAHQ_LOSS_NONE, _SUM, _MEAN (over the tokens that count; 0 if none does) */
    uint32_t accumulate;      /* 1: the weight's gradient is added to what is there, in fp32             */
    int64_t ignore;           /* target of tokens that do not count                                      */
} tahq_loss_config;

#define TAHQ_LOSS_MAX_COLS 65536u       /* more give TAHQ_ERR_UNSUPPORTED */
#define TAHQ_LOSS_MAX_ROWS 8388608u     /* more tokens, and launches of 2^32 lanes and more, too */

void tahq_loss_config_default(tahq_loss_config *cfg);   /* bf16 both, mean, no accumulation, ignore -100, dimensions 0 */

/* Bytes of scratch of the two calls: the hidden states of the tokens that count; per-token statistics of pieces of the vocabulary; backward also a
 * piece of the softmax's gradient and fp32 sums of the hidden states' gradient.  0 for an invalid cfg. */
size_t tahq_loss_forward_workspace_size(const tahq_loss_config *cfg);
size_t tahq_loss_backward_workspace_size(const tahq_loss_config *cfg);

/* Forward.
 *   d_x, d_weight     read
 *   d_target          read     int64 [rows]
 *   d_losses, d_lse   written  float [rows]
 *   d_total           written  float [2]: the reduced loss (the sum with TAHQ_LOSS_NONE), and the number of tokens that count */
tahq_status tahq_loss_forward(const tahq_loss_config *cfg, const void *d_x, const void *d_weight, const int64_t *d_target,
                              float *d_losses, float *d_lse, float *d_total, void *d_workspace, size_t workspace_capacity,
                              tahq_stream stream);

/* Backward.
 *   d_x, d_weight, d_target   as in the forward pass
 *   d_lse                     read     as the forward pass wrote it
 *   d_grad_loss               read     float, gradient of the reduced loss; [rows] with TAHQ_LOSS_NONE; NULL: ones
 *   d_grad_x                  written  [rows, cols]; NULL: not wanted
 *   d_grad_weight             written  [vocab, cols] of cfg->weight_dtype; NULL: not wanted, one of the two is
 * Sums are taken in a fixed order. */
tahq_status tahq_loss_backward(const tahq_loss_config *cfg, const void *d_x, const void *d_weight, const int64_t *d_target,
                               const float *d_lse, const float *d_grad_loss, void *d_grad_x, void *d_grad_weight,
                               void *d_workspace, size_t workspace_capacity, tahq_stream stream);

#ifdef __cplusplus
}
#endif
#endif /* TAHQ_LOSS_H */
