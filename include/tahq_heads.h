/*
 * tahq -- queries and keys behind their projection on AMD MI355X (gfx950): every head normed and rotated by its token's position,
 * forward and backward.
 *
 * For every token and every head x of `head` channels, with RMS(x) = sqrt(mean(x^2) + eps):
 *   norm       n = (x / RMS(x)) . w        w: [head], one for all query heads, one for all key heads; without norms n = x
 *   rotation   channels come in `rotated` / 2 pairs: (i, i + rotated/2) with TAHQ_HEADS_HALVES, (2i, 2i + 1) with TAHQ_HEADS_PAIRS
 *              y_a = magnitude (n_a cos t - n_b sin t),  y_b = magnitude (n_a sin t + n_b cos t),  t = position * frequency_i
 *              channels from `rotated` on: y = n
 * All of it in fp32 from one read, rounded once.  Angles are exact for every position: a frequency is a fraction of a turn in 64
 * bits, and position * frequency modulo one turn is an integer product, off by at most |position| 2^-65 turns; from there the angle is
 * rounded to 2^-32 turns.
 *
 * Layout: heads of a token lie side by side, tokens ldq (ldk) elements apart, so that queries and keys may be views of one packed
 * projection.  Conventions as in tahq.h, but queries, keys, their gradients and positions need no more alignment than their elements' (16 bytes, with
 * strides and heads of whole 16 bytes, are fastest).  An output may be the input that it is made of, if the strides are the same.
 */
#ifndef TAHQ_HEADS_H
#define TAHQ_HEADS_H

#include "tahq.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { TAHQ_HEADS_HALVES = 0, TAHQ_HEADS_PAIRS = 1 };
enum { TAHQ_ROTARY_PLAIN = 0, TAHQ_ROTARY_LINEAR = 1, TAHQ_ROTARY_STRETCHED = 2, TAHQ_ROTARY_PARTS = 3 };

#define TAHQ_HEADS_MAX 512u      /* channels of a head; more give TAHQ_ERR_UNSUPPORTED */

typedef struct {
    uint32_t struct_size;      /* = sizeof(tahq_heads_config)                                                */
    uint32_t tokens;           /* 1 .. 2^31-1                                                                */
    uint32_t q_heads, k_heads; /* 1 and more, 0 and more; together below 2^16                                */
    uint32_t head;             /* channels of a head, 1 .. TAHQ_HEADS_MAX                                    */
    uint32_t rotated;          /* even, 0 .. head                                                            */
    uint32_t layout;           /* TAHQ_HEADS_HALVES or TAHQ_HEADS_PAIRS                                      */
    uint32_t dtype;            /* tahq_dtype of queries, keys, weights and gradients but those of the weights */
    uint32_t norm;             /* 1: heads are normed                                                        */
    uint32_t accumulate;       /* backward: 1 = gradients of the weights are added to what is there          */
    uint32_t ldq, ldk;         /* elements from token to token of q and k and of their gradients; 0 = heads * head    */
    uint32_t ldq_out, ldk_out; /* of the outputs and of the gradients that come back to them                 */
    float eps;                 /* > 0                                                                        */
    float magnitude;           /* finite                                                                     */
} tahq_heads_config;

void tahq_heads_config_default(tahq_heads_config *cfg);   /* bf16, halves, norm, eps 1e-6, magnitude 1, dimensions 0 */

/* Frequencies of the pairs i = 0 .. rotated/2 - 1, f_i = base^(-2 i / rotated) radians per position, for contexts that are `factor` times as
 * long as what a model was trained with:
 *   TAHQ_ROTARY_PLAIN      f_i
 *   TAHQ_ROTARY_LINEAR     f_i / factor
 *   TAHQ_ROTARY_STRETCHED  base is base * factor^(rotated / (rotated - 2)): the slowest pair's is f_i / factor, the fastest's f_i
 *   TAHQ_ROTARY_PARTS      with r = original * f_i / 2 pi, the turns of the pair in the original context, and k = (r - low) / (high - low) cut to
 *                          0 .. 1: k f_i + (1 - k) f_i / factor
 * Published methods: the rotation with plain frequencies, Su, Lu, Pan, Murtadha, Wen, Liu 2021; linear, position interpolation, Chen, Wong, Chen, Tian
 * 2023; stretched, "NTK-aware" scaling, and by parts, "NTK-by-parts", Peng, Quesnelle, Fan, Shippole 2023. */
typedef struct {
    uint32_t struct_size;      /* = sizeof(tahq_rotary_config)                                   */
    uint32_t rotated;          /* even, 2 .. TAHQ_HEADS_MAX                                      */
    uint32_t scaling;          /* TAHQ_ROTARY_*                                                  */
    uint32_t original;         /* PARTS: tokens of the original context, 1 and more              */
    double base;               /* > 0                                                            */
    double factor;             /* > 0                                                            */
    double low, high;          /* PARTS: finite, low < high                                      */
} tahq_rotary_config;

void tahq_rotary_config_default(tahq_rotary_config *cfg);  /* plain, base 10000, factor 1, original 4096, low 1, high 32, rotated 0 */

/* Host code: frequencies[i] = turns per position in units of 2^-64, modulo one turn, rotated/2 of them.  They go into device memory once. */
tahq_status tahq_rotary_frequencies(const tahq_rotary_config *cfg, uint64_t *frequencies);

/* Forward.
 *   d_q, d_k              read     [tokens, heads, head]; d_k NULL exactly if k_heads is 0
 *   d_w_q, d_w_k          read     [head], exactly with norms; d_w_k NULL if k_heads is 0
 *   d_positions           read     int64 [tokens], any sign; NULL exactly if rotated is 0
 *   d_frequencies         read     uint64 [rotated/2]; NULL exactly if rotated is 0
 *   d_q_out, d_k_out      written  [tokens, heads, head] */
tahq_status tahq_heads_forward(const tahq_heads_config *cfg, const void *d_q, const void *d_k, const void *d_w_q, const void *d_w_k,
                               const int64_t *d_positions, const uint64_t *d_frequencies, void *d_q_out, void *d_k_out,
                               tahq_stream stream);

/* Bytes of scratch of the backward pass: sums of the weights' gradients over every workgroup's tokens.  0 for an invalid cfg; may be 0
 * without norms. */
size_t tahq_heads_workspace_size(const tahq_heads_config *cfg);

/* Backward: gradients of q and k from those of the outputs.
 *   d_grad_q_out, d_grad_k_out  read     strides ldq_out, ldk_out
 *   d_q, d_k                    read     as in the forward pass, exactly with norms
 *   d_grad_q, d_grad_k          written  strides ldq, ldk
 *   d_grad_w_q, d_grad_w_k      written  float [head], exactly with norms
 * Sums over tokens and heads are taken in a fixed order. */
tahq_status tahq_heads_backward(const tahq_heads_config *cfg, const void *d_grad_q_out, const void *d_grad_k_out,
                                const void *d_q, const void *d_k, const void *d_w_q, const void *d_w_k,
                                const int64_t *d_positions, const uint64_t *d_frequencies, void *d_grad_q, void *d_grad_k,
                                float *d_grad_w_q, float *d_grad_w_k, void *d_workspace, size_t workspace_capacity,
                                tahq_stream stream);

#ifdef __cplusplus
}
#endif
#endif /* TAHQ_HEADS_H */
