/*
 * tahq -- dropout in front of a residual stream on AMD MI355X (gfx950), with a mask that is computed and never stored.
 *
 *   forward    out[e] = residual[e] + (kept(e) ? scale * x[e] : 0)          without a residual: the second term alone
 *   backward   grad_x[e] = kept(e) ? scale * grad_out[e] : 0                (the residual's gradient is grad_out itself)
 *
 * kept(e) depends on the element's number e, the seed and the offset alone, neither on the type nor on how the tensor is cut:
 *   w = Philox 4x32, ten rounds (Salmon, Moraes, Dror, Shaw 2011), of the counter (e / 8, offset), 64 bits each, low word first, under the
 *   key `seed`, low word first; r = 16 bits of it: the low half of word (e % 8) / 2 if e is even, the high half if e is odd
 *   kept(e) = r >= t,  t = floor(65536 p + 1/2): p counts in steps of 2^-16
 *   scale = 65536 / (65536 - t), rounded to fp32; with t = 65536 nothing is kept
 * Forward and backward passes of the same tensor are given the same seed and offset, different tensors different ones.  Sums are in
 * fp32, rounded once.  What is dropped counts as 0, NaN and infinities too.
 *
 * Tensors hold cfg->elements contiguous elements of cfg->dtype.  Conventions as in tahq.h; an output may be one of the call's inputs,
 * and the 64-bit number at d_offset is aligned to 8 bytes.
 */
#ifndef TAHQ_DROPOUT_H
#define TAHQ_DROPOUT_H

#include "tahq.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct {
    uint32_t struct_size;     /* = sizeof(tahq_dropout_config)                    */
    uint32_t dtype;           /* tahq_dtype                                       */
    uint64_t elements;        /* 1 .. 2^48                                        */
    uint64_t seed;
    uint64_t offset;
    float p;                  /* probability to drop, 0 .. 1                      */
} tahq_dropout_config;

void tahq_dropout_config_default(tahq_dropout_config *cfg);   /* bf16, p 0.1, the rest 0 */

/* d_offset: a 64-bit number in device memory that is added to cfg->offset when the kernel runs, for calls captured into a graph, whose
 * replays take another mask each once the program has changed the number; NULL: nothing is added. */
tahq_status tahq_dropout_forward(const tahq_dropout_config *cfg, const void *d_x, const void *d_residual, void *d_out,
                                 const uint64_t *d_offset, tahq_stream stream);
tahq_status tahq_dropout_backward(const tahq_dropout_config *cfg, const void *d_grad_out, void *d_grad_x,
                                  const uint64_t *d_offset, tahq_stream stream);

#ifdef __cplusplus
}
#endif
#endif /* TAHQ_DROPOUT_H */
