/*
 * tahq -- the norms before and after a block, fused with its gate and residual scale, on AMD MI355X (gfx950).
 *
 * What lies between two blocks of a transformer whose residual stream crosses a pipeline-stage boundary.  For every token
 * (row of `cols` channels), with RMS(v) = sqrt(mean(v^2) + eps):
 *
 *   post half   r' = residual_scale * r + g . (b / RMS(b)) . w_post      b: the block's output, r: the residual stream
 *   pre half    h  = (r' / RMS(r')) . w_pre                              h: the next block's input
 *
 * All of it in fp32 from one read of r and b; r' is rounded when it is stored, h is computed from the unrounded r'.  A row whose
 * mean square is beyond fp32 (values from about 1e19 on) has 1/RMS 0.  A
 * boundary may lie between the halves: without b the post half is r' = residual_scale * r, without w_pre there is no h.
 * h is stored in the tensors' dtype, as a packed mx4 matrix (tahq_mx4.h, blocks along channels, quantized from fp32), or both.
 *
 * Tensors are contiguous row-major [rows, cols] of cfg->dtype, weights and gate of cfg->dtype too; statistics and
 * gradients of weights and gate are fp32.  Conventions as in tahq.h.
 */
#ifndef TAHQ_NORM_H
#define TAHQ_NORM_H

#include "tahq_mx4.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct {
    uint32_t struct_size;     /* = sizeof(tahq_norm_config)                                            */
    uint32_t rows, cols;      /* tokens, 1 .. 2^31-1, and channels, 1 .. TAHQ_NORM_MAX_COLS            */
    uint32_t dtype;           /* tahq_dtype                                                            */
    uint32_t gate_rows;       /* tokens that share a row of the gate [ceil(rows/gate_rows), cols]: rows (or more) = one
                                 gate for all, a sample's tokens = one per sample, 1 = one per token; 0 = no gate  */
    float eps;                /* > 0                                                                   */
    float residual_scale;     /* finite                                                                */
    uint32_t accumulate;      /* backward: 1 = gradients of weights and gate are added to what is there */
    uint32_t transform;       /* of the mx4 form of h, see tahq_mx4_config                             */
    uint32_t scale_rule;
} tahq_norm_config;

#define TAHQ_NORM_MAX_COLS 8192u   /* more give TAHQ_ERR_UNSUPPORTED */

void tahq_norm_config_default(tahq_norm_config *cfg);   /* bf16, no gate, eps 1e-6, residual_scale 1, dimensions 0 */

/* Forward.
 *   d_residual      read     r
 *   d_block         read     b; NULL: no block (then d_w_post and d_gate are NULL, too)
 *   d_w_post        read     [cols]
 *   d_gate          read     [ceil(rows/gate_rows), cols]; NULL exactly if gate_rows is 0 or there is no block
 *   d_w_pre         read     [cols]; NULL: no pre half (then d_h and d_h_mx4 are NULL, too)
 *   d_residual_out  written  r'; may be NULL if there is no block; may be d_residual
 *   d_h, d_h_mx4    written  h in cfg->dtype, and packed ([rows, cols], every byte written); one of them with a pre half
 *   d_stats         written  float [2, rows]: 1/RMS(b), 1/RMS(r') (zeros for a missing half); NULL: not wanted */
tahq_status tahq_norm_forward(const tahq_norm_config *cfg, const void *d_residual, const void *d_block,
                              const void *d_w_post, const void *d_gate, const void *d_w_pre,
                              void *d_residual_out, void *d_h, void *d_h_mx4, size_t h_mx4_capacity,
                              float *d_stats, tahq_stream stream);

/* Bytes of scratch of the backward pass: column sums of every workgroup's tokens.  0 for an invalid cfg. */
size_t tahq_norm_workspace_size(const tahq_norm_config *cfg);

/* Backward: gradients from those of r' and h.
 *   d_grad_residual_out  read     NULL: zeros (needs a pre half)
 *   d_grad_h             read     with a pre half, and d_w_pre and d_residual_out (r' as stored) with it; NULL without
 *   d_block, d_w_post, d_gate     as in the forward pass
 *   d_stats              read     as the forward pass wrote them
 *   d_grad_residual      written  gradient of r
 *   d_grad_block         written  gradient of b
 *   d_grad_w_post, d_grad_w_pre   written, float [cols]
 *   d_grad_gate          written, float [ceil(rows/gate_rows), cols]
 * Outputs of halves that are there are required, the others NULL.  Sums over tokens are taken in a fixed order. */
tahq_status tahq_norm_backward(const tahq_norm_config *cfg, const void *d_grad_residual_out, const void *d_grad_h,
                               const void *d_block, const void *d_w_post, const void *d_gate,
                               const void *d_residual_out, const void *d_w_pre, const float *d_stats,
                               void *d_grad_residual, void *d_grad_block,
                               float *d_grad_w_post, float *d_grad_gate, float *d_grad_w_pre,
                               void *d_workspace, size_t workspace_capacity, tahq_stream stream);

#ifdef __cplusplus
}
#endif
#endif /* TAHQ_NORM_H */
