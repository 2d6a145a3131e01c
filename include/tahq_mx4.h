/*
 * tahq -- microscaled 4-bit matrices ("mx4") on AMD MI355X (gfx950): quantization, and the product of two of them.
 *
 * What a pipeline stage multiplies right behind the decoder and right in front of the encoder, in 4 bits: the matrix
 * cores take 4-bit floating point values with one power-of-two scale for every 32 of them.
 *
 * Values.  A block is 32 consecutive elements of a row (the row's last block is filled up with zeros).
 *   - With transform = 1 a block x is first rotated: y = (1/sqrt(32)) H_32 x, H_32 Sylvester's Hadamard matrix: fp32
 *     butterflies h = 1, 2, 4, 8, 16 in this order, then one multiplication by fp32(1/sqrt(32)).  Products of two
 *     matrices that were both rotated are those of the unrotated ones, as far as 4 bits go.
 *   - Its scale is 2^(s-127), s one byte.  With a the block's largest magnitude and e = floor(log2 a):
 *       TAHQ_MX4_FLOOR   s - 127 = e - 2: the top of the block lies in [4, 8) grid units and saturates at 6
 *       TAHQ_MX4_COVER   the smallest s with a <= 6 * 2^(s-127): nothing saturates, the grid is coarser for a third of blocks
 *     both at least -127 (s = 0), which is also what a block of zeros gets.
 *   - Its 32 codes are the values / 2^(s-127) rounded to the nearest of +-{0, 0.5, 1, 1.5, 2, 3, 4, 6}, ties to the
 *     even code, saturating at 6: sign in bit 3, index of the magnitude in bits 0..2.
 *   - A block with an infinity or a NaN gets s = 255 and stands for 32 NaN; so does everything a product makes of it.
 *
 * Layout of a packed [rows, cols] matrix, made for the matrix instruction's operands; RB = ceil(rows/32),
 * KB = ceil(cols/64), KC = ceil(cols/256):
 *   codes    1024 bytes for every 32 rows x 64 columns, [RB][KB][half: 2][row: 32][16 bytes]: a lane's operand is 16
 *            bytes, a wavefront's 1024 in a row.  Element k of a block is in byte k/2, low half first.
 *   scales   at byte 1024*RB*KB: [RB][KC][half: 2][row: 32][4 bytes], the four bytes being the blocks 64 columns apart
 *   Rows from `rows` to 32*RB, and columns behind `cols`, are zeros with s = 0.
 *
 * Conventions as in tahq.h: d_* are device pointers, 16-byte aligned, no overlap between inputs and outputs; the caller owns every buffer;
 * nothing is allocated, kept or synchronized; argument errors come back before anything is enqueued.  TAHQ_ERR_UNSUPPORTED: matrices
 * of 2^24 tiles of 32 x 256 and more (2^29 rows of up to 256 columns), products of up to 16 rows with n from about 2^27 on, and of 2^24
 * tiles of C of at most 256 x 256 and more: a launch has fewer than 2^32 lanes.
 */
#ifndef TAHQ_MX4_H
#define TAHQ_MX4_H

#include "tahq.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { TAHQ_MX4_FLOOR = 0, TAHQ_MX4_COVER = 1 };

typedef struct {
    uint32_t struct_size;   /* = sizeof(tahq_mx4_config); set by tahq_mx4_config_default       */
    uint32_t rows;          /* rows of the tensor in fp32/bf16, row-major; 1 .. 2^31-1         */
    uint32_t cols;          /* columns, 1 .. 2^31-1                                            */
    uint32_t ld;            /* elements from one row to the next, >= cols; 0 = cols            */
    uint32_t dtype;         /* tahq_dtype                                                      */
    uint32_t transform;     /* 0 = none, 1 = rotate every block by H_32 / sqrt(32)             */
    uint32_t scale_rule;    /* TAHQ_MX4_FLOOR or TAHQ_MX4_COVER                                */
} tahq_mx4_config;

/* Fills *cfg with dtype bf16, no transform, TAHQ_MX4_FLOOR, dimensions 0.  NULL is ignored. */
void tahq_mx4_config_default(tahq_mx4_config *cfg);

/* Bytes of a packed [rows, cols] matrix; 0 if a dimension is 0 or 2^31 or more. */
size_t tahq_mx4_packed_size(uint32_t rows, uint32_t cols);

/* Quantize the [rows, cols] tensor at d_in, read once.
 *   d_packed      written: the packed [rows, cols] matrix, blocks along rows; NULL = not wanted
 *   d_packed_t    written: the packed [cols, rows] matrix, i.e. of the transposed tensor, blocks along columns (what a
 *                 product that sums over rows takes: the weight's gradient); NULL = not wanted, one of the two is
 * Every byte of a wanted matrix is written. */
tahq_status tahq_mx4_quantize(const tahq_mx4_config *cfg, const void *d_in,
                              void *d_packed, size_t packed_capacity,
                              void *d_packed_t, size_t packed_t_capacity, tahq_stream stream);

/* The values of a packed [rows, cols] matrix as a tensor of cfg->dtype with row stride cfg->ld (rounded to nearest even;
 * with transform = 1 the rotation is undone, by the same butterflies; of a block with magnitudes near the type's largest, grid
 * points beyond it become infinite). */
tahq_status tahq_mx4_dequantize(const tahq_mx4_config *cfg, const void *d_packed, size_t packed_bytes,
                                void *d_out, tahq_stream stream);

typedef struct {
    uint32_t struct_size;   /* = sizeof(tahq_mx4_matmul_config)                                */
    uint32_t m, n, k;       /* C[m, n] = sum over k of A[m, k] * B[n, k]                       */
    uint32_t ldc;           /* elements from one row of C to the next, >= n; 0 = n             */
    uint32_t out_dtype;     /* tahq_dtype of C                                                 */
    uint32_t accumulate;    /* 0: C is overwritten, 1: added to (in fp32, rounded once)        */
} tahq_mx4_matmul_config;

void tahq_mx4_matmul_config_default(tahq_mx4_matmul_config *cfg);   /* bf16, no accumulation, dimensions 0 */

/* Bytes of scratch that tahq_mx4_matmul needs for this shape: partial sums of products with few tiles and a long k.
 * May be 0.  Also 0 for an invalid cfg. */
size_t tahq_mx4_matmul_workspace_size(const tahq_mx4_matmul_config *cfg);

/* C = A B^T of a packed [m, k] matrix A and a packed [n, k] matrix B, summed in fp32.  A layer's forward pass (x, W), the
 * gradient of its input (dy, W^T along W's columns) and of its weight (dy and x, both along tokens) are all this. */
tahq_status tahq_mx4_matmul(const tahq_mx4_matmul_config *cfg, const void *d_a, size_t a_bytes,
                            const void *d_b, size_t b_bytes, void *d_c,
                            void *d_workspace, size_t workspace_capacity, tahq_stream stream);

/* y = quantized(x) B^T: tahq_mx4_quantize of x and tahq_mx4_matmul in one call, with the same result; a few tokens are
 * quantized inside the product's launch.  x->rows == cfg->m and x->cols == cfg->k.  Scratch:
 * tahq_mx4_linear_workspace_size(x, cfg) bytes. */
size_t tahq_mx4_linear_workspace_size(const tahq_mx4_config *x, const tahq_mx4_matmul_config *cfg);
tahq_status tahq_mx4_linear(const tahq_mx4_config *x, const tahq_mx4_matmul_config *cfg, const void *d_x,
                            const void *d_b, size_t b_bytes, void *d_y,
                            void *d_workspace, size_t workspace_capacity, tahq_stream stream);

#ifdef __cplusplus
}
#endif
#endif /* TAHQ_MX4_H */
