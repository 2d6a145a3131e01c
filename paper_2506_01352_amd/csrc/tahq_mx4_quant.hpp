// Quantization to mx4 along rows, along columns or both from one read, and back.
//
// Both are bound by memory: an element takes 2 or 4 bytes to read, 17/32 of a byte to write per orientation, and about ten vector
// instructions.  bf16 32768 x 8192, tensors of which no cache holds a part: both ways 162 us, back 128, i.e. 5.1 and 5.3 TB/s, as a large copy; fp32
// 16384 x 8192, rotated or not, both ways 125 to 147, back 140.  Where a compute unit has one workgroup or two, latency: 2048 x 2047 fp32 with the
// transform 6.4 and 6.8 us, of which a launch takes 2; 8.4 and 7.3 out of HBM.
#pragma once
#include "tahq_mx4_common.hpp"

namespace tahq {

constexpr uint32_t kQuantRows = 32, kQuantCols = 256, kQuantThreads = 256;

// 32 elements of a column, a block of the transposed matrix: its codes and scale byte
template <bool BF16, bool ROTATE>
__device__ __forceinline__ void quantize_column(const uint8_t *tile, uint32_t stride, uint32_t cover, uint32_t (&w)[4], uint32_t &s)
{
    if constexpr (BF16 && !ROTATE) {                       // two rows to a word; magnitudes as in quantize_quad
        typedef uint16_t pair __attribute__((ext_vector_type(2)));
        uint32_t y[16];
        pair m = {0, 0};
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const pair p = {*reinterpret_cast<const uint16_t *>(tile + 2 * i * stride), *reinterpret_cast<const uint16_t *>(tile + (2 * i + 1) * stride)};
            y[i] = __builtin_bit_cast(uint32_t, p);
            m = __builtin_elementwise_max(m, __builtin_bit_cast(pair, y[i] & 0x7fff7fffu));
        }
        s = block_scale((uint32_t)max(m.x, m.y) << 16, cover);
#pragma unroll
        for (int q = 0; q < 4; ++q) w[q] = codes8(make_uint4(y[4 * q], y[4 * q + 1], y[4 * q + 2], y[4 * q + 3]), s);
    } else {
        float y[32];
#pragma unroll
        for (int i = 0; i < 32; ++i) y[i] = load1<BF16>(tile + i * stride, 0);
        if constexpr (ROTATE) {
            butterfly(y);
#pragma unroll
            for (int i = 0; i < 32; ++i) y[i] *= kRoot32;
        }
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 32; ++i) top = max(top, __float_as_uint(y[i]) & 0x7fffffffu);
        s = block_scale(top, cover);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            float part[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) part[i] = y[8 * q + i];
            w[q] = codes8(part, s);
        }
    }
}

// A workgroup takes a tile of 32 rows x 256 columns.  Along rows: a lane loads 16 bytes of bf16 (32 of fp32), neighbours in a row next to each
// other, and four lanes share a block; the tile is a unit of rows x four of columns, 4 KB of codes, which are put in order in LDS and leave in
// whole lines.  Along columns: the tile passes through LDS once, and a lane takes a column, i.e. a whole block, whose 16 bytes of codes are
// next to its neighbours' in the transposed matrix.  Both use the same LDS, one after the other.
//   Why 32 rows: the work between load and store is a chain, which only other workgroups hide.  With 64 rows, and two columns to a lane, both
// ways of 2048 x 1600 bf16 5.7 us (rotated 8.0) against 4.6 (6.6); of 8192 x 4096 21.6 against 18.6; of 32768 x 8192, 820 MB, 146 against 146
// (rotated 199 against 182): 5.6 TB/s.
template <bool BF16, bool ROW, bool COL, bool ROTATE>
__global__ __launch_bounds__(kQuantThreads)
void k_mx4_quantize(const void *in, uint8_t *packed, uint8_t *packed_t, uint32_t rows, uint32_t cols, uint64_t ld,
                    uint32_t cover, uint32_t tiles_x)
{
    constexpr uint32_t RUN = 512 + 32;              // a half unit of codes in LDS: the skew spreads a wavefront's words over the banks
    constexpr int ES = BF16 ? 2 : 4;
    __shared__ __attribute__((aligned(16))) uint8_t lds[COL ? kQuantRows * kQuantCols * ES : 8 * RUN + 256];
    uint8_t *const scale_bytes = lds + 8 * RUN;
    const uint32_t tid = threadIdx.x;
    const uint32_t tile_y = blockIdx.x / tiles_x, r0 = tile_y * kQuantRows, c0 = blockIdx.x % tiles_x * kQuantCols;
    const uint32_t chunk = tid % 32, row = tid / 32;
    const uint32_t wide = cols - c0;                // columns from the tile's first on

    Eight<BF16> x[4] = {};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t r = r0 + row + 8 * i;
        if (r < rows && 8 * chunk < wide) x[i] = fetch<BF16, false>(static_cast<const uint8_t *>(in) + ((uint64_t)r * ld + c0) * ES, 8 * chunk, wide, more_behind(r, rows, ld));
    }
    uint32_t w[4] = {}, s[4] = {};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (COL) __builtin_memcpy(lds + ((row + 8 * i) * kQuantCols + 8 * chunk) * ES, x[i].q, sizeof x[i].q);
        if constexpr (ROW)
            if (r0 + 8 * i < rows) w[i] = quantize_quad<BF16, ROTATE>(x[i], cover, s[i]);
    }
    if constexpr (COL) {
        // block tile_y of row c of the transposed matrix
        const Mx4Layout L(cols, rows);
        const uint32_t c = c0 + tid;
        uint32_t w4[4], e;
        __syncthreads();
        quantize_column<BF16, ROTATE>(lds + tid * ES, kQuantCols * ES, cover, w4, e);
        if (c < 32 * L.rb) {                                               // rows behind `cols` hold zeros, as the tile does
            if (tile_y / 2 < L.kb) *reinterpret_cast<uint4 *>(packed_t + L.code(c, tile_y)) = make_uint4(w4[0], w4[1], w4[2], w4[3]);
            packed_t[L.scale(c, tile_y)] = (uint8_t)e;                     // also of the blocks that fill up the last four units
        }
        if constexpr (ROW) __syncthreads();
    }
    if constexpr (ROW) {
        const Mx4Layout L(rows, cols);
        const uint32_t half = chunk / 4 % 2;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t r = row + 8 * i;
            *reinterpret_cast<uint32_t *>(lds + (chunk / 8 * 2 + half) * RUN + r * 16 + chunk % 4 * 4) = w[i];
            if (chunk % 4 == 0) scale_bytes[(half * 32 + r) * 4 + chunk / 8] = (uint8_t)s[i];
        }
        __syncthreads();
        const uint32_t kb = c0 / 64 + tid / 64, at = tid * 16;
        if (tile_y < L.rb) {
            if (kb < L.kb)
                *reinterpret_cast<uint4 *>(packed + ((uint64_t)tile_y * L.kb + kb) * 1024 + at % 1024) = *reinterpret_cast<const uint4 *>(lds + at / 512 * RUN + at % 512);
            if (tid < 64)
                reinterpret_cast<uint32_t *>(packed + L.scales())[((uint64_t)tile_y * L.kc + c0 / 256) * 64 + tid] = reinterpret_cast<const uint32_t *>(scale_bytes)[tid];
        }
    }
}

// The 32 fp32 of a block that four lanes hold eight each of: lanes trade halves, so that each of the two stores writes 64 bytes in a row
__device__ __forceinline__ void keep_block(float *to, const float (&x)[8])
{
    const uint32_t lane = threadIdx.x % 4;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        float v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float a = half ? quadf<0xfa>(x[i]) : quadf<0x50>(x[i]), b = half ? quadf<0xfa>(x[4 + i]) : quadf<0x50>(x[4 + i]);
            v[i] = lane % 2 ? b : a;
        }
        __builtin_memcpy(to + 16 * half + 4 * lane, v, 16);
    }
}

// Values of a packed matrix.  A workgroup takes 32 rows x 256 columns, 4 KB of codes; four lanes share a block, as above.
template <bool BF16, bool ROTATE>
__global__ __launch_bounds__(kQuantThreads)
void k_mx4_dequantize(const uint8_t *packed, void *out, uint32_t rows, uint32_t cols, uint64_t ld, uint32_t tiles_x)
{
    const Mx4Layout L(rows, cols);
    const uint32_t tid = threadIdx.x;
    const uint32_t r0 = blockIdx.x / tiles_x * 32, c0 = blockIdx.x % tiles_x * kQuantCols;
    const uint32_t chunk = tid % 32, row = tid / 32;
    const uint32_t wide = cols - c0;
    const uint32_t b = c0 / 32 + chunk / 4;
    uint32_t w[4];
    uint8_t s[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t r = r0 + row + 8 * i;                               // below 32 * L.rb
        w[i] = b / 2 < L.kb ? *reinterpret_cast<const uint32_t *>(packed + L.code(r, b) + chunk % 4 * 4) : 0u;
        s[i] = packed[L.scale(r, b)];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t r = r0 + row + 8 * i;
        float x[8];
        values8(w[i], s[i], x);
        if constexpr (ROTATE) rotate_quad(x);
        if constexpr (!BF16) {
            if (r < rows && 8 * (chunk | 3) + 8 <= wide) {
                keep_block(static_cast<float *>(out) + (uint64_t)r * ld + c0 + 32 * (chunk / 4), x);
                continue;
            }
        }
        if (r < rows && 8 * chunk < wide) keep<BF16, false>(static_cast<uint8_t *>(out) + ((uint64_t)r * ld + c0) * (BF16 ? 2 : 4), 8 * chunk, wide, x);
    }
}

}  // namespace tahq
