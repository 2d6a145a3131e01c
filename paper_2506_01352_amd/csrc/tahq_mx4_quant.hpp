// Quantization to mx4 along rows, along columns or both from one read, and back.
//
// Both are bound by memory: an element takes 2 or 4 bytes to read, 17/32 of a byte to write per orientation, and about ten vector
// instructions.
#pragma once
#include "tahq_mx4_common.hpp"

namespace tahq {

constexpr uint32_t kQuantRows = 64, kQuantCols = 256, kQuantThreads = 256;

// 32 elements of two neighbouring columns: the codes and scale byte of column J.  bf16 stays packed, the columns side by side in a word.
template <bool BF16, bool ROTATE>
struct TwoColumns {
    float y[2][32];
    __device__ __forceinline__ void take(const uint8_t *tile, uint32_t stride)
    {
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            if constexpr (BF16) {
                const uint32_t w = *reinterpret_cast<const uint32_t *>(tile + i * stride);
                y[0][i] = __uint_as_float(w << 16);
                y[1][i] = __uint_as_float(w & 0xffff0000u);
            } else {
                const float2 w = *reinterpret_cast<const float2 *>(tile + i * stride);
                y[0][i] = w.x;
                y[1][i] = w.y;
            }
        }
    }
    __device__ __forceinline__ void codes(int j, uint32_t cover, uint32_t (&w)[4], uint32_t &s)
    {
        if constexpr (ROTATE) {
            butterfly(y[j]);
#pragma unroll
            for (int i = 0; i < 32; ++i) y[j][i] *= kRoot32;
        }
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 32; ++i) top = max(top, __float_as_uint(y[j][i]) & 0x7fffffffu);
        s = block_scale(top, cover);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            float part[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) part[i] = y[j][8 * q + i];
            w[q] = codes8(part, s);
        }
    }
};
template <>
struct TwoColumns<true, false> {
    uint32_t y[32];
    uint32_t top[2];
    __device__ __forceinline__ void take(const uint8_t *tile, uint32_t stride)
    {
        typedef uint16_t pair __attribute__((ext_vector_type(2)));
        pair m = {0, 0};
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            y[i] = *reinterpret_cast<const uint32_t *>(tile + i * stride);
            m = __builtin_elementwise_max(m, __builtin_bit_cast(pair, y[i] & 0x7fff7fffu));
        }
        top[0] = (uint32_t)m.x << 16;
        top[1] = (uint32_t)m.y << 16;
    }
    __device__ __forceinline__ void codes(int j, uint32_t cover, uint32_t (&w)[4], uint32_t &s)
    {
        s = block_scale(top[j], cover);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            uint4 p;                                       // rows 8 q .. 8 q + 7 of column j, two to a word
            auto two = [&](int i) { return __builtin_amdgcn_perm(y[i + 1], y[i], j ? 0x07060302u : 0x05040100u); };
            p.x = two(8 * q);
            p.y = two(8 * q + 2);
            p.z = two(8 * q + 4);
            p.w = two(8 * q + 6);
            w[q] = codes8(p, s);
        }
    }
};

// A workgroup takes a tile of 64 rows x 256 columns.  Along rows: a lane loads 16 bytes of bf16 (32 of fp32), neighbours in a row
// next to each other, and four lanes share a block; the tile is two units of rows x four of columns, 8 KB of codes, which
// are put in order in LDS and leave in whole lines.  Along columns: the tile passes through LDS once, and a lane takes two columns of 32
// rows, i.e. two whole blocks, whose 16-byte codes are neighbours in the transposed matrix.  Both use the same LDS, one after the other.
template <bool BF16, bool ROW, bool COL, bool ROTATE>
__global__ __launch_bounds__(kQuantThreads)
void k_mx4_quantize(const void *in, uint8_t *packed, uint8_t *packed_t, uint32_t rows, uint32_t cols, uint64_t ld,
                    uint32_t cover, uint32_t tiles_x)
{
    constexpr uint32_t RUN = 512 + 32;              // a half unit of codes in LDS: the skew spreads a wavefront's words over the banks
    constexpr int ES = BF16 ? 2 : 4;
    __shared__ __attribute__((aligned(16))) uint8_t lds[COL ? kQuantRows * kQuantCols * ES : 16 * RUN + 512];
    uint8_t *const scale_bytes = lds + 16 * RUN;
    const uint32_t tid = threadIdx.x;
    const uint32_t r0 = blockIdx.x / tiles_x * kQuantRows, c0 = blockIdx.x % tiles_x * kQuantCols;
    const uint32_t chunk = tid % 32, row = tid / 32;
    const uint32_t wide = cols - c0;                // columns from the tile's first on

    Eight<BF16> x[8] = {};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t r = r0 + row + 8 * i;
        if (r < rows && 8 * chunk < wide) x[i] = fetch<BF16, false>(static_cast<const uint8_t *>(in) + ((uint64_t)r * ld + c0) * ES, 8 * chunk, wide, more_behind(r, rows, ld));
    }
    uint32_t w[8] = {}, s[8] = {};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if constexpr (COL) __builtin_memcpy(lds + ((row + 8 * i) * kQuantCols + 8 * chunk) * ES, x[i].q, sizeof x[i].q);
        if constexpr (ROW)
            if (r0 + 8 * i < rows) w[i] = quantize_quad<BF16, ROTATE>(x[i], cover, s[i]);
    }
    TwoColumns<BF16, ROTATE> two;
    if constexpr (COL) {
        __syncthreads();
        two.take(lds + (tid / 128 * 32 * kQuantCols + 2 * (tid % 128)) * ES, kQuantCols * ES);
        if constexpr (ROW) __syncthreads();
    }
    if constexpr (ROW) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t r = row + 8 * i, unit = r / 32 * 4 + chunk / 8, half = chunk / 4 % 2;
            *reinterpret_cast<uint32_t *>(lds + (unit * 2 + half) * RUN + r % 32 * 16 + chunk % 4 * 4) = w[i];
            if (chunk % 4 == 0) scale_bytes[(r / 32 * 64 + half * 32 + r % 32) * 4 + chunk / 8] = (uint8_t)s[i];
        }
        __syncthreads();
        const Mx4Layout L(rows, cols);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t at = (i * kQuantThreads + tid) * 16, unit = at / 1024;
            const uint32_t rb = r0 / 32 + unit / 4, kb = c0 / 64 + unit % 4;
            if (rb < L.rb && kb < L.kb)
                *reinterpret_cast<uint4 *>(packed + ((uint64_t)rb * L.kb + kb) * 1024 + at % 1024) =
                    *reinterpret_cast<const uint4 *>(lds + at / 512 * RUN + at % 512);
        }
        if (tid < 128) {
            const uint32_t rb = r0 / 32 + tid / 64;
            if (rb < L.rb)
                reinterpret_cast<uint32_t *>(packed + L.scales())[((uint64_t)rb * L.kc + c0 / 256) * 64 + tid % 64] =
                    reinterpret_cast<const uint32_t *>(scale_bytes)[tid];
        }
    }
    if constexpr (COL) {
        // two columns x 32 rows: blocks r0/32 + tid/128 of rows c0 + 2 * (tid % 128) of the transposed matrix
        const Mx4Layout L(cols, rows);
        const uint32_t c = c0 + 2 * (tid % 128), b = r0 / 32 + tid / 128;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            uint32_t w4[4], e;
            two.codes(j, cover, w4, e);
            if (c + j < 32 * L.rb) {                                       // rows behind `cols` hold zeros, as the tile does
                if (b / 2 < L.kb) *reinterpret_cast<uint4 *>(packed_t + L.code(c + j, b)) = make_uint4(w4[0], w4[1], w4[2], w4[3]);
                packed_t[L.scale(c + j, b)] = (uint8_t)e;                  // also of the blocks that fill up the last four
            }
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
