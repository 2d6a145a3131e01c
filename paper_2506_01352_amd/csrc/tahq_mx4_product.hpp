// C = A B^T of two packed mx4 matrices on the matrix cores (v_mfma_scale_f32_32x32x64_f8f6f4, 4-bit operands, fp32 sums).
#pragma once
#include "tahq_mx4_common.hpp"

namespace tahq {

typedef int int8v __attribute__((ext_vector_type(8)));
typedef float float16v __attribute__((ext_vector_type(16)));

// One instruction: 32 rows of each operand, 64 columns.  A lane holds row lane % 32 of both operands, columns 32 * (lane / 32) on,
// and of D column lane % 32 (second operand's row), rows 8 * (i / 4) + 4 * (lane / 32) + i % 4 (first operand's).  B goes first, so that a lane's
// results are four neighbours of a row of C.  BYTE: which of the four scale bytes.
template <int BYTE>
__device__ __forceinline__ float16v mfma(const uint4 &b, const uint4 &a, const float16v &c, uint32_t sb, uint32_t sa)
{
    const int8v vb = {(int)b.x, (int)b.y, (int)b.z, (int)b.w, 0, 0, 0, 0};
    const int8v va = {(int)a.x, (int)a.y, (int)a.z, (int)a.w, 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(vb, va, c, 4, 4, BYTE, (int)sb, BYTE, (int)sa);
}

// Four neighbours of a row of C: row m, columns n .. n + 3
template <bool BF16>
__device__ __forceinline__ void store4(void *c, uint64_t ldc, uint32_t m, uint32_t n, uint32_t N, float (&v)[4], bool accumulate)
{
    const uint64_t at = (uint64_t)m * ldc + n;
    const bool whole = n + 4 <= N;
    if (accumulate) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (whole || n + i < N) v[i] += load1<BF16>(c, at + i);
    }
    if (whole) {
        if constexpr (BF16) {
            const uint32_t w[2] = {two_bf16(v[0], v[1]), two_bf16(v[2], v[3])};
            __builtin_memcpy(static_cast<uint16_t *>(c) + at, w, 8);
        } else {
            __builtin_memcpy(static_cast<float *>(c) + at, v, 16);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (n + i < N) store1<BF16>(c, at + i, v[i]);
    }
}

// A wavefront takes 64 x 64 of C and reads its operands straight from memory: a unit of codes is 1 KB in a row.
template <bool BF16>
__global__ __launch_bounds__(64)
void k_mx4_product(const uint8_t *__restrict__ a, const uint8_t *__restrict__ b, void *c, uint32_t M, uint32_t N, uint32_t K,
                   uint64_t ldc, uint32_t accumulate, uint32_t tiles_n)
{
    const Mx4Layout LA(M, K), LB(N, K);
    const uint32_t lane = threadIdx.x;
    const uint32_t m0 = blockIdx.x / tiles_n * 64, n0 = blockIdx.x % tiles_n * 64;
    // units behind the last row are not there: the last one again, whose results are not stored
    uint32_t ra[2], rb[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        ra[i] = min(m0 / 32 + i, LA.rb - 1);
        rb[i] = min(n0 / 32 + i, LB.rb - 1);
    }
    float16v acc[2][2] = {};
    for (uint32_t kc = 0; kc < LA.kc; ++kc) {
        uint32_t sa[2], sb[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            sa[i] = reinterpret_cast<const uint32_t *>(a + LA.scales())[((uint64_t)ra[i] * LA.kc + kc) * 64 + lane];
            sb[i] = reinterpret_cast<const uint32_t *>(b + LB.scales())[((uint64_t)rb[i] * LB.kc + kc) * 64 + lane];
        }
        auto step = [&](auto byte) {
            const uint32_t kb = kc * 4 + byte;
            if (kb >= LA.kb) return;
            uint4 va[2], vb[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                va[i] = reinterpret_cast<const uint4 *>(a)[((uint64_t)ra[i] * LA.kb + kb) * 64 + lane];
                vb[i] = reinterpret_cast<const uint4 *>(b)[((uint64_t)rb[i] * LB.kb + kb) * 64 + lane];
            }
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) acc[i][j] = mfma<decltype(byte)::value>(vb[j], va[i], acc[i][j], sb[j], sa[i]);
        };
        step(std::integral_constant<int, 0>{});
        step(std::integral_constant<int, 1>{});
        step(std::integral_constant<int, 2>{});
        step(std::integral_constant<int, 3>{});
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const uint32_t m = m0 + 32 * i + lane % 32, n = n0 + 32 * j + 8 * g + 4 * (lane / 32);
                float v[4] = {acc[i][j][4 * g], acc[i][j][4 * g + 1], acc[i][j][4 * g + 2], acc[i][j][4 * g + 3]};
                if (m < M && n < N) store4<BF16>(c, ldc, m, n, N, v, accumulate != 0);
            }
}

}  // namespace tahq
