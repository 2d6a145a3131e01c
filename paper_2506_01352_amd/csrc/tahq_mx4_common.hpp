// Layout and numerics of packed mx4 matrices (include/tahq_mx4.h), shared by the quantizer, the products and the norm that
// quantizes its output.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "tahq_mx4.h"

namespace tahq {

constexpr float kRoot32 = 0.17677669529663687f;            // fp32(1 / sqrt(32))
constexpr uint32_t kCover = 0x3fffffu;                     // see block_scale

// Rows and columns come in units of the matrix instruction's operand, 32 rows x 64 columns; a lane's four scale bytes belong to
// four such units side by side, so that one register serves 256 columns (the instruction picks the byte).
struct Mx4Layout {
    uint32_t rb, kb, kc;
    __host__ __device__ Mx4Layout(uint32_t rows, uint32_t cols) : rb((rows + 31) / 32), kb((cols + 63) / 64), kc((cols + 255) / 256) {}
    __host__ __device__ uint64_t scales() const { return (uint64_t)rb * kb * 1024; }
    __host__ __device__ uint64_t total() const { return scales() + (uint64_t)rb * kc * 256; }
    // 16 bytes of codes, and the scale's byte, of row r's block b
    __host__ __device__ uint64_t code(uint32_t r, uint32_t b) const
    {
        return ((uint64_t)(r / 32) * kb + b / 2) * 1024 + (b % 2) * 512 + (r % 32) * 16;
    }
    __host__ __device__ uint64_t scale(uint32_t r, uint32_t b) const
    {
        return scales() + ((uint64_t)(r / 32) * kc + b / 8) * 256 + (b % 2) * 128 + (r % 32) * 4 + b / 2 % 4;
    }
};

__device__ __forceinline__ uint32_t uniform(uint32_t v) { return __builtin_amdgcn_readfirstlane(v); }

// ---------------------------------------------------------------- loads

template <bool BF16>
__device__ __forceinline__ float load1(const void *base, uint64_t at)
{
    if constexpr (BF16) return __uint_as_float((uint32_t)static_cast<const uint16_t *>(base)[at] << 16);
    else return static_cast<const float *>(base)[at];
}
// two fp32 to bf16, nearest even (v_cvt_pk_bf16_f32)
__device__ __forceinline__ uint32_t two_bf16(float lo, float hi)
{
    typedef __bf16 pair __attribute__((ext_vector_type(2)));
    const pair p = {(__bf16)lo, (__bf16)hi};
    return __builtin_bit_cast(uint32_t, p);
}
template <bool BF16>
__device__ __forceinline__ void store1(void *base, uint64_t at, float x)
{
    if constexpr (BF16) static_cast<uint16_t *>(base)[at] = (uint16_t)two_bf16(x, 0.0f);
    else static_cast<float *>(base)[at] = x;
}
// Eight elements of a lane as they lie in memory
template <bool BF16>
struct Eight {
    uint4 q[BF16 ? 1 : 2];
    __device__ __forceinline__ float operator[](int i) const
    {
        const uint4 &p = q[BF16 ? 0 : i / 4];
        const int k = BF16 ? i / 2 : i % 4;
        const uint32_t w = k == 0 ? p.x : k == 1 ? p.y : k == 2 ? p.z : p.w;
        return __uint_as_float(!BF16 ? w : i % 2 ? w & 0xffff0000u : w << 16);
    }
};
// Rows need no alignment beyond their elements': a 16-byte access may start anywhere.  EIGHTS: rows of whole eights.
// Elements c .. c + 7 of a row of C, of which the first is there; zeros behind the row's end.  `more`: seven elements behind it can be
// read, too, as they can in all rows but the last: a row's end then takes no more loads than the rest of it (norms of 16384 x 2047 bf16,
// which wait for a row's last wavefront: backward 172 -> 118 us, forward 112 -> 84).
template <bool BF16, bool EIGHTS>
__device__ __forceinline__ Eight<BF16> fetch(const void *row, uint32_t c, uint32_t C, bool more)
{
    constexpr uint32_t ES = BF16 ? 2 : 4, WORDS = BF16 ? 4 : 8;
    Eight<BF16> e;
    if (EIGHTS || more || c + 8 <= C) {
        __builtin_memcpy(e.q, static_cast<const uint8_t *>(row) + c * ES, sizeof e.q);
        if (!EIGHTS && c + 8 > C) {
            uint32_t w[WORDS];
            __builtin_memcpy(w, e.q, sizeof w);
#pragma unroll
            for (uint32_t i = 0; i < WORDS; ++i) {
                if constexpr (BF16) w[i] = c + 2 * i + 1 < C ? w[i] : c + 2 * i < C ? w[i] & 0xffffu : 0u;
                else w[i] = c + i < C ? w[i] : 0u;
            }
            __builtin_memcpy(e.q, w, sizeof w);
        }
        return e;
    }
    asm volatile("");                                      // keeps the two ways apart: joined, both would go element by element
    uint32_t w[WORDS] = {};
#pragma unroll
    for (uint32_t i = 0; i < 7; ++i)
        if (c + i < C) {
            if constexpr (BF16) w[i / 2] |= (uint32_t)static_cast<const uint16_t *>(row)[c + i] << (i % 2 * 16);
            else w[i] = static_cast<const uint32_t *>(row)[c + i];
        }
    __builtin_memcpy(e.q, w, sizeof e.q);
    return e;
}
// Whether seven elements behind row r's end are still in the tensor
__device__ __forceinline__ bool more_behind(uint32_t r, uint32_t rows, uint64_t ld) { return r + 7 < rows || (r + 1 < rows && ld >= 7); }
// what fetch reads
template <bool BF16, bool EIGHTS>
__device__ __forceinline__ void keep(void *row, uint32_t c, uint32_t C, const float (&x)[8])
{
    constexpr uint32_t ES = BF16 ? 2 : 4, WORDS = BF16 ? 4 : 8;
    uint8_t *to = static_cast<uint8_t *>(row) + c * ES;
    uint32_t w[WORDS];
#pragma unroll
    for (uint32_t i = 0; i < WORDS; ++i) w[i] = BF16 ? two_bf16(x[2 * i % 8], x[(2 * i + 1) % 8]) : __float_as_uint(x[i]);
    if (EIGHTS || c + 8 <= C) {
        __builtin_memcpy(to, w, sizeof w);
        return;
    }
    asm volatile("");
    if constexpr (BF16) {
        const uint32_t left = C - c;                       // 1 .. 7: four, two and one of them
        if (left & 4) {
            __builtin_memcpy(to, w, 8);
            to += 8;
            w[0] = w[2];
            w[1] = w[3];
        }
        if (left & 2) {
            __builtin_memcpy(to, w, 4);
            to += 4;
            w[0] = w[1];
        }
        if (left & 1) *reinterpret_cast<uint16_t *>(to) = (uint16_t)w[0];
    } else {
#pragma unroll
        for (uint32_t i = 0; i < 7; ++i)
            if (c + i < C) __builtin_memcpy(to + 4 * i, w + i, 4);
    }
}

// ---------------------------------------------------------------- a block

// the value of the lane whose number differs in bit 0 (CTRL 0xb1) or bit 1 (0x4e): quad permutations
template <int CTRL>
__device__ __forceinline__ uint32_t quad(uint32_t v)
{
    return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, CTRL, 0xf, 0xf, true);
}
template <int CTRL>
__device__ __forceinline__ float quadf(float v) { return __uint_as_float(quad<CTRL>(__float_as_uint(v))); }

// butterflies h = 1, 2, .. N/2 on the N elements of one lane
template <int N>
__device__ __forceinline__ void butterfly(float (&x)[N])
{
#pragma unroll
    for (int h = 1; h < N; h *= 2)
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (!(i & h)) {
                const float a = x[i], b = x[i + h];
                x[i] = a + b;
                x[i + h] = a - b;
            }
}
// a block whose four lanes hold eight elements each
__device__ __forceinline__ void rotate_quad(float (&x)[8])
{
    butterfly(x);
    const uint32_t lane = threadIdx.x;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float o = quadf<0xb1>(x[i]);
        x[i] = lane & 1 ? o - x[i] : x[i] + o;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float o = quadf<0x4e>(x[i]);
        x[i] = (lane & 2 ? o - x[i] : x[i] + o) * kRoot32;
    }
}

// The scale byte of a block from the bits of its largest magnitude (as an integer the largest, too; infinities and NaN are above
// all others).  The exponent field less 2; the cover rule counts a magnitude above 1.5 * 2^e, i.e. above 6 units, to the next
// exponent: adding 0x3fffff to the bits carries into the exponent exactly for a fraction above 0x400000.
__device__ __forceinline__ uint32_t block_scale(uint32_t top, uint32_t cover)
{
    const uint32_t e = (top + cover) >> 23;
    const uint32_t s = e > 2 ? e - 2 : 0;
    return top >= 0x7f800000u ? 255u : s;
}
// 2^(s - 127), as the conversion takes it
__device__ __forceinline__ float scale_value(uint32_t s) { return __uint_as_float(s ? s << 23 : 0x400000u); }

// eight elements to codes, low half of the first byte first
__device__ __forceinline__ uint32_t codes8(const float (&x)[8], uint32_t s)
{
    const float v = scale_value(s);
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], v, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], v, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], v, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], v, 3);
    return s == 255u ? 0u : w;
}

// eight bf16, two to a word
__device__ __forceinline__ uint32_t codes8(const uint4 &q, uint32_t s)
{
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    const float v = scale_value(s);
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, q.x), v, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, q.y), v, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, q.z), v, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, q.w), v, 3);
    return s == 255u ? 0u : w;
}

template <bool BF16>
__device__ __forceinline__ void unpack(const Eight<BF16> &e, float (&x)[8])
{
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = e[i];
}
// A block of which four neighbouring lanes hold eight elements each: its codes (this lane's) and scale byte
template <bool ROTATE>
__device__ __forceinline__ uint32_t quantize_quad(float (&x)[8], uint32_t cover, uint32_t &s)
{
    if constexpr (ROTATE) rotate_quad(x);
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
    top = max(top, quad<0xb1>(top));
    top = max(top, quad<0x4e>(top));
    s = block_scale(top, cover);
    return codes8(x, s);
}

// The same of bf16 as it lies in memory: magnitudes of bf16 are ordered like 16-bit integers
__device__ __forceinline__ uint32_t quantize_quad(const uint4 &q, uint32_t cover, uint32_t &s)
{
    typedef uint16_t pair __attribute__((ext_vector_type(2)));
    auto magnitude = [](uint32_t w) { return __builtin_bit_cast(pair, w & 0x7fff7fffu); };
    const pair m = __builtin_elementwise_max(__builtin_elementwise_max(magnitude(q.x), magnitude(q.y)),
                                             __builtin_elementwise_max(magnitude(q.z), magnitude(q.w)));
    uint32_t top = (uint32_t)max(m.x, m.y) << 16;
    top = max(top, quad<0xb1>(top));
    top = max(top, quad<0x4e>(top));
    s = block_scale(top, cover);
    return codes8(q, s);
}

template <bool BF16, bool ROTATE>
__device__ __forceinline__ uint32_t quantize_quad(const Eight<BF16> &e, uint32_t cover, uint32_t &s)
{
    if constexpr (BF16 && !ROTATE) {
        return quantize_quad(e.q[0], cover, s);
    } else {
        float x[8];
        unpack(e, x);
        return quantize_quad<ROTATE>(x, cover, s);
    }
}

// the numbers that eight codes and their block's scale byte stand for
__device__ __forceinline__ void values8(uint32_t w, uint32_t s, float (&x)[8])
{
    typedef float pair __attribute__((ext_vector_type(2)));
    const float v = scale_value(s);
    const pair p[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, v, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, v, 1),
                       __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, v, 2), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, v, 3)};
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = s == 255u ? __uint_as_float(0x7fc00000u) : i % 2 ? p[i / 2].y : p[i / 2].x;
}

}  // namespace tahq
