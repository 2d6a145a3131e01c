// What kernels that multiply tiles on the matrix cores share: the order of tiles, waits, results' stores.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "tahq_mx4_common.hpp"

namespace tahq {

typedef float float16v __attribute__((ext_vector_type(16)));

// Workgroups go around the eight dies, each with a cache of its own: numbers that a die gets follow each other.
__device__ __forceinline__ uint32_t by_die(uint32_t id, uint32_t total)
{
    const uint32_t die = id % 8, extra = total % 8;
    return die * (total / 8) + min(die, extra) + id / 8;
}
// Tiles one after another in strips of eight rows of tiles
__device__ __forceinline__ void tile_at(uint32_t id, uint32_t tiles_m, uint32_t tiles_n, uint32_t &tm, uint32_t &tn)
{
    const uint32_t strip = id / (8 * tiles_n), at = id % (8 * tiles_n), height = min(tiles_m - strip * 8, 8u);
    tm = strip * 8 + at % height;
    tn = at / height;
}
// A die gets neighbouring tiles
__device__ __forceinline__ void tile_of(uint32_t id, uint32_t tiles_m, uint32_t tiles_n, uint32_t &tm, uint32_t &tn)
{
    tile_at(by_die(id, tiles_m * tiles_n), tiles_m, tiles_n, tm, tn);
}

// s_waitcnt's operand: at most `vm` loads and `lgkm` LDS accesses outstanding (no exports are)
constexpr int waitcnt(int vm, int lgkm) { return (vm & 15) | 7 << 4 | lgkm << 8 | (vm >> 4) << 14; }

// what was read is used here: the reads are not moved behind this place
__device__ __forceinline__ void pin(uint4 &v) { asm volatile("" : "+v"(v.x), "+v"(v.y), "+v"(v.z), "+v"(v.w)); }

typedef const __attribute__((address_space(1))) void *GlobalPtr;
typedef __attribute__((address_space(3))) void *LdsPtr;

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

// ---------------------------------------------------------------- tiles through LDS

// Eight bf16 or four fp32 neighbours of a row of C, of which `valid` are there; fp32 may be added to what is there
template <bool BF16>
__device__ __forceinline__ void store16(void *c, uint64_t at, uint32_t valid, uint4 x, bool accumulate)
{
    constexpr uint32_t COUNT = BF16 ? 8 : 4;
    uint32_t w[4] = {x.x, x.y, x.z, x.w};
    if constexpr (!BF16) {
        if (accumulate)
#pragma unroll
            for (uint32_t i = 0; i < 4; ++i)
                if (i < valid) w[i] = __float_as_uint(__uint_as_float(w[i]) + static_cast<const float *>(c)[at + i]);
    }
    if (valid >= COUNT) {
        __builtin_memcpy(static_cast<uint8_t *>(c) + at * (16 / COUNT), w, 16);
    } else {
#pragma unroll
        for (uint32_t i = 0; i < COUNT; ++i)
            if (i < valid) {
                if constexpr (BF16) static_cast<uint16_t *>(c)[at + i] = (uint16_t)(w[i / 2] >> (i % 2 * 16));
                else static_cast<uint32_t *>(c)[at + i] = w[i];
            }
    }
}

}  // namespace tahq
