// Sums over the lanes of a wavefront: device functions that several translation units use.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace tahq {

// Sum over a wavefront, the same in every lane: pairs, quads, eights and sixteens by permutations within rows of sixteen lanes, then the four rows.
template <int CTRL>
__device__ __forceinline__ float add_permuted(float v)
{
    return v + __uint_as_float((uint32_t)__builtin_amdgcn_mov_dpp((int)__float_as_uint(v), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ float wave_sum(float v)
{
    v = add_permuted<0xb1>(v);                             // lane ^ 1
    v = add_permuted<0x4e>(v);                             // lane ^ 2
    v = add_permuted<0x141>(v);                            // mirrored in eight: the other quad
    v = add_permuted<0x140>(v);                            // mirrored in sixteen: the other eight
    const int w = (int)__float_as_uint(v);
    auto row = [&](int lane) { return __uint_as_float((uint32_t)__builtin_amdgcn_readlane(w, lane)); };
    return (row(0) + row(16)) + (row(32) + row(48));
}

}  // namespace tahq
