// Dropout with a residual (include/tahq_dropout.h): kernel, validation, launch.
#include "tahq_dropout.h"
#include "tahq_enqueue.hpp"
#include "tahq_mx4_common.hpp"

using namespace tahq;

namespace {

constexpr uint32_t kDropLanes = 256;

struct Mask {
    uint64_t seed, offset;
    uint32_t threshold;
    float scale;
};

// Philox 4x32, ten rounds: two products of 32 bits a round, whose halves change places with what the key turns over
__device__ __forceinline__ uint4 philox(uint64_t counter, uint64_t offset, uint64_t seed)
{
    uint32_t c0 = (uint32_t)counter, c1 = (uint32_t)(counter >> 32), c2 = (uint32_t)offset, c3 = (uint32_t)(offset >> 32);
    uint32_t k0 = (uint32_t)seed, k1 = (uint32_t)(seed >> 32);
#pragma unroll
    for (int i = 0; i < 10; ++i) {
        const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
        c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
        c1 = (uint32_t)b;
        c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
        c3 = (uint32_t)a;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return make_uint4(c0, c1, c2, c3);
}

// Eight elements to a lane, which are one counter's (ten rounds of two products): bound by memory, three tensors with a residual and two without.  bf16
// 32768 x 8192 with a residual 266 us, 6.05 TB/s; fp32 2331 x 1600 without 7.8 us out of the last cache, 10.0 out of HBM; 128 x 512 2.5 us, a launch.  A
// workgroup to every 2048 elements: they are so many, and so short, that they balance by themselves.
template <bool BF16, bool RESIDUAL>
__global__ __launch_bounds__(kDropLanes)
void k_dropout(const void *x, const void *residual, void *out, const uint64_t *more_offset, Mask mask, uint64_t elements)
{
    constexpr uint32_t ES = BF16 ? 2 : 4;
    const uint64_t offset = mask.offset + (more_offset ? *more_offset : 0), blocks = (elements + 7) / 8;
    for (uint64_t b = (uint64_t)blockIdx.x * kDropLanes + threadIdx.x; b < blocks; b += (uint64_t)gridDim.x * kDropLanes) {
        const uint32_t valid = (uint32_t)min(elements - 8 * b, (uint64_t)8);
        const uint8_t *const from = static_cast<const uint8_t *>(x) + 8 * b * ES;
        const Eight<BF16> v = fetch<BF16, false>(from, 0, valid, false);
        Eight<BF16> r = {};
        if constexpr (RESIDUAL) r = fetch<BF16, false>(static_cast<const uint8_t *>(residual) + 8 * b * ES, 0, valid, false);
        const uint4 w = philox(b, offset, mask.seed);
        float y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t word = i < 2 ? w.x : i < 4 ? w.y : i < 6 ? w.z : w.w;
            const bool kept = (i % 2 ? word >> 16 : word & 0xffffu) >= mask.threshold;
            y[i] = kept ? v[i] * mask.scale : 0.0f;
            if constexpr (RESIDUAL) y[i] = r[i] + y[i];
        }
        keep<BF16, false>(static_cast<uint8_t *>(out) + 8 * b * ES, 0, valid, y);
    }
}

tahq_status check(const tahq_dropout_config *c)
{
    if (!c) return TAHQ_ERR_NULL;
    if (c->struct_size != sizeof *c || c->dtype > TAHQ_BF16) return TAHQ_ERR_INVALID_ARG;
    if (c->elements == 0 || c->elements > (uint64_t)1 << 48) return TAHQ_ERR_INVALID_ARG;
    if (!(c->p >= 0.0f && c->p <= 1.0f)) return TAHQ_ERR_INVALID_ARG;
    return TAHQ_OK;
}

tahq_status enqueue(const tahq_dropout_config *cfg, const void *d_x, const void *d_residual, void *d_out, const uint64_t *d_offset, tahq_stream stream)
{
    const tahq_status rc = check(cfg);
    if (rc != TAHQ_OK) return rc;
    if (!d_x || !d_out) return TAHQ_ERR_NULL;
    for (const void *p : {d_x, d_residual, (const void *)d_out})
        if (misaligned(p)) return TAHQ_ERR_MISALIGNED;
    if (reinterpret_cast<uintptr_t>(d_offset) % sizeof *d_offset) return TAHQ_ERR_MISALIGNED;
    const uint32_t t = (uint32_t)__builtin_floor((double)cfg->p * 65536.0 + 0.5);
    const Mask mask = {cfg->seed, cfg->offset, t, t < 65536u ? (float)(65536.0 / (65536.0 - t)) : 0.0f};
    const uint64_t groups = ((cfg->elements + 7) / 8 + kDropLanes - 1) / kDropLanes, most = 1u << 20;
    const dim3 grid((uint32_t)(groups < most ? groups : most));
    const bool bf16 = cfg->dtype == TAHQ_BF16;
    Enqueue q{(hipStream_t)stream};
    q(d_residual ? (bf16 ? k_dropout<true, true> : k_dropout<false, true>) : (bf16 ? k_dropout<true, false> : k_dropout<false, false>), grid,
      dim3(kDropLanes), d_x, d_residual, d_out, d_offset, mask, cfg->elements);
    return q.result();
}

}  // namespace

extern "C" {

void tahq_dropout_config_default(tahq_dropout_config *cfg)
{
    if (!cfg) return;
    *cfg = tahq_dropout_config{};
    cfg->struct_size = (uint32_t)sizeof *cfg;
    cfg->dtype = TAHQ_BF16;
    cfg->p = 0.1f;
}

tahq_status tahq_dropout_forward(const tahq_dropout_config *cfg, const void *d_x, const void *d_residual, void *d_out,
                                 const uint64_t *d_offset, tahq_stream stream)
{
    return enqueue(cfg, d_x, d_residual, d_out, d_offset, stream);
}

tahq_status tahq_dropout_backward(const tahq_dropout_config *cfg, const void *d_grad_out, void *d_grad_x, const uint64_t *d_offset,
                                  tahq_stream stream)
{
    return enqueue(cfg, d_grad_out, nullptr, d_grad_x, d_offset, stream);
}

}  // extern "C"
