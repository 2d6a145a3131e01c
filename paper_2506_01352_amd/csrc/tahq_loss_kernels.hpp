// Softmax cross entropy over a vocabulary and its gradients (include/tahq_loss.h).
//
// Forward: the hidden states of the tokens that count are gathered, with their rows filled up to whole stages; every tile of logits leaves the
// largest logit and the sum of exp(l - largest) of each of its rows and the logits of the targets in it; these are joined.  Backward, for a
// piece of the vocabulary at a time: the piece's logits again, turned into p - [v = t], which go to the workspace; their product with the
// weight's piece, added up over the pieces; their product with the hidden states, the piece of the weight's gradient.
#pragma once
#include "tahq_lanes.hpp"
#include "tahq_loss.h"
#include "tahq_loss_tiles.hpp"

namespace tahq {

constexpr uint32_t kLossScan = 4096;         // tokens whose number of those that count is known in front of the gather
constexpr uint32_t kBadTarget = 0xffffffffu;

// What the workspace holds of the tokens that count, in their order: row numbers, targets, and how many there are
struct LossTokens {
    uint32_t *rows, *targets, *count;
};

// ---------------------------------------------------------------- tokens that count

__device__ __forceinline__ uint32_t group_count(uint32_t v, uint32_t (&places)[4])
{
    for (int step = 1; step < 64; step *= 2) v += __shfl_xor(v, step);
    __syncthreads();
    if (threadIdx.x % 64 == 0) places[threadIdx.x / 64] = v;
    __syncthreads();
    return places[0] + places[1] + places[2] + places[3];
}

__global__ __launch_bounds__(256)
void k_loss_count(const int64_t *target, int64_t ignore, uint32_t rows, uint32_t *counts)
{
    __shared__ uint32_t places[4];
    uint32_t n = 0;
    for (uint32_t i = threadIdx.x; i < kLossScan; i += 256) {
        const uint64_t row = (uint64_t)blockIdx.x * kLossScan + i;
        n += row < rows && target[row] != ignore;
    }
    n = group_count(n, places);
    if (threadIdx.x == 0) counts[blockIdx.x] = n;
}

constexpr uint32_t kGatherRows = 16;

// Sixteen tokens to a workgroup, four to a wavefront.  counts: of the spans of kLossScan tokens, NULL if there is one.  zero, zero_also: float
// results of tokens that do not count (NULL: none); grad_x: their gradients.
template <bool BF16>
__global__ __launch_bounds__(256)
void k_loss_gather(const void *x, const int64_t *target, const uint32_t *counts, uint32_t rows, uint32_t cols, uint32_t vocab, int64_t ignore,
                   void *gathered, uint32_t ld, LossTokens tokens, float *zero, float *zero_also, void *grad_x)
{
    constexpr uint32_t ES = BF16 ? 2 : 4, WHOLE = kStageCols<BF16>;
    __shared__ uint32_t places[4];
    const uint32_t first = blockIdx.x * kGatherRows, span = first / kLossScan;
    uint32_t before = 0;
    for (uint32_t i = threadIdx.x; i < span; i += 256) before += counts[i];
    for (uint32_t i = span * kLossScan + threadIdx.x; i < first; i += 256) before += target[i] != ignore;
    before = group_count(before, places);
    const uint32_t lane = threadIdx.x % 64, wave = uniform(threadIdx.x / 64);
    // all sixteen tokens, the same in every wavefront
    const uint32_t row = first + lane % kGatherRows;
    const int64_t t = row < rows ? target[row] : ignore;
    const uint32_t counted = (uint32_t)__ballot(t != ignore) & ((1u << kGatherRows) - 1);
    auto copy = [&](uint32_t from, uint32_t to, bool there) {
        const uint8_t *src = static_cast<const uint8_t *>(x) + (uint64_t)from * cols * ES;
        uint8_t *dst = static_cast<uint8_t *>(gathered) + (uint64_t)to * ld * ES;
        for (uint32_t c = lane * 8; c < ld; c += 512) {
            Eight<BF16> e = {};
            if (there && c < cols) e = fetch<BF16, false>(src, c, cols, false);
            __builtin_memcpy(__builtin_assume_aligned(dst + c * ES, 16), e.q, sizeof e.q);
        }
    };
    for (uint32_t i = wave * 4; i < wave * 4 + 4; ++i) {
        if (first + i >= rows) break;
        const uint32_t rank = before + __popc(counted & ((1u << i) - 1));
        if (counted >> i & 1) {
            copy(first + i, rank, true);
        } else {
            if (lane == 0) {
                if (zero) zero[first + i] = 0.0f;
                if (zero_also) zero_also[first + i] = 0.0f;
            }
            if (grad_x) {
                const float zeros[8] = {};
                for (uint32_t c = lane * 8; c < cols; c += 512) keep<BF16, false>(static_cast<uint8_t *>(grad_x) + (uint64_t)(first + i) * cols * ES, c, cols, zeros);
            }
        }
    }
    if (wave == 0 && lane < kGatherRows && (counted >> lane & 1)) {
        const uint32_t rank = before + __popc(counted & ((1u << lane) - 1));
        tokens.rows[rank] = row;
        tokens.targets[rank] = t >= 0 && t < (int64_t)vocab ? (uint32_t)t : kBadTarget;
    }
    if (blockIdx.x == gridDim.x - 1) {
        // rows behind the last token up to a whole stage are zeros: they are summed over
        const uint32_t total = before + __popc(counted), end = (max(total, 1u) + WHOLE - 1) / WHOLE * WHOLE;
        for (uint32_t r = total + wave; r < end; r += 4) copy(0, r, false);
        if (threadIdx.x == 0) *tokens.count = total;
    }
}

// A piece of the weight with rows of whole stages, for odd numbers of channels
template <bool BF16>
__global__ __launch_bounds__(256)
void k_loss_pad(const void *weight, void *padded, uint64_t rows, uint32_t cols, uint32_t ld)
{
    constexpr uint32_t ES = BF16 ? 2 : 4;
    const uint64_t per_row = ld / 8;
    for (uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x; i < rows * per_row; i += (uint64_t)gridDim.x * 256) {
        const uint64_t row = i / per_row;
        const uint32_t c = (uint32_t)(i % per_row) * 8;
        Eight<BF16> e = {};
        if (c < cols) e = fetch<BF16, false>(static_cast<const uint8_t *>(weight) + row * cols * ES, c, cols, more_behind((uint32_t)min(row, (uint64_t)0xffffffff), (uint32_t)rows, cols));
        __builtin_memcpy(__builtin_assume_aligned(static_cast<uint8_t *>(padded) + (row * ld + c) * ES, 16), e.q, sizeof e.q);
    }
}

// ---------------------------------------------------------------- tiles

struct LogitArgs {
    const uint8_t *x, *weight;               // gathered hidden states, the piece's first row
    uint64_t ldx, ldw;                       // bytes
    LossTokens tokens;
    uint32_t stages, first, vocab;           // of columns; the piece's first row of the vocabulary, and rows of the vocabulary up to the piece's end
    uint32_t tiles_n;
    float2 *parts;                           // forward: (largest logit, sum of exp(l - it)), [part][padded tokens]
    float *at_target;                        // logits of the targets
    uint32_t part, padded;                   // number of the piece's first part
    const float *lse, *grad_loss;            // backward; grad_loss: of every token, or NULL
    uint8_t *grads;                          // p - [v = t] of the piece, rows of ldg bytes
    uint64_t ldg;
};

enum { kStats = 0, kGrads = 1 };

template <bool BF16, int WM, int WN, int MF, int NF, int PER_CU, int MODE>
__global__ __launch_bounds__(256, PER_CU)
void k_loss_logits(LogitArgs g)
{
    using T = TileKind_<BF16, WM, WN, MF, NF>;
    __shared__ __attribute__((aligned(1024))) uint8_t s0[T::STAGE], s1[T::STAGE], s2[T::STAGE], s3[T::STAGE];
    uint8_t *const stages[4] = {s0, s1, s2, s3};
    const uint32_t count = *g.tokens.count, tiles_m = (max(count, 1u) + T::UM * 32 - 1) / (T::UM * 32);
    if (blockIdx.x >= (uint64_t)tiles_m * g.tiles_n) return;
    uint32_t tm, tn;
    tile_of(blockIdx.x, tiles_m, g.tiles_n, tm, tn);
    TileResult<T> r;
    const Operand a = {g.x, g.ldx, max(count, 1u), 0}, b = {g.weight, g.ldw, g.vocab - g.first, 0};
    multiply_tile<T, BF16, false, false, false>(a, b, tm, tn, 0, g.stages, stages, r);
    const uint32_t lane = threadIdx.x % 64, half = lane / 32, wave = uniform(threadIdx.x / 64);
    const uint32_t m0 = tm * T::UM * 32 + r.m0, n0 = g.first + tn * T::UN * 32 + r.n0;         // n0: in the vocabulary
    auto column = [&](int j, int k) { return n0 + 32 * j + 8 * (k / 4) + 4 * half + k % 4; };
    constexpr float kLog2e = 1.4426950408889634f;
    if constexpr (MODE == kStats) {
#pragma unroll
        for (int i = 0; i < MF; ++i) {
            const uint32_t m = m0 + 32 * i + lane % 32, target = m < count ? g.tokens.targets[m] : kBadTarget;
            float top = -INFINITY;
#pragma unroll
            for (int j = 0; j < NF; ++j)
#pragma unroll
                for (int k = 0; k < 16; ++k) {
                    if (column(j, k) >= g.vocab) r.acc[i][j][k] = -INFINITY;
                    top = fmaxf(top, r.acc[i][j][k]);
                }
            if (target - n0 < (uint32_t)NF * 32) {
#pragma unroll
                for (int j = 0; j < NF; ++j)
#pragma unroll
                    for (int k = 0; k < 16; ++k)
                        if (column(j, k) == target) g.at_target[m] = r.acc[i][j][k];
            }
            top = fmaxf(top, __shfl_xor(top, 32));
            const float shift = top == -INFINITY ? 0.0f : top;               // a part without a logit above -infinity: its sum is 0
            float sum = 0.0f;
#pragma unroll
            for (int j = 0; j < NF; ++j)
#pragma unroll
                for (int k = 0; k < 16; ++k) sum += __builtin_amdgcn_exp2f((r.acc[i][j][k] - shift) * kLog2e);
            sum += __shfl_xor(sum, 32);
            if (half == 0 && m < count) g.parts[(uint64_t)(g.part + tn * WN + wave % WN) * g.padded + m] = make_float2(top, sum);
        }
    } else {
        constexpr uint32_t WHOLE = kStageCols<BF16>;
        const uint32_t end = (max(count, 1u) + WHOLE - 1) / WHOLE * WHOLE;   // rows that are summed over: zeros behind the last token
        float lse[MF], factor[MF];
        uint32_t target[MF];
#pragma unroll
        for (int i = 0; i < MF; ++i) {
            const uint32_t m = m0 + 32 * i + lane % 32;
            const bool there = m < count;
            const uint32_t row = there ? g.tokens.rows[m] : 0;
            target[i] = there ? g.tokens.targets[m] : kBadTarget;
            lse[i] = there ? g.lse[row] : 0.0f;
            factor[i] = there && g.grad_loss ? g.grad_loss[row] : 1.0f;
            if (there && target[i] == kBadTarget) factor[i] = NAN;
        }
        store_tile<T>(r, stages, [&](int i, int j, int k) {
            const uint32_t m = m0 + 32 * i + lane % 32, v = column(j, k);
            const float p = __builtin_amdgcn_exp2f((r.acc[i][j][k] - lse[i]) * kLog2e);
            return m < count && v < g.vocab ? (v == target[i] ? p - 1.0f : p) * factor[i] : 0.0f;
        }, [&](uint32_t m, uint32_t n, const float (&x)[4]) {
            m += tm * T::UM * 32;
            const uint64_t at = (uint64_t)(tn * T::UN * 32 + n) * T::ES;
            if (m < end && at < g.ldg) {
                uint8_t *to = g.grads + m * g.ldg + at;
                if constexpr (BF16) *reinterpret_cast<uint2 *>(to) = make_uint2(two_bf16(x[0], x[1]), two_bf16(x[2], x[3]));
                else *reinterpret_cast<float4 *>(to) = make_float4(x[0], x[1], x[2], x[3]);
            }
        });
    }
}

// The gradient that the reduced loss came back with, over the number of tokens if it is their mean
__device__ __forceinline__ float loss_scale(const float *grad_loss, uint32_t mean, uint32_t count)
{
    const float g = grad_loss ? *grad_loss : 1.0f;
    return mean ? g / (float)max(count, 1u) : g;
}

// Sums over the vocabulary's piece: [part][tokens][cols], part blockIdx.y of the piece's stages, `run` each; `add` to what earlier pieces left
struct GradXArgs {
    const uint8_t *grads, *weight;
    uint64_t ldg, ldw;
    LossTokens tokens;
    uint32_t rows, cols, stages, run, tiles_n, padded, add;
    float *sums;
};
template <bool BF16, int WM, int WN, int MF, int NF, int PER_CU>
__global__ __launch_bounds__(256, PER_CU)
void k_loss_grad_x(GradXArgs g)
{
    using T = TileKind_<BF16, WM, WN, MF, NF>;
    __shared__ __attribute__((aligned(1024))) uint8_t s0[T::STAGE], s1[T::STAGE], s2[T::STAGE], s3[T::STAGE];
    uint8_t *const stages[4] = {s0, s1, s2, s3};
    const uint32_t count = *g.tokens.count, tiles_m = (count + T::UM * 32 - 1) / (T::UM * 32);
    if (blockIdx.x >= (uint64_t)tiles_m * g.tiles_n) return;
    uint32_t tm, tn;
    tile_of(blockIdx.x, tiles_m, g.tiles_n, tm, tn);
    TileResult<T> r;
    const Operand a = {g.grads, g.ldg, count, 0}, b = {g.weight, g.ldw, g.cols, g.rows};
    const uint32_t from = blockIdx.y * g.run;
    multiply_tile<T, BF16, false, true, true>(a, b, tm, tn, from, min(g.run, g.stages - from), stages, r);
    float *to = g.sums + (uint64_t)blockIdx.y * g.padded * g.cols;
    store_tile<T>(r, stages, [&](int i, int j, int k) { return r.acc[i][j][k]; }, [&](uint32_t m, uint32_t n, const float (&x)[4]) {
        m += tm * T::UM * 32;
        n += tn * T::UN * 32;
        if (m < count && n < g.cols)
            store16<false>(to, (uint64_t)m * g.cols + n, g.cols - n, make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])), g.add != 0);
    });
}

// The hidden states' gradient from its sums, to the tokens' own rows
template <bool BF16>
__global__ __launch_bounds__(256)
void k_loss_scatter(const float *sums, uint32_t parts, uint32_t padded, LossTokens tokens, uint32_t cols, const float *grad_loss, uint32_t mean, void *grad_x)
{
    constexpr uint32_t ES = BF16 ? 2 : 4;
    const uint32_t lane = threadIdx.x % 64, count = *tokens.count;
    const float scale = loss_scale(grad_loss, mean, count);
    for (uint32_t r = blockIdx.x * 4 + uniform(threadIdx.x / 64); r < count; r += gridDim.x * 4) {
        uint8_t *to = static_cast<uint8_t *>(grad_x) + (uint64_t)tokens.rows[r] * cols * ES;
        for (uint32_t c = lane * 8; c < cols; c += 512) {
            float v[8] = {};
            for (uint32_t p = 0; p < parts; ++p) {
                const Eight<false> e = fetch<false, false>(sums + ((uint64_t)p * padded + r) * cols, c, cols, false);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] += e[i];
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] *= scale;
            keep<BF16, false>(to, c, cols, v);
        }
    }
}

struct GradWArgs {
    const uint8_t *grads, *x;
    uint64_t ldg, ldx;
    LossTokens tokens;
    uint32_t rows, cols, tiles_m, tiles_n;   // rows of the piece
    const float *grad_loss;                  // of the reduced loss, or NULL
    uint32_t mean, out_bf16, accumulate;
    void *out;                               // the gradient's first row of the piece
};
template <bool BF16, int WM, int WN, int MF, int NF, int PER_CU>
__global__ __launch_bounds__(256, PER_CU)
void k_loss_grad_w(GradWArgs g)
{
    using T = TileKind_<BF16, WM, WN, MF, NF>;
    __shared__ __attribute__((aligned(1024))) uint8_t s0[T::STAGE], s1[T::STAGE], s2[T::STAGE], s3[T::STAGE];
    uint8_t *const stages[4] = {s0, s1, s2, s3};
    const uint32_t count = *g.tokens.count, depth = (max(count, 1u) + T::COLS - 1) / T::COLS;
    uint32_t tm, tn;
    tile_of(blockIdx.x, g.tiles_m, g.tiles_n, tm, tn);
    TileResult<T> r;
    const Operand a = {g.grads, g.ldg, g.rows, 0}, b = {g.x, g.ldx, g.cols, 0};
    multiply_tile<T, BF16, true, true, false>(a, b, tm, tn, 0, depth, stages, r);
    const float scale = loss_scale(g.grad_loss, g.mean, count);
    store_tile<T>(r, stages, [&](int i, int j, int k) { return r.acc[i][j][k] * scale; }, [&](uint32_t m, uint32_t n, const float (&x)[4]) {
        m += tm * T::UM * 32;
        n += tn * T::UN * 32;
        if (m >= g.rows || n >= g.cols) return;
        float y[4] = {x[0], x[1], x[2], x[3]};
        if (g.out_bf16) store4<true>(g.out, g.cols, m, n, g.cols, y, g.accumulate != 0);
        else store4<false>(g.out, g.cols, m, n, g.cols, y, g.accumulate != 0);
    });
}

// ---------------------------------------------------------------- joining

// 32 tokens to a workgroup, the parts in eight runs.  `later`: with what earlier pieces of the vocabulary left in `running`; `last`: there is no
// piece after this one.
__global__ __launch_bounds__(256)
void k_loss_join(const float2 *from, uint32_t parts, uint32_t padded, LossTokens tokens, const float *at_target, float2 *running, uint32_t later,
                 uint32_t last, float *losses, float *lse)
{
    __shared__ float2 places[8][32];
    const uint32_t lane = threadIdx.x % 32, run = threadIdx.x / 32, count = *tokens.count, r = blockIdx.x * 32 + lane;
    if (blockIdx.x * 32 >= count) return;
    auto joined = [](float2 a, float2 b) {
        const float top = fmaxf(a.x, b.x), shift = top == -INFINITY ? 0.0f : top;
        return make_float2(top, a.y * __expf(a.x - shift) + b.y * __expf(b.x - shift));
    };
    float2 v = make_float2(-INFINITY, 0.0f);
    if (r < count)
        for (uint32_t p = run; p < parts; p += 8) v = joined(v, from[(uint64_t)p * padded + r]);
    places[run][lane] = v;
    __syncthreads();
    if (run == 0 && r < count) {
        for (int i = 1; i < 8; ++i) v = joined(v, places[i][lane]);
        if (later) v = joined(running[r], v);
        if (!last) {
            running[r] = v;
            return;
        }
        const float all = v.x + logf(v.y);
        const uint32_t row = tokens.rows[r];
        lse[row] = all;
        losses[row] = tokens.targets[r] == kBadTarget ? NAN : all - at_target[r];
    }
}

// The reduced loss and the number of tokens that count
__global__ __launch_bounds__(1024)
void k_loss_total(const float *losses, uint32_t rows, LossTokens tokens, uint32_t mean, float *total)
{
    __shared__ float sums[1024];
    float sum = 0.0f;
    for (uint64_t i = threadIdx.x; i < rows; i += 1024) sum += losses[i];
    sums[threadIdx.x] = sum;
    __syncthreads();
    for (uint32_t half = 512; half; half /= 2) {
        if (threadIdx.x < half) sums[threadIdx.x] += sums[threadIdx.x + half];
        __syncthreads();
    }
    if (threadIdx.x == 0) {
        const uint32_t count = *tokens.count;
        total[0] = mean ? sums[0] / (float)max(count, 1u) : sums[0];
        total[1] = (float)count;
    }
}

}  // namespace tahq
