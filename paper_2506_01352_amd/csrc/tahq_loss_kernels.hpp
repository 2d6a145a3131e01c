// Softmax cross entropy over a vocabulary and its gradients (include/tahq_loss.h).
//
// Forward: the hidden states of the tokens that count are gathered, with their rows filled up to whole stages; every tile of logits leaves the largest
// logit and the sum of exp(l - largest) of each of its rows and the logits of the targets in it; these are joined.  Backward, for a piece of the vocabulary
// at a time: the piece's logits again, turned into p - [v = t], which go to the workspace; their product with the weight's piece, added up over the pieces;
// their product with the hidden states, the piece of the weight's gradient.
//
// Bound by the matrix cores where there are hundreds of tokens and more: four products of 2 rows cols vocab operations each, one of them the logits again,
// which costs a fourth of the time and saves logits of 2 rows vocab bytes and more (8192 x 131072 in bf16: 2.1 GB).  8192 x 4096 x 131072 in bf16, by the
// clock that power leaves: logits 6.5 to 6.9 ms, 1.36 to 1.28 PFLOP/s; backward, in pieces of 16384 rows, logits 852 to 887 us, 1.29 to 1.24 PFLOP/s, the
// hidden states' gradient 814 to 841, the weight's 808 to 837.  The matrix cores are busy in 68 to 72 % of the cycles, at 1.7 to 1.8 GHz.  By the weight's
// bytes where there are few: 5 x 1600 x 50257 33 us, 4.9 TB/s, out of the last cache in part; 47 out of HBM, 25 with the weight in the last cache.
#pragma once
#include "tahq_lanes.hpp"
#include "tahq_loss.h"
#include "tahq_loss_plan.hpp"
#include "tahq_loss_tiles.hpp"

namespace tahq {

constexpr uint32_t kBadTarget = 0xffffffffu;

// What the workspace holds of the tokens that count, in their order: row numbers, targets, and how many there are
struct LossTokens {
    uint32_t *rows, *targets, *count;
};

// ---------------------------------------------------------------- tokens that count

template <int WAVES>
__device__ __forceinline__ uint32_t group_count(uint32_t v, uint32_t (&places)[WAVES])
{
    for (int step = 1; step < 64; step *= 2) v += __shfl_xor(v, step);
    if (threadIdx.x % 64 == 0) places[threadIdx.x / 64] = v;
    __syncthreads();
    v = places[0];
#pragma unroll
    for (int i = 1; i < WAVES; ++i) v += places[i];
    return v;
}

__global__ __launch_bounds__(1024)
void k_loss_count(const int64_t *target, int64_t ignore, uint32_t rows, uint32_t *counts)
{
    __shared__ uint32_t places[16];
    uint32_t n = 0;
#pragma unroll
    for (uint32_t i = 0; i < kLossSpan / 1024; ++i) {
        const uint32_t row = min(blockIdx.x * kLossSpan + i * 1024 + threadIdx.x, rows - 1);
        n += target[row] != ignore && row == blockIdx.x * kLossSpan + i * 1024 + threadIdx.x;
    }
    n = group_count(n, places);
    if (threadIdx.x == 0) counts[blockIdx.x] = n;
}

// Eight elements to their place in blocks, or in three planes of them
template <bool BF16, int PLANES>
__device__ __forceinline__ void put_eight(const Eight<BF16> &e, uint8_t *base, uint64_t plane, uint64_t at)
{
    if constexpr (PLANES == 3) {
        float x[8];
        unpack(e, x);
        uint4 p[3];
        split_planes(x, p);
#pragma unroll
        for (int i = 0; i < 3; ++i) *reinterpret_cast<uint4 *>(base + i * plane + at) = p[i];
    } else {
        __builtin_memcpy(__builtin_assume_aligned(base + at, 16), e.q, sizeof e.q);
    }
}

constexpr uint32_t kGatherRows = 4;          // of a workgroup, one to a wavefront

// gathered: blocks of 64 bytes of every row, `padded` rows each, `blocks` of them, of fp32 in planes of bf16 three times.  counts: of the spans of
// kLossSpan tokens, NULL if there is one. Four rows to a workgroup: 8192 x 4096 28 us, 4.8 TB/s; eight would leave compute units idle below 2048 tokens.
// zero, zero_also: float results of tokens that do not count (NULL: none); grad_x: their gradients.
template <bool BF16, int PLANES>
__global__ __launch_bounds__(256)
void k_loss_gather(const void *x, const int64_t *target, const uint32_t *counts, uint32_t rows, uint32_t cols, uint32_t vocab, int64_t ignore,
                   uint8_t *gathered, uint32_t blocks, uint32_t padded, LossTokens tokens, float *zero, float *zero_also, void *grad_x)
{
    constexpr uint32_t ES = BF16 ? 2 : 4, WHOLE = kStageCols<BF16 || PLANES == 3>, AHEAD = 4;
    __shared__ uint32_t places[4];
    const uint32_t first = blockIdx.x * kGatherRows, span = first / kLossSpan, lane = threadIdx.x % 64, wave = uniform(threadIdx.x / 64), row = first + wave;
    // the row is on its way while its place is counted
    Eight<BF16> e[AHEAD];
    auto ask = [&](uint32_t c0) {
        const uint8_t *src = static_cast<const uint8_t *>(x) + (uint64_t)row * cols * ES;
#pragma unroll
        for (uint32_t k = 0; k < AHEAD; ++k) {
            const uint32_t c = c0 + k * 512 + lane * 8;
            e[k] = Eight<BF16>{};
            if (row < rows && c < cols) e[k] = fetch<BF16, false>(src, c, cols, more_behind(row, rows, cols));
        }
    };
    auto put = [&](uint32_t c0, uint32_t to) {
#pragma unroll
        for (uint32_t k = 0; k < AHEAD; ++k) {
            const uint32_t c = c0 + k * 512 + lane * 8;
            if (c < blocks * WHOLE) put_eight<BF16, PLANES>(e[k], gathered, (uint64_t)blocks * padded * 64, ((uint64_t)(c / WHOLE) * padded + to) * 64 + c % WHOLE * (64 / WHOLE));
        }
    };
    ask(0);
    const uint32_t any = first + lane % kGatherRows;         // the workgroup's tokens, the same in every wavefront
    const int64_t t = any < rows ? target[any] : ignore;
    uint32_t before = 0;
    for (uint32_t i = threadIdx.x; i < span; i += 256) before += counts[i];
#pragma unroll 4
    for (uint32_t i = span * kLossSpan + threadIdx.x; i < first; i += 256) before += target[i] != ignore;
    before = group_count(before, places);
    const uint32_t counted = (uint32_t)__ballot(t != ignore) & ((1u << kGatherRows) - 1);
    if (row < rows) {
        const uint32_t rank = before + __popc(counted & ((1u << wave) - 1));
        if (counted >> wave & 1) {
            put(0, rank);
            for (uint32_t c0 = AHEAD * 512; c0 < blocks * WHOLE; c0 += AHEAD * 512) {
                ask(c0);
                put(c0, rank);
            }
            if (lane == wave) {
                tokens.rows[rank] = row;
                tokens.targets[rank] = t >= 0 && t < (int64_t)vocab ? (uint32_t)t : kBadTarget;
            }
        } else {
            if (lane == 0) {
                if (zero) zero[row] = 0.0f;
                if (zero_also) zero_also[row] = 0.0f;
            }
            if (grad_x) {
                const float zeros[8] = {};
                for (uint32_t c = lane * 8; c < cols; c += 512) keep<BF16, false>(static_cast<uint8_t *>(grad_x) + (uint64_t)row * cols * ES, c, cols, zeros);
            }
        }
    }
    if (blockIdx.x == gridDim.x - 1) {
        // rows behind the last token up to a whole stage are zeros: they are summed over
        const uint32_t total = before + __popc(counted), end = (max(total, 1u) + WHOLE - 1) / WHOLE * WHOLE;
#pragma unroll
        for (uint32_t k = 0; k < AHEAD; ++k) e[k] = Eight<BF16>{};
        for (uint32_t r = total + wave; r < end; r += 4)
            for (uint32_t c0 = 0; c0 < blocks * WHOLE; c0 += AHEAD * 512) put(c0, r);
        if (threadIdx.x == 0) *tokens.count = total;
    }
}

// A piece of the weight in blocks, for numbers of channels that are not whole stages, and of fp32 in planes; rows up to whole stages, and channels, are
// filled up with zeros.  Sixteen rows to a workgroup, so that it writes runs of 1 KB.  Bound by memory: fp32 32003 x 1001 to planes 58 us, 5.5 TB/s.
template <bool BF16, int PLANES>
__global__ __launch_bounds__(256)
void k_loss_blocks(const void *weight, uint8_t *blocks, uint32_t rows, uint32_t cols, uint32_t padded)
{
    constexpr uint32_t ES = BF16 ? 2 : 4, WHOLE = kStageCols<BF16 || PLANES == 3>, RUNS = WHOLE / 8;
    constexpr uint32_t TOGETHER = 256 / (16 * RUNS);
    const uint32_t row = blockIdx.x * 16 + threadIdx.x / RUNS % 16, count = (cols + WHOLE - 1) / WHOLE;
    if (row >= padded) return;
    for (uint32_t c = (blockIdx.y * TOGETHER + threadIdx.x / (16 * RUNS)) * WHOLE + threadIdx.x % RUNS * 8; c < count * WHOLE; c += gridDim.y * TOGETHER * WHOLE) {
        Eight<BF16> e = {};
        if (row < rows && c < cols)
            e = fetch<BF16, false>(static_cast<const uint8_t *>(weight) + (uint64_t)row * cols * ES, c, cols, more_behind(row, rows, cols));
        put_eight<BF16, PLANES>(e, blocks, (uint64_t)count * padded * 64, ((uint64_t)(c / WHOLE) * padded + row) * 64 + c % WHOLE * (64 / WHOLE));
    }
}

// ---------------------------------------------------------------- tiles

struct LogitArgs {
    const uint8_t *x, *weight;               // gathered hidden states, the piece's first row
    uint64_t ldw;                            // bytes from row to row, or from block to block
    uint64_t x_plane, w_plane, g_plane;      // bytes from plane to plane
    LossTokens tokens;
    uint32_t stages, first, vocab;           // of columns; the piece's first row of the vocabulary, and rows of the vocabulary up to the piece's end
    uint32_t tiles_n;
    float2 *parts;                           // forward: (largest logit, sum of exp(l - it)), [part][padded tokens]
    float *at_target;                        // logits of the targets
    uint32_t padded;
    const float *lse, *grad_loss;            // backward; grad_loss: of every token, or NULL
    uint8_t *grads;                          // p - [v = t] of the piece, in blocks
};

enum { kStats = 0, kGrads = 1 };

// exp(l - top) as 2^(l log2(e) + shift), one fused multiply-add, with shift = -top log2(e), whose rounding, 2^-24 of it, is in the exponent.  Where a shift
// is larger than kFar (logits of thousands; nothing but masks, -1e30, whose rounding is more than any exponent, or the lowest number, whose shift is
// infinite) as 2^((l - top) log2(e)).
constexpr float kLog2e = 1.4426950408889634f, kFar = 4096.0f;

__device__ __forceinline__ float2 joined(float2 a, float2 b)
{
    const float top = fmaxf(a.x, b.x), shift = top == -INFINITY ? 0.0f : top;
    return make_float2(top, a.y * __expf(a.x - shift) + b.y * __expf(b.x - shift));
}
// A wavefront's part of the statistics of its logits, of tokens from m0 and rows of the vocabulary from n0 on, up to `vocab` of them.  Columns behind the
// vocabulary are asked for in the tiles that have them alone, targets in the 32 tokens that have one here.  `more`: joined to what is
// there.
template <class T, class Target>
__device__ __forceinline__ void leave_stats(const TileResult<T> &r, uint32_t m0, uint32_t n0, uint32_t vocab, uint32_t count, Target target_of, float *at_target, float2 *parts,
                                            bool more = false)
{
    constexpr int MF = T::MF, NF = T::NF;
    uint32_t lane = threadIdx.x % 64;
    asm volatile("" : "+v"(lane));                           // what follows from it is not kept in registers all along
    const uint32_t half = lane / 32;
    auto column = [&](int j, int k) { return n0 + 32 * j + 8 * (k / 4) + 4 * half + k % 4; };
    auto stats = [&](auto edge) {
#pragma unroll
        for (int i = 0; i < MF; ++i) {
            __builtin_amdgcn_sched_barrier(0);
            uint32_t m = m0 + 32 * i + lane % 32;
            asm volatile("" : "+v"(m));
            const uint32_t target = m < count ? target_of(m) : kBadTarget;
            float l[NF][16], top = -INFINITY;
#pragma unroll
            for (int j = 0; j < NF; ++j)
#pragma unroll
                for (int k = 0; k < 16; ++k) {
                    l[j][k] = !decltype(edge)::value || column(j, k) < vocab ? r.acc[i][j][k] : -INFINITY;
                    top = fmaxf(top, l[j][k]);
                }
            if (target - n0 < (uint32_t)NF * 32) {
#pragma unroll
                for (int j = 0; j < NF; ++j)
#pragma unroll
                    for (int k = 0; k < 16; ++k)
                        if (column(j, k) == target) at_target[m] = l[j][k];
            }
            top = fmaxf(top, __shfl_xor(top, 32));
            const float shift = top == -INFINITY ? 0.0f : -top * kLog2e;             // a part without a logit above -infinity: its sum is 0
            float sum[4] = {};
            if (__ballot(__builtin_fabsf(shift) > kFar)) {
                const float from = top == -INFINITY ? 0.0f : top;
#pragma unroll
                for (int j = 0; j < NF; ++j)
#pragma unroll
                    for (int k = 0; k < 16; ++k) sum[k % 4] += __builtin_amdgcn_exp2f((l[j][k] - from) * kLog2e);
            } else {
#pragma unroll
                for (int j = 0; j < NF; ++j)
#pragma unroll
                    for (int k = 0; k < 16; ++k) sum[k % 4] += __builtin_amdgcn_exp2f(__builtin_fmaf(l[j][k], kLog2e, shift));
            }
            float all = (sum[0] + sum[1]) + (sum[2] + sum[3]);
            all += __shfl_xor(all, 32);
            if (half == 0 && m < count) parts[m] = more ? joined(parts[m], make_float2(top, all)) : make_float2(top, all);
        }
    };
    if (n0 + NF * 32 > vocab) stats(std::true_type{});
    else stats(std::false_type{});
}

// A wavefront's part of p - [v = t] of the piece, from its logits of tokens from m0 and rows of the vocabulary from n0 on.  Of bf16 tensors it is rounded to
// bf16, up to 2^-8 of it: a matrix instruction's operands are both of one type, and a second plane of bf16 would double two of the pass's products (8192 x
// 4096 x 131072 27 to about 40 ms in all).  Gradients are off by 1.85e-3 of their norm, of which rounding the results makes 1.66e-3 alone (2048 x 1600 x
// 50257, hidden states' and weight's; 8192 x 4096 x 131072 1.83e-3 of 1.66e-3, and 1.53e-3 of 1.34e-3).  fp32 is in three planes, or as it is.
template <bool BF16, int PLANES, class T>
__device__ __forceinline__ void leave_gradients(const TileResult<T> &r, uint32_t m0, uint32_t n0, uint32_t count, const LogitArgs &g)
{
    constexpr int MF = T::MF, NF = T::NF;
    uint32_t lane = threadIdx.x % 64;
    asm volatile("" : "+v"(lane));                           // what follows from it is not kept in registers all along
    const uint32_t half = lane / 32;
    auto column = [&](int j, int k) { return n0 + 32 * j + 8 * (k / 4) + 4 * half + k % 4; };
    constexpr uint32_t WHOLE = kStageCols<BF16>;
    const uint32_t end = (max(count, 1u) + WHOLE - 1) / WHOLE * WHOLE;   // rows that are summed over: zeros behind the last token
    auto gradients = [&](auto edge) {
#pragma unroll
        for (int i = 0; i < MF; ++i) {
            uint32_t m = m0 + 32 * i + lane % 32;
            asm volatile("" : "+v"(m));
            const bool there = m < count;
            const uint32_t row = there ? g.tokens.rows[m] : 0, target = there ? g.tokens.targets[m] : kBadTarget;
            const float lse = there ? g.lse[row] : 0.0f, shift = -lse * kLog2e;
            const bool far = __ballot(__builtin_fabsf(shift) > kFar) != 0;
            float factor = there && g.grad_loss ? g.grad_loss[row] : 1.0f;
            if (there && target == kBadTarget) factor = NAN;
            const bool here = target - n0 < (uint32_t)NF * 32, any = __ballot(here) != 0, behind = __ballot(!there) != 0;
#pragma unroll
            for (int j = 0; j < NF; ++j) {
                __builtin_amdgcn_sched_barrier(0);
                float d[16];
#pragma unroll
                for (int k = 0; k < 16; ++k) {
                    d[k] = __builtin_amdgcn_exp2f(__builtin_fmaf(r.acc[i][j][k], kLog2e, shift));
                    if (decltype(edge)::value && column(j, k) >= g.vocab) d[k] = 0.0f;
                }
                if (far) {
#pragma unroll
                    for (int k = 0; k < 16; ++k) {
                        d[k] = __builtin_amdgcn_exp2f((r.acc[i][j][k] - lse) * kLog2e);
                        if (decltype(edge)::value && column(j, k) >= g.vocab) d[k] = 0.0f;
                    }
                }
                if (any) {
#pragma unroll
                    for (int k = 0; k < 16; ++k)
                        if (column(j, k) == target) d[k] -= 1.0f;
                }
#pragma unroll
                for (int k = 0; k < 16; ++k) d[k] *= factor;
                if (behind) {                            // the last token; these rows' logits may be NaN, as products of zeros and infinite weights
#pragma unroll
                    for (int k = 0; k < 16; ++k) d[k] = there ? d[k] : 0.0f;
                }
                // of the vocabulary's last block all columns: zeros behind its end
                const uint32_t n = n0 - g.first + 32 * j;                // in the piece
                if constexpr (BF16) {
                    uint8_t *to = g.grads + ((uint64_t)(n / 32) * g.padded + m) * 64 + half * 16;
#pragma unroll
                    for (int plane = 0; plane < PLANES; ++plane) {
                        uint2 w[4];
#pragma unroll
                        for (int q = 0; q < 4; ++q) w[q] = four_bf16(d, 4 * q);
                        if (plane + 1 < PLANES) {                        // what is left for the next one
#pragma unroll
                            for (int k = 0; k < 16; ++k) {
                                const uint32_t two = k % 4 < 2 ? w[k / 4].x : w[k / 4].y;
                                d[k] -= __uint_as_float(k % 2 ? two & 0xffff0000u : two << 16);
                            }
                        }
                        const uint4 w0 = eight_of(w[0], w[1]), w1 = eight_of(w[2], w[3]);
                        if (m < end && g.first + n < g.vocab) {
                            *reinterpret_cast<uint4 *>(to + plane * g.g_plane) = w0;
                            *reinterpret_cast<uint4 *>(to + plane * g.g_plane + 32) = w1;
                        }
                    }
                } else {
#pragma unroll
                    for (int b = 0; b < 2; ++b) {
                        uint8_t *to = g.grads + ((uint64_t)(n / 16 + b) * g.padded + m) * 64 + half * 16;
                        if (m < end && g.first + n + 16 * b < g.vocab) {
                            *reinterpret_cast<float4 *>(to) = make_float4(d[8 * b], d[8 * b + 1], d[8 * b + 2], d[8 * b + 3]);
                            *reinterpret_cast<float4 *>(to + 32) = make_float4(d[8 * b + 4], d[8 * b + 5], d[8 * b + 6], d[8 * b + 7]);
                        }
                    }
                }
            }
        }
    };
    if (n0 + NF * 32 > g.vocab) gradients(std::true_type{});
    else gradients(std::false_type{});
}

// LIES: how the weight does
template <bool BF16, int PLANES, int WM, int WN, int MF, int NF, int PER_CU, Lies LIES, int MODE>
__global__ __launch_bounds__(256, PER_CU)
void k_loss_logits(LogitArgs g)
{
    using T = TileKind<BF16, WM, WN, MF, NF>;
    const Stages stages = stages_of<T, LIES>();
    const uint32_t count = *g.tokens.count, tiles_m = (max(count, 1u) + T::UM * 32 - 1) / (T::UM * 32);
    if (blockIdx.x >= (uint64_t)tiles_m * g.tiles_n) return;
    uint32_t tm, tn;
    tile_of(blockIdx.x, tiles_m, g.tiles_n, tm, tn);
    TileResult<T> r;
    const Operand a = {g.x, (uint64_t)g.padded * 64, g.padded, 0, g.x_plane}, b = {g.weight, g.ldw, g.vocab - g.first, 0, g.w_plane};
    multiply_tile<T, BF16, PLANES, kBlocks, LIES>(a, b, tm, tn, 0, g.stages, stages, r);
    const uint32_t wave = uniform(threadIdx.x / 64), m0 = tm * T::UM * 32 + r.m0, n0 = g.first + tn * T::UN * 32 + r.n0;         // n0: in the vocabulary
    auto leave = [&](const auto &results, uint32_t m, uint32_t n, bool more) {
        if constexpr (MODE == kStats)
            leave_stats(results, m, n, g.vocab, count, [&](uint32_t token) { return g.tokens.targets[token]; }, g.at_target, g.parts + (uint64_t)(tn * WN + wave % WN) * g.padded, more);
        else
            leave_gradients<BF16, PLANES>(results, m, n, count, g);
    };
    if constexpr (PLANES == 3) {
        if (any_nan(r, m0, count)) {                         // an infinite operand, or a NaN: a unit after the other
            for (uint32_t unit = 0; unit < MF * NF; ++unit) {
                const uint32_t m = m0 + unit / NF * 32, n = n0 + unit % NF * 32;
                TileResult<OneUnit> one;
                one.acc[0][0] = as_fp32(a, b, m, n - g.first, g.stages);
                leave(one, m, n, unit % NF != 0);
            }
            return;
        }
    }
    leave(r, m0, n0, false);
}

// Up to 32 tokens forward, with rows of no whole stages or few rows of the vocabulary (then WAVES wavefronts to the channels), from where they lie: the
// weight goes straight to registers, a wavefront 32 rows of the vocabulary and 256 bytes of each at a time, the next 256 on their way.  Which columns a
// product's operands hold does not matter as long as both hold the same: a lane has 128 bytes of a row, or the other 128. Bound by addresses, a line for
// each lane: bf16 21 x 7999 x 50257 282 us, 2.9 TB/s, by way of a copy 605; 32 x 1001 x 131071 116 and 181; fp32 20 x 3001 x 32000 123 and 325.  Rows of
// whole stages are faster through LDS, four lanes to a line of them (11 x 2560 x 131072 137 us, straight to registers 158).
struct FewArgs {
    const void *x, *weight;                  // the piece's first row
    const int64_t *target;
    int64_t ignore;
    uint32_t rows, cols, first, end, vocab;  // the piece's rows of the vocabulary
    uint32_t padded;
    LossTokens tokens;                       // written, as by k_loss_gather
    float2 *parts;
    float *at_target, *zero, *zero_also;     // results of tokens that do not count
};
constexpr int kFewWaves = 8;
template <bool BF16, int WAVES>
__global__ __launch_bounds__(64 * WAVES)
void k_loss_few(FewArgs g)
{
    using T = TileKind<BF16, 1, 4, 1, 1>;
    constexpr uint32_t ES = BF16 ? 2 : 4, EACH = 16 / ES, RUN = 8;
    __shared__ uint32_t places[32];
    const uint32_t lane = threadIdx.x % 64, wave = uniform(threadIdx.x / 64), half = lane / 32, n = lane % 32, n0 = g.first + blockIdx.x * 32;
    const int64_t t = n < g.rows ? g.target[n] : g.ignore;
    const uint8_t *const w = static_cast<const uint8_t *>(g.weight) + (uint64_t)(min(n0 + n, g.end - 1) - g.first) * g.cols * ES;
    // bf16 lie at any even address: words from the one before on, shifted by half a word.  At least one number is left behind the last run, so they stay
    // within the row.
    uint4 a[2][RUN], b[2][RUN];
    uint32_t a_end[2] = {}, b_end[2] = {};
    const uint32_t runs = (g.cols - 1) / (2 * RUN * EACH);
    auto ask = [&](uint4 (&to)[RUN], uint32_t &end, const uint8_t *row, uint32_t run) {
        const uint8_t *from = row + (uint64_t)run * RUN * 32 + half * RUN * 16;
        const uint32_t off = BF16 ? (uint32_t)reinterpret_cast<uintptr_t>(from) & 2 : 0;
        from -= off;
#pragma unroll
        for (uint32_t k = 0; k < RUN; ++k) __builtin_memcpy(&to[k], __builtin_assume_aligned(from + k * 16, 4), 16);
        if (BF16 && off) __builtin_memcpy(&end, __builtin_assume_aligned(from + RUN * 16, 4), 4);
    };
    // what was asked for, as the products take it
    auto shifted = [&](const uint4 (&v)[RUN], uint32_t end, uint32_t k, const uint8_t *row) {
        if constexpr (!BF16) return v[k];
        const uint32_t by = ((uint32_t)reinterpret_cast<uintptr_t>(row) & 2) * 8, next = k + 1 < RUN ? v[(k + 1) % RUN].x : end;
        return make_uint4(__builtin_amdgcn_alignbit(v[k].y, v[k].x, by), __builtin_amdgcn_alignbit(v[k].z, v[k].y, by), __builtin_amdgcn_alignbit(v[k].w, v[k].z, by),
                          __builtin_amdgcn_alignbit(next, v[k].w, by));
    };
    if (wave < runs) ask(b[0], b_end[0], w, wave);
    const uint32_t counted = (uint32_t)__ballot(t != g.ignore), count = __popc(counted), rank = __popc(counted & ((1u << n) - 1));
    if (threadIdx.x < 32) places[n] = 0;
    __syncthreads();
    if (threadIdx.x < 32 && (counted >> n & 1)) places[rank] = n;
    __syncthreads();
    const uint32_t row = places[n];          // of the n-th token that counts; behind the last one any, whose results nobody takes
    const uint32_t mine = (uint32_t)__shfl((int)(t >= 0 && t < (int64_t)g.vocab ? (uint32_t)t : kBadTarget), (int)row);
    const uint8_t *const x = static_cast<const uint8_t *>(g.x) + (uint64_t)row * g.cols * ES;
    TileResult<T> r;
    r.m0 = r.n0 = 0;
    if (wave < runs) ask(a[0], a_end[0], x, wave);
    float16v sums_of[BF16 ? 1 : 4] = {};     // four of fp32, as sums of thousands of columns one after another would be off by more
    for (uint32_t i = wave; i < runs; i += 2 * WAVES) {
#pragma unroll
        for (uint32_t k = 0; k < 2; ++k)
            if (i + k * WAVES < runs) {
                const uint32_t next = min(i + (k + 1) * WAVES, runs - 1);    // behind the last run that one again
                ask(b[1 - k], b_end[1 - k], w, next);
                ask(a[1 - k], a_end[1 - k], x, next);
                __builtin_amdgcn_sched_barrier(0);           // not after the products
#pragma unroll
                for (uint32_t j = 0; j < RUN; ++j) sums_of[BF16 ? 0 : j % 4] = multiply32<BF16>(shifted(b[k], b_end[k], j, w), shifted(a[k], a_end[k], j, x), sums_of[BF16 ? 0 : j % 4]);
            }
    }
    // what is left of the rows, and zeros behind their end
    if (wave == 0) {
        const uint32_t from = runs * 2 * RUN * EACH;
        auto rest = [&](uint4 (&to)[RUN], const uint8_t *of) {
#pragma unroll
            for (uint32_t k = 0; k < RUN; ++k) {
                const uint32_t c = from + (2 * k + half) * EACH;
                uint32_t v[4] = {};
                if (c + EACH <= g.cols) {
                    __builtin_memcpy(v, of + (uint64_t)c * ES, 16);
                } else {
#pragma unroll
                    for (uint32_t e = 0; e < EACH; ++e)
                        if (c + e < g.cols) {
                            if constexpr (BF16) v[e / 2] |= (uint32_t)reinterpret_cast<const uint16_t *>(of)[c + e] << e % 2 * 16;
                            else v[e] = reinterpret_cast<const uint32_t *>(of)[c + e];
                        }
                }
                to[k] = make_uint4(v[0], v[1], v[2], v[3]);
            }
        };
        rest(b[0], w);
        rest(a[0], x);
#pragma unroll
        for (uint32_t j = 0; j < RUN; ++j) sums_of[BF16 ? 0 : j % 4] = multiply32<BF16>(b[0][j], a[0][j], sums_of[BF16 ? 0 : j % 4]);
    }
    r.acc[0][0] = sums_of[0];
    if constexpr (!BF16) r.acc[0][0] = (sums_of[0] + sums_of[1]) + (sums_of[2] + sums_of[3]);
    if constexpr (WAVES > 1) {
        __shared__ float sums[WAVES - 1][16][64];
        if (wave) {
#pragma unroll
            for (int k = 0; k < 16; ++k) sums[wave - 1][k][lane] = r.acc[0][0][k];
        }
        __syncthreads();
        if (wave) return;
#pragma unroll
        for (int v = 0; v < WAVES - 1; ++v)
#pragma unroll
            for (int k = 0; k < 16; ++k) r.acc[0][0][k] += sums[v][k][lane];
    }
    leave_stats(r, 0, n0, g.end, count, [&](uint32_t) { return mine; }, g.at_target, g.parts + (uint64_t)blockIdx.x * g.padded);
    if (blockIdx.x == 0 && half == 0) {
        if (n < count) {
            g.tokens.rows[n] = row;
            g.tokens.targets[n] = mine;
        }
        if (n < g.rows && !(counted >> n & 1)) g.zero[n] = g.zero_also[n] = 0.0f;
        if (n == 0) *g.tokens.count = count;
    }
}

// The gradient that the reduced loss came back with, over the number of tokens if it is their mean; without a token 0, whatever it is
__device__ __forceinline__ float loss_scale(const float *grad_loss, uint32_t mean, uint32_t count)
{
    if (count == 0) return 0.0f;
    const float g = grad_loss ? *grad_loss : 1.0f;
    return mean ? g / (float)count : g;
}

// Sums over the vocabulary's piece, in parts; `add`: to what earlier pieces left.  They stay in the order that the lanes have them in, [part][tile]
// [wavefront][i][j][group of four][lane] of four numbers: 1 KB in a row.
struct GradXArgs {
    const uint8_t *grads, *weight;
    uint64_t ldw, g_plane, w_plane;
    LossTokens tokens;
    uint32_t rows, cols, stages, first_stages, slots, tiles_n, padded, add;
    float4 *sums;
};
template <bool BF16, int PLANES, int WM, int WN, int MF, int NF, int PER_CU, Lies LIES>
__global__ __launch_bounds__(256, PER_CU)
void k_loss_grad_x(GradXArgs g)
{
    using T = TileKind<BF16, WM, WN, MF, NF>;
    const Stages stages = stages_of<T, LIES>();
    const uint32_t count = *g.tokens.count, tiles_m = (count + T::UM * 32 - 1) / (T::UM * 32);
    const Shares shares(tiles_m * g.tiles_n, g.first_stages, g.stages, g.slots);
    const uint32_t all = shares.tiles * shares.parts;
    if (blockIdx.x >= all) return;
    const uint32_t id = by_die(blockIdx.x, all), part = id / shares.tiles;      // a die has as few parts, which share their operands, as there are
    uint32_t tm, tn;
    tile_at(id % shares.tiles, tiles_m, g.tiles_n, tm, tn);
    TileResult<T> r;
    const Operand a = {g.grads, (uint64_t)g.padded * 64, g.padded, 0, g.g_plane}, b = {g.weight, g.ldw, g.rows, (g.cols + T::COLS - 1) / T::COLS, g.w_plane};
    const uint32_t from = part * shares.run, count_stages = min(shares.run, g.stages - from);
    auto run = [&](uint32_t begin, uint32_t columns, bool add) {
        multiply_tile<T, BF16, PLANES, kBlocks, LIES>(a, b, tm, tn, begin, columns, stages, r);
        uint32_t lane = threadIdx.x % 64;
        asm volatile("" : "+v"(lane));                       // not an address to keep in registers all along
        float4 *to = g.sums + (((uint64_t)part * shares.tiles + (uint64_t)tm * g.tiles_n + tn) * 4 + uniform(threadIdx.x / 64)) * (MF * NF * 256) + lane;
#pragma unroll
        for (int i = 0; i < MF; ++i)
#pragma unroll
            for (int j = 0; j < NF; ++j) {
                __builtin_amdgcn_sched_barrier(0);
                asm volatile("" : "+v"(to));                 // one by one: addresses of all of them would not fit the registers
                float4 x[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) x[k] = add ? to[((i * NF + j) * 4 + k) * 64] : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const float16v &v = r.acc[i][j];
                    to[((i * NF + j) * 4 + k) * 64] = make_float4(x[k].x + v[4 * k], x[k].y + v[4 * k + 1], x[k].z + v[4 * k + 2], x[k].w + v[4 * k + 3]);
                }
            }
    };
    if constexpr (T::template runs<PLANES>())
        for (uint32_t done = 0; done < count_stages; done += kPlanesChain) run(from + done, min(kPlanesChain, count_stages - done), done || g.add);
    else
        run(from, count_stages, g.add != 0);
}

// Up to four neighbours
template <bool BF16>
__device__ __forceinline__ void store_four(void *to, uint64_t at, uint32_t valid, const float (&v)[4])
{
    if (valid >= 4) {
        if constexpr (BF16) {
            const uint2 w = four_bf16(v, 0);
            __builtin_memcpy(static_cast<uint16_t *>(to) + at, &w, 8);
        } else {
            __builtin_memcpy(static_cast<float *>(to) + at, v, 16);
        }
    } else {
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i)
            if (i < valid) store1<BF16>(to, at + i, v[i]);
    }
}

// The hidden states' gradient from its sums, to the tokens' own rows.  How the sums lie: tiles of tm x tn, wavefronts of wm x wn in them.  A wavefront
// takes eight tokens, whose numbers lie side by side, and 32 columns at a time; workgroups have up to eight runs of 128 columns one after another (2048 x
// 1600 of six parts: 20 us; a workgroup to each run, parts one by one, 77).
struct SumsLayout {
    uint32_t tm, tn, wm, wn;
};
// stages: of the first piece
template <bool BF16>
__global__ __launch_bounds__(256)
void k_loss_scatter(const float4 *sums, uint32_t stages, uint32_t slots, uint32_t tiles_n, SumsLayout s, LossTokens tokens, uint32_t cols, const float *grad_loss, uint32_t mean,
                    void *grad_x)
{
    const uint32_t lane = threadIdx.x % 64, wave = uniform(threadIdx.x / 64), count = *tokens.count, r = blockIdx.x * 8 + lane % 8;
    if (blockIdx.x * 8 >= count) return;
    const Shares shares((count + s.tm - 1) / s.tm * tiles_n, stages, stages, slots);
    const float scale = loss_scale(grad_loss, mean, count);
    const bool there = r < count;
    const uint64_t row = there ? (uint64_t)tokens.rows[r] * cols : 0;
    const uint32_t m = r % s.tm, units = s.wn / 32, piece = s.wm * s.wn / 4;              // piece: of a wavefront, in fours
    for (uint32_t c = blockIdx.y * 128 + wave * 32 + lane / 8 * 4; c < cols; c += gridDim.y * 128) {
        const uint32_t n = c % s.tn, w = m / s.wm * (s.tn / s.wn) + n / s.wn, unit = m % s.wm / 32 * units + n % s.wn / 32;
        const float4 *from = sums + ((uint64_t)(r / s.tm) * tiles_n + c / s.tn) * 4 * piece + w * piece + (unit * 4 + n % 32 / 8) * 64 + n % 8 / 4 * 32 + m % 32;
        float v[4] = {};
        if (there)
            for (uint32_t p = 0; p < shares.parts; p += 8) {
                float4 x[8];
#pragma unroll
                for (uint32_t k = 0; k < 8; ++k) x[k] = p + k < shares.parts ? from[(uint64_t)(p + k) * shares.tiles * 4 * piece] : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
                for (uint32_t k = 0; k < 8; ++k) {
                    v[0] += x[k].x;
                    v[1] += x[k].y;
                    v[2] += x[k].z;
                    v[3] += x[k].w;
                }
            }
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] *= scale;
        if (there) store_four<BF16>(grad_x, row + c, cols - c, v);
    }
}

struct GradWArgs {
    const uint8_t *grads, *x;
    uint64_t g_plane, x_plane;
    LossTokens tokens;
    uint32_t rows, cols, tiles_m, tiles_n, padded;           // rows of the piece
    const float *grad_loss;                  // of the reduced loss, or NULL
    uint32_t mean, out_bf16, accumulate;
    void *out;                               // the gradient's first row of the piece
};
template <bool BF16, int PLANES, int WM, int WN, int MF, int NF, int PER_CU>
__global__ __launch_bounds__(256, PER_CU)
void k_loss_grad_w(GradWArgs g)
{
    using T = TileKind<BF16, WM, WN, MF, NF>;
    const Stages stages = stages_of<T, kBlocksTurned>();
    const uint32_t count = *g.tokens.count, depth = (max(count, 1u) + T::COLS - 1) / T::COLS;
    uint32_t tm, tn;
    tile_of(blockIdx.x, g.tiles_m, g.tiles_n, tm, tn);
    TileResult<T> r;
    const Operand a = {g.grads, (uint64_t)g.padded * 64, g.padded, (g.rows + T::COLS - 1) / T::COLS, g.g_plane},
                  b = {g.x, (uint64_t)g.padded * 64, g.padded, (g.cols + T::COLS - 1) / T::COLS, g.x_plane};
    const float scale = loss_scale(g.grad_loss, g.mean, count);
    auto run = [&](uint32_t begin, uint32_t columns, bool add) {
        multiply_tile<T, BF16, PLANES, kBlocksTurned, kBlocksTurned>(a, b, tm, tn, begin, columns, stages, r);
        const uint32_t m0 = tm * T::UM * 32 + r.m0, n0 = tn * T::UN * 32 + r.n0;
        if (g.out_bf16) store_rows<true, T>(r, m0, n0, g.rows, g.cols, scale, g.out, add);
        else store_rows<false, T>(r, m0, n0, g.rows, g.cols, scale, g.out, add);
    };
    if constexpr (T::template runs<PLANES>())               // bf16: a single run
        for (uint32_t done = 0; done < depth; done += kPlanesChain) run(done, min(kPlanesChain, depth - done), done || g.accumulate);
    else
        run(0, depth, g.accumulate != 0);
}

// ---------------------------------------------------------------- joining

// The parts of some tokens' statistics, and at the end of the vocabulary (`last`) lse and losses; `later`: with what earlier pieces left in `running`.
// A workgroup takes `width` tokens, a power of two up to 32, and the parts in kJoinLanes / width runs, four at a time.
constexpr uint32_t kJoinLanes = 1024;

// Sum over a workgroup of kJoinLanes, in every lane
__device__ __forceinline__ float lanes_sum(float v, float *sums)
{
    v = wave_sum(v);
    if (threadIdx.x % 64 == 0) sums[threadIdx.x / 64] = v;
    __syncthreads();
    v = sums[threadIdx.x % 16];
    static_assert(kJoinLanes == 16 * 64, "a row of sixteen lanes adds the wavefronts' sums");
    v = add_permuted<0xb1>(v);
    v = add_permuted<0x4e>(v);
    v = add_permuted<0x141>(v);
    return add_permuted<0x140>(v);
}

__global__ __launch_bounds__(kJoinLanes)
void k_loss_join(const float2 *from, uint32_t parts, uint32_t padded, LossTokens tokens, const float *at_target, float2 *running, uint32_t later,
                 uint32_t last, uint32_t width, float *losses, float *lse, uint32_t mean, float *total)
{
    __shared__ float2 places[kJoinLanes];
    const uint32_t lane = threadIdx.x % width, run = threadIdx.x / width, runs = kJoinLanes / width, count = *tokens.count, r = blockIdx.x * width + lane;
    float2 v = make_float2(-INFINITY, 0.0f);
    if (r < count)
        for (uint32_t p = run; p < parts; p += 4 * runs) {
            // behind the last part the first of the four again, which then does not count
            const float2 *const at = from + (uint64_t)p * padded + r;
            const uint64_t step = (uint64_t)runs * padded;
            float2 w0 = *at, w1 = at[p + runs < parts ? step : 0], w2 = at[p + 2 * runs < parts ? 2 * step : 0], w3 = at[p + 3 * runs < parts ? 3 * step : 0];
            if (p + runs >= parts) w1.x = -INFINITY, w1.y = 0.0f;
            if (p + 2 * runs >= parts) w2.x = -INFINITY, w2.y = 0.0f;
            if (p + 3 * runs >= parts) w3.x = -INFINITY, w3.y = 0.0f;
            v = joined(v, joined(joined(w0, w1), joined(w2, w3)));
        }
    places[threadIdx.x] = v;
    __syncthreads();
    for (uint32_t half = kJoinLanes / 2; half >= width; half /= 2) {
        if (threadIdx.x < half) places[threadIdx.x] = joined(places[threadIdx.x], places[threadIdx.x + half]);
        __syncthreads();
    }
    float loss = 0.0f;
    if (run == 0 && r < count) {
        v = places[lane];
        if (later) v = joined(running[r], v);
        if (last) {
            const float all = v.x + logf(v.y);
            const uint32_t row = tokens.rows[r];
            loss = tokens.targets[r] == kBadTarget ? NAN : all - at_target[r];
            lse[row] = all;
            losses[row] = loss;
        } else {
            running[r] = v;
        }
    }
    if (!total) return;
    // the only workgroup: the reduced loss, too
    __syncthreads();
    const float sum = lanes_sum(loss, reinterpret_cast<float *>(places));
    if (threadIdx.x == 0) {
        total[0] = mean ? sum / (float)max(count, 1u) : sum;
        total[1] = (float)count;
    }
}

// The reduced loss and the number of tokens that count
__global__ __launch_bounds__(kJoinLanes)
void k_loss_total(const float *losses, uint32_t rows, LossTokens tokens, uint32_t mean, float *total)
{
    __shared__ float sums[kJoinLanes / 64];
    const uint32_t count = *tokens.count;
    float sum = 0.0f;
    for (uint32_t i = threadIdx.x; i < rows; i += 8 * kJoinLanes) {
        float v[8];
#pragma unroll
        for (uint32_t k = 0; k < 8; ++k) v[k] = i + k * kJoinLanes < rows ? losses[i + k * kJoinLanes] : 0.0f;
        sum += ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
    }
    sum = lanes_sum(sum, sums);
    if (threadIdx.x == 0) {
        total[0] = mean ? sum / (float)max(count, 1u) : sum;
        total[1] = (float)count;
    }
}

}  // namespace tahq
