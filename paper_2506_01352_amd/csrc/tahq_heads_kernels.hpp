// Heads of queries and keys, normed and rotated (include/tahq_heads.h), forward and backward.
//
// Bound by memory: forward two tensors, backward three, each once.  A wavefront takes a token at a time and several of its heads side by side, a group of
// `lanes` lanes to a head, or several tokens where they have few heads.  A lane holds both channels of each of its pairs, so that rotations stay within it,
// and the same channels of every head, so that it works out its angles once for a token. bf16 32768 x (40 + 8) x 128: forward 151 us, 5.3 TB/s; backward
// 243 and 5, 5.0 TB/s.  One token: 3.4 us, a launch and its loads one after another.  fp32 777 x 50 x 64 forward 7.2 us, 2331 x 25 x 80 backward 14.2 and
// 3.8: 40 and 56 MB, a launch's start and two rounds of memory's latency, positions before angles, in it. Numbers one by one, for halves of odd size, take
// three times the bytes' time (bf16 7432 x 40 x 58 backward 65 us).
#pragma once
#include "tahq_heads.h"
#include "tahq_lanes.hpp"
#include "tahq_mx4_common.hpp"

namespace tahq {

struct HeadShape {
    uint32_t tokens, heads[2], head, rotated, lanes, split;     // heads: of queries, of keys; split: a token's heads go to as many wavefronts as there are for
    uint64_t ld[2], ld_out[2];
    float eps, magnitude;
};
struct HeadTensors {                         // queries', keys'
    const void *of[2];
};
struct HeadOutputs {
    void *of[2];
};
constexpr uint32_t kHeadWaves = 4;           // of a workgroup

// cos and sin of a fraction of a turn in units of 2^-32.  The nearest quarter turn is taken off, exactly; what is left, up to pi/4, goes into
// the sums' first terms: the next ones are below 2^-28 of the result.
__device__ __forceinline__ void cos_sin(uint32_t turn, float &c, float &s)
{
    const uint32_t quarter = (turn + 0x20000000u) >> 30;
    const float t = (float)(int)(turn - (quarter << 30)) * 1.4629180792671596e-09f;       // 2 pi / 2^32
    const float x = t * t;
    const float sine = __builtin_fmaf(t * x, __builtin_fmaf(x, __builtin_fmaf(x, __builtin_fmaf(x, 2.7557319e-6f, -1.9841270e-4f), 8.3333333e-3f), -1.6666667e-1f), t);
    const float cosine = __builtin_fmaf(x, __builtin_fmaf(x, __builtin_fmaf(x, __builtin_fmaf(x, __builtin_fmaf(x, -2.7557319e-7f, 2.4801587e-5f), -1.3888889e-3f), 4.1666667e-2f), -0.5f), 1.0f);
    const bool swapped = quarter & 1;
    c = swapped ? sine : cosine;
    s = swapped ? cosine : sine;
    c = (quarter + 1) & 2 ? -c : c;
    s = quarter & 2 ? -s : s;
}

// The channels that a lane holds of every head: E pairs.  CHUNK > 1: two chunks of so many channels, at channels `at[0]` and `at[1]`; otherwise pair by
// pair, whatever the sizes.
template <bool BF16, int CHUNK, bool PAIRS>
struct HeadLane {
    static constexpr bool WIDE = CHUNK > 1;
    static constexpr int E = WIDE ? CHUNK : 4, ES = BF16 ? 2 : 4, WORDS = CHUNK * ES / 4;
    uint32_t u, at[2];
    bool there[2];
    __device__ __forceinline__ HeadLane(const HeadShape &s) : u(threadIdx.x % s.lanes), at{0, 0}, there{false, false}
    {
        if constexpr (WIDE) {
            const uint32_t turned = PAIRS ? 0 : s.rotated / (2 * E);         // lanes of which both chunks are turned, against each other
            at[0] = u < turned ? u * E : (PAIRS ? 0 : s.rotated) + 2 * (u - turned) * E;
            at[1] = u < turned ? s.rotated / 2 + u * E : at[0] + E;
            there[0] = at[0] < s.head;
            there[1] = at[1] < s.head;
        }
    }
    // number of pair i among the pairs of a head; of WIDE halves, where it is turned
    __device__ __forceinline__ uint32_t pair(const HeadShape &s, int i) const
    {
        if constexpr (!WIDE) return u + s.lanes * i;
        else if constexpr (PAIRS) return at[i / (E / 2)] / 2 + i % (E / 2);
        else return u * E + i;
    }
    __device__ __forceinline__ bool turned(const HeadShape &s, int i) const { return 2 * pair(s, i) < s.rotated; }
    // channel of pair i's first (0) or second (1) number; may be behind the head's end
    __device__ __forceinline__ uint32_t channel(const HeadShape &s, int i, int which) const
    {
        if constexpr (WIDE) {
            if constexpr (PAIRS) return at[i / (E / 2)] + 2 * (i % (E / 2)) + which;
            else return at[which] + i;
        } else {
            const uint32_t p = pair(s, i);
            if (PAIRS || 2 * p >= s.rotated) return 2 * p + which;           // behind the rotated channels neighbours are together, too
            return p + which * (s.rotated / 2);
        }
    }
    // A head's channels as they lie in memory, and as numbers: pair i is a[i], b[i]; zeros for what there is not
    struct Raw {
        uint32_t q[2][WIDE ? WORDS : 1];
        float x[WIDE ? 1 : 2 * E];
    };
    __device__ __forceinline__ Raw load(const HeadShape &s, const void *base, uint64_t from, bool mine) const
    {
        Raw r = {};
        if constexpr (WIDE) {
            const uint8_t *p = static_cast<const uint8_t *>(base) + from * ES;
#pragma unroll
            for (int k = 0; k < 2; ++k)
                if (mine && there[k]) __builtin_memcpy(r.q[k], p + at[k] * ES, sizeof r.q[k]);
        } else {
#pragma unroll
            for (int i = 0; i < 2 * E; ++i) {
                const uint32_t c = channel(s, i / 2, i % 2);
                if (mine && c < s.head) r.x[i] = load1<BF16>(base, from + c);
            }
        }
        return r;
    }
    __device__ __forceinline__ void unpack(const Raw &r, float (&a)[E], float (&b)[E]) const
    {
        if constexpr (WIDE) {
            float x[2][E];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
#pragma unroll
                for (int i = 0; i < E; ++i) x[k][i] = __uint_as_float(!BF16 ? r.q[k][i % WORDS] : i % 2 ? r.q[k][i / 2] & 0xffff0000u : r.q[k][i / 2] << 16);
            }
#pragma unroll
            for (int i = 0; i < E; ++i) {
                a[i] = PAIRS ? x[i / (E / 2)][2 * (i % (E / 2))] : x[0][i];
                b[i] = PAIRS ? x[i / (E / 2)][2 * (i % (E / 2)) + 1] : x[1][i];
            }
        } else {
#pragma unroll
            for (int i = 0; i < E; ++i) {
                a[i] = r.x[2 * i];
                b[i] = r.x[2 * i + 1];
            }
        }
    }
    __device__ __forceinline__ void store(const HeadShape &s, void *base, uint64_t from, bool mine, const float (&a)[E], const float (&b)[E]) const
    {
        if constexpr (WIDE) {
            float x[2][E];
#pragma unroll
            for (int i = 0; i < E; ++i) {
                if constexpr (PAIRS) {
                    x[i / (E / 2)][2 * (i % (E / 2))] = a[i];
                    x[i / (E / 2)][2 * (i % (E / 2)) + 1] = b[i];
                } else {
                    x[0][i] = a[i];
                    x[1][i] = b[i];
                }
            }
            uint8_t *p = static_cast<uint8_t *>(base) + from * ES;
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                uint32_t w[WORDS];
#pragma unroll
                for (int i = 0; i < WORDS; ++i) w[i] = BF16 ? two_bf16(x[k][2 * i % E], x[k][(2 * i + 1) % E]) : __float_as_uint(x[k][i]);
                if (mine && there[k]) __builtin_memcpy(p + at[k] * ES, w, sizeof w);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 2 * E; ++i) {
                const uint32_t c = channel(s, i / 2, i % 2);
                if (mine && c < s.head) store1<BF16>(base, from + c, i % 2 ? b[i / 2] : a[i / 2]);
            }
        }
    }
    // of its pairs, 0 of those that are not turned
    __device__ __forceinline__ void ask_frequencies(const HeadShape &s, const uint64_t *frequencies, uint64_t (&f)[E]) const
    {
        // WIDE: runs of pairs are turned as a whole or not at all, and are asked for as a whole
        constexpr int RUN = !WIDE ? 1 : PAIRS ? E / 2 : E;
#pragma unroll
        for (int i = 0; i < E; i += RUN) {
#pragma unroll
            for (int k = 0; k < RUN; ++k) f[i + k] = 0;
            if (turned(s, i)) __builtin_memcpy(f + i, frequencies + pair(s, i), RUN * sizeof *f);
        }
    }
    __device__ __forceinline__ void angles(const HeadShape &s, uint64_t position, const uint64_t (&f)[E], float (&c)[E], float (&n)[E]) const
    {
#pragma unroll
        for (int i = 0; i < E; ++i) {
            cos_sin((uint32_t)((position * f[i] + 0x80000000u) >> 32), c[i], n[i]);
            c[i] = turned(s, i) ? c[i] * s.magnitude : 1.0f;
            n[i] = turned(s, i) ? n[i] * s.magnitude : 0.0f;
        }
    }
};

// Sum over the lanes of a head, a power of two of them, the same in each
__device__ __forceinline__ float head_sum(float v, uint32_t lanes)
{
    if (lanes > 1) v = add_permuted<0xb1>(v);
    if (lanes > 2) v = add_permuted<0x4e>(v);
    if (lanes > 4) v = add_permuted<0x141>(v);
    if (lanes > 8) v = add_permuted<0x140>(v);
    if (lanes > 16) v += __shfl_xor(v, 16);
    if (lanes > 32) v += __shfl_xor(v, 32);
    return v;
}

// A wavefront's way through tokens and groups of `heads` heads: every splits-th group of a token, then the token that all wavefronts are further.  Where
// a group has room for all heads of several tokens, it takes those; `at` is where the lane is, token and head.
struct HeadWay {
    uint32_t heads, tokens, groups, splits, split, step_split, each, mine, side;
    uint64_t first, step_first;              // of `side` tokens
    uint32_t group;
    __device__ __forceinline__ HeadWay(const HeadShape &s, uint32_t heads_, uint32_t waves, uint32_t wave) : heads(heads_), tokens(s.tokens)
    {
        each = 64 / s.lanes;
        groups = (heads + each - 1) / each;
        side = max(each / heads, 1u);
        splits = s.split ? groups : 1u;
        first = (uint64_t)(wave / splits) * side;
        group = split = wave % splits;
        step_first = (uint64_t)(waves / splits) * side;
        step_split = waves % splits;
        const uint32_t place = threadIdx.x % 64 / s.lanes, off = place / heads;
        // the token that it is further in a group of several, and its head; behind the last token of a group: no token at all
        mine = side > 1 ? place - off * heads : place;
        ahead = side == 1 ? 0 : off < side ? off : ~0u;
    }
    uint32_t ahead;
    __device__ __forceinline__ bool more() const { return first < tokens; }
    __device__ __forceinline__ uint64_t token() const { return first + ahead; }
    __device__ __forceinline__ uint32_t head() const { return group * each + mine; }
    __device__ __forceinline__ bool valid() const { return head() < heads && token() < tokens; }
    __device__ __forceinline__ uint64_t position(const int64_t *positions) const { return (uint64_t)positions[min(token(), (uint64_t)tokens - 1)]; }
    // to the next group; whether it is another token's
    __device__ __forceinline__ bool next()
    {
        group += splits;
        if (group < groups) return false;
        first += step_first;
        split += step_split;
        if (split >= splits) {
            split -= splits;
            first += side;
        }
        group = split;
        return true;
    }
};

// Queries and keys are one row of heads.
template <bool BF16, int CHUNK, bool PAIRS, bool NORM>
__global__ __launch_bounds__(64 * kHeadWaves)
void k_heads_forward(HeadTensors in, HeadTensors weights, const int64_t *positions, const uint64_t *frequencies, HeadOutputs out, HeadShape s)
{
    using Lane = HeadLane<BF16, CHUNK, PAIRS>;
    constexpr int E = Lane::E;
    const Lane lane(s);
    HeadWay way(s, s.heads[0] + s.heads[1], gridDim.x * kHeadWaves, blockIdx.x * kHeadWaves + uniform(threadIdx.x / 64));
    const float inv = 1.0f / (float)s.head;
    float c[E], n[E];
    bool another = true;
    while (way.more()) {
        const bool valid = way.valid(), key = way.head() >= s.heads[0];
        const uint32_t h = key ? way.head() - s.heads[0] : way.head();
        const typename Lane::Raw raw = lane.load(s, key ? in.of[1] : in.of[0], way.token() * (key ? s.ld[1] : s.ld[0]) + (uint64_t)h * s.head, valid);
        const uint64_t to = way.token() * (key ? s.ld_out[1] : s.ld_out[0]) + (uint64_t)h * s.head;
        if (another) {
            uint64_t f[E];
            lane.ask_frequencies(s, frequencies, f);
            lane.angles(s, s.rotated ? way.position(positions) : 0, f, c, n);
        }
        another = way.next();
        float a[E], b[E];
        lane.unpack(raw, a, b);
        if constexpr (NORM) {
            float wa[E], wb[E], sum = 0.0f;
            lane.unpack(lane.load(s, key ? weights.of[1] : weights.of[0], 0, valid), wa, wb);
#pragma unroll
            for (int i = 0; i < E; ++i) sum = __builtin_fmaf(b[i], b[i], __builtin_fmaf(a[i], a[i], sum));
            const float rstd = rsqrtf(head_sum(sum, s.lanes) * inv + s.eps);
#pragma unroll
            for (int i = 0; i < E; ++i) {
                a[i] = a[i] * rstd * wa[i];
                b[i] = b[i] * rstd * wb[i];
            }
        }
#pragma unroll
        for (int i = 0; i < E; ++i) {
            const float x = a[i], y = b[i];
            a[i] = x * c[i] - y * n[i];
            b[i] = x * n[i] + y * c[i];
        }
        lane.store(s, key ? out.of[1] : out.of[0], to, valid, a, b);
    }
}

// Workgroups of the backward pass that a compute unit's registers hold: 168, 128 or 96 of them to a lane.  (In 96, fp32 pairs and numbers one by one would
// be in memory: 1507 x 48 x 192 53 us and not 45, 5000 x 25 x 50 47 and not 28.)
constexpr uint32_t backward_per_cu(bool bf16, int chunk, bool pairs) { return chunk == 8 ? 3 : chunk == 1 || (!bf16 && chunk == 4 && pairs) ? 4 : 5; }

// With u the gradient of the normed head, turned back and times w: dx = rstd (u - n mean(u n)), n = x rstd; w's gradient is the sum of the turned
// gradient times n over tokens and heads: in a lane's registers, then over the wavefront and the workgroup, which leaves its part in the workspace,
// [workgroup][head].  The first `queries` workgroups take queries, the others keys, as sums for both would take a quarter of the registers; the next
// group's numbers are on their way while a group is worked on.
template <bool BF16, int CHUNK, bool PAIRS, bool NORM>
__global__ __launch_bounds__(64 * kHeadWaves, backward_per_cu(BF16, CHUNK, PAIRS))
void k_heads_backward(HeadTensors grads, HeadTensors in, HeadTensors weights, const int64_t *positions, const uint64_t *frequencies, HeadOutputs out, float *parts, uint32_t queries, HeadShape s)
{
    using Lane = HeadLane<BF16, CHUNK, PAIRS>;
    constexpr int E = Lane::E;
    __shared__ float sums[NORM ? kHeadWaves : 1][NORM ? TAHQ_HEADS_MAX : 1];
    const Lane lane(s);
    const uint32_t wave = uniform(threadIdx.x / 64);
    const float inv = 1.0f / (float)s.head;
    const int which = blockIdx.x < queries ? 0 : 1;
    HeadWay way(s, s.heads[which], (which ? gridDim.x - queries : queries) * kHeadWaves, (which ? blockIdx.x - queries : blockIdx.x) * kHeadWaves + wave);
    float da[E] = {}, db[E] = {}, c[E], n[E];
    // frequencies stay in registers where that leaves room for as many workgroups
    constexpr bool HELD = !NORM || CHUNK == 2 || (BF16 && CHUNK == 4);
    uint64_t f[E], next_position = 0;
    if constexpr (HELD) lane.ask_frequencies(s, frequencies, f);
    typename Lane::Raw next_grad = {}, next_x = {};
    const typename Lane::Raw weight = NORM ? lane.load(s, weights.of[which], 0, true) : typename Lane::Raw{};
    auto ask = [&] {
        if (!way.more()) return;
        const uint64_t at = (uint64_t)way.head() * s.head;
        next_grad = lane.load(s, grads.of[which], way.token() * s.ld_out[which] + at, way.valid());
        if constexpr (NORM) next_x = lane.load(s, in.of[which], way.token() * s.ld[which] + at, way.valid());
        if (s.rotated) next_position = way.position(positions);
    };
    ask();
    bool another = true;
    while (way.more()) {
        const bool valid = way.valid();
        const uint64_t to = way.token() * s.ld[which] + (uint64_t)way.head() * s.head;
        float a[E], b[E], xa[E], xb[E];
        lane.unpack(next_grad, a, b);
        if constexpr (NORM) lane.unpack(next_x, xa, xb);
        if (another) {
            if constexpr (!HELD) lane.ask_frequencies(s, frequencies, f);
            lane.angles(s, next_position, f, c, n);
        }
        another = way.next();
        ask();
#pragma unroll
        for (int i = 0; i < E; ++i) {
            const float x = a[i], y = b[i];
            a[i] = x * c[i] + y * n[i];
            b[i] = y * c[i] - x * n[i];
        }
        if constexpr (NORM) {
            float wa[E], wb[E], square = 0.0f, dot = 0.0f;
            lane.unpack(weight, wa, wb);
#pragma unroll
            for (int i = 0; i < E; ++i) square = __builtin_fmaf(xb[i], xb[i], __builtin_fmaf(xa[i], xa[i], square));
            const float rstd = rsqrtf(head_sum(square, s.lanes) * inv + s.eps);
#pragma unroll
            for (int i = 0; i < E; ++i) {
                xa[i] *= rstd;
                xb[i] *= rstd;
                da[i] = __builtin_fmaf(a[i], xa[i], da[i]);
                db[i] = __builtin_fmaf(b[i], xb[i], db[i]);
                a[i] *= wa[i];
                b[i] *= wb[i];
                dot = __builtin_fmaf(b[i], xb[i], __builtin_fmaf(a[i], xa[i], dot));
            }
            const float mean = head_sum(dot, s.lanes) * inv;
#pragma unroll
            for (int i = 0; i < E; ++i) {
                a[i] = rstd * __builtin_fmaf(-xa[i], mean, a[i]);
                b[i] = rstd * __builtin_fmaf(-xb[i], mean, b[i]);
            }
        }
        lane.store(s, out.of[which], to, valid, a, b);
    }
    if constexpr (NORM) {
#pragma unroll
        for (int i = 0; i < E; ++i) {
            float a = da[i], b = db[i];
            for (uint32_t step = s.lanes; step < 64; step *= 2) {
                a += __shfl_xor(a, (int)step);
                b += __shfl_xor(b, (int)step);
            }
            if (threadIdx.x % 64 < s.lanes) {
                const uint32_t ca = lane.channel(s, i, 0), cb = lane.channel(s, i, 1);
                if (ca < s.head) sums[wave][ca] = a;
                if (cb < s.head) sums[wave][cb] = b;
            }
        }
        __syncthreads();
        for (uint32_t at = threadIdx.x; at < s.head; at += 64 * kHeadWaves) {
            float sum = sums[0][at];
            for (uint32_t w = 1; w < kHeadWaves; ++w) sum += sums[w][at];
            parts[(uint64_t)blockIdx.x * s.head + at] = sum;
        }
    }
}

// The workgroups' parts, added in a fixed order: 16 channels of 64 runs of workgroups to a block.  blockIdx.y: queries', keys'.
__global__ __launch_bounds__(1024)
void k_heads_reduce(const float *parts, float *grad_w_q, float *grad_w_k, uint32_t head, uint32_t queries, uint32_t workgroups, uint32_t accumulate)
{
    __shared__ float sums[1024];
    const uint32_t base = blockIdx.y ? queries : 0, count = blockIdx.y ? workgroups - queries : queries;
    const uint32_t c = blockIdx.x * 16 + threadIdx.x % 16, run = threadIdx.x / 16, each = (count + 63) / 64;
    float sum = 0.0f;
    if (c < head)
        for (uint32_t i = run * each, end = min((run + 1) * each, count); i < end; i += 8) {
            float v[8];
#pragma unroll
            for (uint32_t k = 0; k < 8; ++k) v[k] = i + k < end ? parts[(uint64_t)(base + i + k) * head + c] : 0.0f;
            sum += ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
        }
    sums[threadIdx.x] = sum;
    __syncthreads();
    for (uint32_t half = 512; half >= 16; half /= 2) {
        if (threadIdx.x < half) sums[threadIdx.x] += sums[threadIdx.x + half];
        __syncthreads();
    }
    float *to = blockIdx.y ? grad_w_k : grad_w_q;
    if (run == 0 && c < head) to[c] = accumulate ? to[c] + sums[threadIdx.x] : sums[threadIdx.x];
}

}  // namespace tahq
