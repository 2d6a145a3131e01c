// The norms before and after a block with its gate and residual scale (include/tahq_norm.h), forward and backward.
//
// Bound by memory: four tensors forward (three and 17/32 of a byte an element where h leaves in mx4), six backward, each once.  A
// workgroup takes a row at a time, eight channels to a lane and no more wavefronts than that needs, so that both of its row sums come
// from registers; the next row is on its way meanwhile.
//   Measured, bf16: forward 8192 x 4096 to mx4 with a gate 50 us (219 MB, 4.4 TB/s), one row of 4096 2.9 us, a launch's time (5.0 out
// of HBM); backward 32768 x 5120 386 to 398 us (2.0 GB, 5.1 TB/s, as a large copy) and its column sums 10.  Halves alone, 32768 x 5120:
// forward post 188, pre 178 (1.0 GB), backward post 252 (1.3 GB), pre without a gradient of r' 214 (1.0 GB).
#pragma once
#include "tahq_lanes.hpp"
#include "tahq_mx4_common.hpp"

namespace tahq {

struct NormShape {
    uint32_t rows, cols, gate_rows, waves;     // waves: of a workgroup
    float eps, alpha;
};
constexpr int kNormWaves = TAHQ_NORM_MAX_COLS / 512;       // at most, in a workgroup

// A gate of ones, for where there is none
template <bool BF16>
__device__ __forceinline__ Eight<BF16> ones()
{
    constexpr uint32_t one = BF16 ? 0x3f803f80u : 0x3f800000u;
    Eight<BF16> e;
    for (uint4 &p : e.q) p = make_uint4(one, one, one, one);
    return e;
}
// A row's address, the same in all lanes, so that a lane's own part of an address is its 32-bit offset in the row; worked out anew for every row
// in scalar registers, where a pointer per tensor carried along would take two vector registers
template <bool BF16>
__device__ __forceinline__ const void *row_of(const void *t, uint32_t row, uint32_t C)
{
    return static_cast<const uint8_t *>(t) + (uint64_t)uniform(row) * C * (BF16 ? 2 : 4);
}
template <bool BF16>
__device__ __forceinline__ void *row_of(void *t, uint32_t row, uint32_t C)
{
    return static_cast<uint8_t *>(t) + (uint64_t)uniform(row) * C * (BF16 ? 2 : 4);
}
// Keeps a lane's channels as they lie in memory: unpacked once for all rows they would take twice the registers
template <bool BF16>
__device__ __forceinline__ void stay_packed(Eight<BF16> &e)
{
    if constexpr (BF16) asm volatile("" : "+v"(e.q[0].x), "+v"(e.q[0].y), "+v"(e.q[0].z), "+v"(e.q[0].w));
}

// Sum over a workgroup of `waves` wavefronts, the same in every lane; places of wavefronts that there are not hold zeros.  `turn` alternates
// between two places, so that one barrier per sum is enough: nobody writes a place again before all have passed the barrier of the sum in between.
struct Places {
    float of[2][16];
};
static_assert(kNormWaves <= 16, "a row of sixteen lanes adds the wavefronts' sums");

__device__ __forceinline__ float group_sum(float v, uint32_t waves, Places &places, uint32_t &turn)
{
    v = wave_sum(v);
    if (waves == 1) return v;
    if (threadIdx.x % 64 == 0) places.of[turn][threadIdx.x / 64] = v;
    __syncthreads();
    v = places.of[turn][threadIdx.x % 16];
    turn ^= 1;
    v = add_permuted<0xb1>(v);
    v = add_permuted<0x4e>(v);
    v = add_permuted<0x141>(v);
    return add_permuted<0x140>(v);
}
__device__ __forceinline__ void clear(Places &places)
{
    if (threadIdx.x < 32) reinterpret_cast<float *>(&places)[threadIdx.x] = 0.0f;
    __syncthreads();
}
// Sums that are up to date here: otherwise the compiler keeps what they are of over the barrier, in registers that would be another workgroup's
__device__ __forceinline__ void settle(float (&v)[8])
{
#pragma unroll
    for (int i = 0; i < 8; ++i) asm volatile("" : "+v"(v[i]));
}

// Forward, elements are rounded operation by operation, in the formulas' order: h is then what unfused operations give, and its codes are, too,
// but in rows whose sum comes out differently in the last place.  Of 2000 x 4096 fp32 elements 72 % have the same bits; with explicit fused
// multiply-adds and 1 / sqrt 49 %, and no less time, as memory is waited for.  Against 64 bits both err alike: the rounding that a fused
// multiply-add saves is given up for equal bits.
__device__ __forceinline__ float rstd_of(float sum, float inv_c, float eps) { return rsqrtf(sum * inv_c + eps); }

// POST, PRE: whether the halves are there
template <bool BF16, bool EIGHTS, bool POST, bool PRE>
__global__ __launch_bounds__(64 * kNormWaves)
void k_norm_forward(const void *residual, const void *block, const void *w_post, const void *gate, const void *w_pre,
                    void *residual_out, void *h, uint8_t *h_mx4, float *stats, NormShape s, uint32_t cover, uint32_t rotate,
                    uint32_t rows_each, uint32_t together)
{
    __shared__ Places places;
    uint32_t turn = 0;
    const uint32_t C = s.cols, c = 8 * threadIdx.x;
    const bool mine = c < C;
    const Mx4Layout L(s.rows, C);
    const uint32_t end = h_mx4 ? 32 * L.rb : s.rows;       // rows behind the last one fill up the packed matrix with zeros
    // The workgroups of 256 rows in another order, so that a unit's rows, whose codes lie side by side in a line, are on one XCD and merge in its
    // L2: 8192 x 4096 bf16 to mx4 57 -> 52 us, to h and mx4 58 -> 51.  `together`, workgroups for 256 rows, is a power of two;
    // 1: their own order.
    uint32_t place = blockIdx.x;
    const uint32_t in = place & (together - 1);
    if (h_mx4 && place - in + together <= gridDim.x) place += in % 8 * (together / 8) + in / 8 - in;
    const uint32_t first = place * rows_each, last = min(first + rows_each, end);
    Eight<BF16> next_r = {}, next_b = {}, post = {}, pre = {}, next_k = ones<BF16>();
    auto ask = [&](uint32_t row) {
        if (row < s.rows && row < last && mine) {
            next_r = fetch<BF16, EIGHTS>(row_of<BF16>(residual, row, C), c, C, more_behind(row, s.rows, C));
            if constexpr (POST) {
                next_b = fetch<BF16, EIGHTS>(row_of<BF16>(block, row, C), c, C, more_behind(row, s.rows, C));
                if (gate) next_k = fetch<BF16, EIGHTS>(row_of<BF16>(gate, row / s.gate_rows, C), c, C, false);
            }
        }
    };
    ask(first);
    if (mine) {
        if constexpr (POST) post = fetch<BF16, EIGHTS>(w_post, c, C, false);
        if constexpr (PRE) pre = fetch<BF16, EIGHTS>(w_pre, c, C, false);
    }
    clear(places);
    const float inv_c = 1.0f / (float)C;
    for (uint32_t row = first; row < last; ++row) {
        const bool there = row < s.rows;
        stay_packed(post);
        stay_packed(pre);
        float x[8], rstd_b = 0.0f, rstd_r = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = there ? s.alpha * next_r[i] : 0.0f;
        if constexpr (POST) {
            const Eight<BF16> b = next_b, k = next_k;
            ask(row + 1);
            float sum = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) sum = __builtin_fmaf(b[i], b[i], sum);
            rstd_b = rstd_of(group_sum(sum, s.waves, places, turn), inv_c, s.eps);
            if (there) {
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = x[i] + b[i] * rstd_b * post[i] * k[i];
            }
        } else {
            ask(row + 1);
        }
        if (residual_out && there && mine) keep<BF16, EIGHTS>(row_of<BF16>(residual_out, row, C), c, C, x);
        if constexpr (PRE) {
            float sum = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) sum = __builtin_fmaf(x[i], x[i], sum);
            rstd_r = rstd_of(group_sum(sum, s.waves, places, turn), inv_c, s.eps);
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = x[i] * rstd_r * pre[i];
            if (h && there && mine) keep<BF16, EIGHTS>(row_of<BF16>(h, row, C), c, C, x);
            if (h_mx4) {
                // what fills up the packed matrix: zeros, also where the statistics or the weight's sign would make NaN or -0 of them
#pragma unroll
                for (uint32_t i = 0; i < 8; ++i) x[i] = there && (EIGHTS ? mine : c + i < C) ? x[i] : 0.0f;
                uint32_t e;
                const uint32_t codes = rotate ? quantize_quad<true>(x, cover, e) : quantize_quad<false>(x, cover, e);
                const uint32_t blk = c / 32;
                if (blk / 2 < L.kb) *reinterpret_cast<uint32_t *>(h_mx4 + L.code(row, blk) + threadIdx.x % 4 * 4) = codes;
                if (threadIdx.x % 4 == 0 && blk / 8 < L.kc) h_mx4[L.scale(row, blk)] = (uint8_t)e;
            }
        }
        if (stats && there && threadIdx.x == 0) {
            stats[row] = rstd_b;
            stats[(uint64_t)s.rows + row] = rstd_r;
        }
    }
}

// Teams of workgroups share a span of rows, `rows_each` for each workgroup, and take them in turn, so that what all of them work on at a time lies
// close together in memory.  Where there is a gate, a span is no longer than the rows that share one of its rows, so that it has rows of two of these
// groups at most; in a team of one workgroup it may have any number of them.
struct NormSpan {
    uint32_t base, last, first, step;          // rows base .. last - 1; this workgroup's: first, first + step, .., one at least
    __device__ __forceinline__ NormSpan(uint32_t wg, uint32_t workgroups, uint32_t team, uint32_t rows_each, uint32_t rows)
    {
        const uint32_t member = wg % team;
        base = (wg - member) * rows_each;
        step = min(team, workgroups - (wg - member));
        last = min(base + step * rows_each, rows);
        first = base + member;
    }
};
// Column sums of a workgroup's rows, in the workspace: post [W][C], pre [W][C], gate [W][2][C].  A group of rows that share a row of
// the gate and lie in one workgroup has its sum written at once; of a group that several workgroups have rows of, each keeps its part: in slot 0
// if the first row of its span is in the group, in slot 1 otherwise.
struct NormPartials {
    float *post, *pre, *gate;
};

template <bool EIGHTS>
__device__ __forceinline__ void put(float *row, uint32_t c, uint32_t C, float (&v)[8], bool add)
{
    if (c >= C) return;
    if (add) {
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i)
            if (EIGHTS || c + i < C) v[i] += row[c + i];
    }
    keep<false, EIGHTS>(row, c, C, v);
}

template <bool BF16, bool EIGHTS, bool POST, bool PRE>
__global__ __launch_bounds__(64 * kNormWaves)
void k_norm_backward(const void *grad_out, const void *grad_h, const void *block, const void *w_post, const void *gate,
                     const void *residual_out, const void *w_pre, const float *__restrict__ stats, void *grad_residual, void *grad_block,
                     float *grad_gate, NormPartials parts, NormShape s, uint32_t rows_each, uint32_t team, uint32_t accumulate)
{
    __shared__ Places places;
    uint32_t turn = 0;
    const uint32_t C = s.cols, c = 8 * threadIdx.x;
    const bool mine = c < C;
    const NormSpan span(blockIdx.x, gridDim.x, team, rows_each, s.rows);
    const uint32_t first = span.first, last = span.last, step = span.step;
    const float inv_c = 1.0f / (float)C;
    // the row that is worked on, loaded again as soon as it is used up
    Eight<BF16> go = {}, gh = {}, ro = {}, bl = {}, k = ones<BF16>(), wpost = {}, wpre = {};
    auto ask_pre = [&](uint32_t row) {
        if (row < last && mine) {
            if constexpr (PRE) {
                gh = fetch<BF16, EIGHTS>(row_of<BF16>(grad_h, row, C), c, C, more_behind(row, s.rows, C));
                ro = fetch<BF16, EIGHTS>(row_of<BF16>(residual_out, row, C), c, C, more_behind(row, s.rows, C));
            }
            if (grad_out) go = fetch<BF16, EIGHTS>(row_of<BF16>(grad_out, row, C), c, C, more_behind(row, s.rows, C));
        }
    };
    auto ask_post = [&](uint32_t row) {
        if (POST && row < last && mine) bl = fetch<BF16, EIGHTS>(row_of<BF16>(block, row, C), c, C, more_behind(row, s.rows, C));
    };
    // the rows of one gate row; they change on the way
    uint32_t group = 0, stop = 0;
    auto ask_gate = [&](uint32_t row) {
        group = row / s.gate_rows;
        stop = (uint32_t)min((uint64_t)group * s.gate_rows + s.gate_rows, (uint64_t)s.rows);
        if (mine) k = fetch<BF16, EIGHTS>(row_of<BF16>(gate, group, C), c, C, false);
    };
    ask_pre(first);
    ask_post(first);
    if (mine) {
        if constexpr (POST) wpost = fetch<BF16, EIGHTS>(w_post, c, C, false);
        if constexpr (PRE) wpre = fetch<BF16, EIGHTS>(w_pre, c, C, false);
    }
    if (POST && gate) ask_gate(first);
    clear(places);
    float post[8] = {}, pre[8] = {}, gates[8] = {};
    for (uint32_t row = first; row < last; row += step) {
        stay_packed(wpost);
        stay_packed(wpre);
        stay_packed(k);
        float g[8];
        if constexpr (PRE) {
            const float rstd = stats[(uint64_t)s.rows + row];
            float sum = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float x2 = ro[i] * rstd;
                pre[i] = __builtin_fmaf(gh[i], x2, pre[i]);
                sum = __builtin_fmaf(gh[i] * wpre[i], x2, sum);
            }
            settle(pre);
            stay_packed(gh);
            stay_packed(ro);
            stay_packed(wpre);
            const float mean = group_sum(sum, s.waves, places, turn) * inv_c;
#pragma unroll
            for (int i = 0; i < 8; ++i) g[i] = __builtin_fmaf(rstd, __builtin_fmaf(-(ro[i] * rstd), mean, gh[i] * wpre[i]), go[i]);
            settle(g);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) g[i] = go[i];
        }
        ask_pre(row + step);
        float d[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) d[i] = s.alpha * g[i];
        if (mine) keep<BF16, EIGHTS>(row_of<BF16>(grad_residual, row, C), c, C, d);
        if constexpr (POST) {
            const float rstd = stats[row];
            float sum = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float x1 = bl[i] * rstd;
                gates[i] = __builtin_fmaf(g[i] * x1, wpost[i], gates[i]);
                g[i] *= k[i];
                post[i] = __builtin_fmaf(g[i], x1, post[i]);
                g[i] *= wpost[i];
                sum = __builtin_fmaf(g[i], x1, sum);
            }
            settle(gates);
            settle(post);
            settle(g);
            stay_packed(bl);
            const float mean = group_sum(sum, s.waves, places, turn) * inv_c;
#pragma unroll
            for (int i = 0; i < 8; ++i) d[i] = rstd * __builtin_fmaf(-(bl[i] * rstd), mean, g[i]);
            ask_post(row + step);
            if (mine) keep<BF16, EIGHTS>(row_of<BF16>(grad_block, row, C), c, C, d);
            if (gate && (row + step >= last || row + step >= stop)) {
                const uint32_t begin = group * s.gate_rows;
                const bool whole = team == 1 && begin >= first && stop <= last;
                float *to = whole ? grad_gate + (uint64_t)group * C
                                  : parts.gate + ((uint64_t)blockIdx.x * 2 + (begin <= span.base ? 0 : 1)) * C;
                put<EIGHTS>(to, c, C, gates, whole && accumulate);
#pragma unroll
                for (int i = 0; i < 8; ++i) gates[i] = 0.0f;
                if (row + step < last) ask_gate(row + step);
            }
        }
    }
    if (POST && gate && team > 1) {
        // groups of the span that none of this workgroup's rows are in: their parts are zeros, as `gates` is now
        const uint32_t next = (uint32_t)min((uint64_t)(span.base / s.gate_rows + 1) * s.gate_rows, (uint64_t)s.rows);      // the second group's first row
        if (first >= next)
            put<EIGHTS>(parts.gate + (uint64_t)blockIdx.x * 2 * C, c, C, gates, false);
        if (first < next && next < last && next + (step - (next - first) % step) % step >= last)
            put<EIGHTS>(parts.gate + ((uint64_t)blockIdx.x * 2 + 1) * C, c, C, gates, false);
    }
    if constexpr (POST) put<EIGHTS>(parts.post + (uint64_t)blockIdx.x * C, c, C, post, false);
    if constexpr (PRE) put<EIGHTS>(parts.pre + (uint64_t)blockIdx.x * C, c, C, pre, false);
}

// The workgroups' column sums, added in a fixed order by blocks of 1024 lanes: `width` columns (64; 16 where there are few, to have more blocks) x
// 1024 / width runs of workgroups, eight loads of a run on their way at a time.  blockIdx.y: 0 post, 1 pre, then the groups of the gate.
constexpr uint32_t kReduceLanes = 1024;

__global__ __launch_bounds__(kReduceLanes)
void k_norm_reduce(NormPartials parts, float *grad_w_post, float *grad_w_pre, float *grad_gate, uint32_t C, uint32_t W,
                   uint32_t rows, uint32_t gate_rows, uint32_t rows_each, uint32_t team, uint32_t groups, uint32_t accumulate, uint32_t width)
{
    __shared__ float sums[kReduceLanes];
    const uint32_t lane = threadIdx.x % width, run = threadIdx.x / width, runs = kReduceLanes / width, c = blockIdx.x * width + lane;
    auto total = [&](auto part, uint32_t n, float *to) {
        const uint32_t each = (n + runs - 1) / runs, from = min(run * each, n), till = min(from + each, n);
        float sum = 0.0f;
        if (c < C)
            for (uint32_t i = from; i < till; i += 8) {
                float v[8];
#pragma unroll
                for (uint32_t k = 0; k < 8; ++k) v[k] = i + k < till ? part(i + k)[c] : 0.0f;
                sum += ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
            }
        sums[threadIdx.x] = sum;
        __syncthreads();
        for (uint32_t half = kReduceLanes / 2; half >= width; half /= 2) {
            if (threadIdx.x < half) sums[threadIdx.x] += sums[threadIdx.x + half];
            __syncthreads();
        }
        if (run == 0 && c < C) to[c] = accumulate ? to[c] + sums[lane] : sums[lane];
        __syncthreads();
    };
    if (blockIdx.y == 0) {
        if (grad_w_post) total([&](uint32_t i) { return parts.post + (uint64_t)i * C; }, W, grad_w_post);
    } else if (blockIdx.y == 1) {
        if (grad_w_pre) total([&](uint32_t i) { return parts.pre + (uint64_t)i * C; }, W, grad_w_pre);
    } else {
        // Groups in more than one workgroup: each of them holds the last row in front of some workgroup's first.  Teams of several have at most as
        // many groups as there are workgroups, and none is written yet.
        const uint32_t stride = gridDim.y - 2, span = team * rows_each;
        const bool by_group = groups <= W;
        const uint32_t count = by_group ? groups : W - 1;
        for (uint32_t i = blockIdx.y - 2; i < count; i += stride) {
            const uint32_t group = by_group ? i : ((i + 1) * rows_each - 1) / gate_rows;
            const uint32_t begin = group * gate_rows, stop = (uint32_t)min((uint64_t)begin + gate_rows, (uint64_t)rows);
            const uint32_t w0 = begin / span * team, w1 = min((stop - 1) / span * team + team, W) - 1;
            if (team == 1 && (w0 == w1 || (!by_group && w0 != i))) continue;
            // slot 1 in those whose span begins before the group
            const uint32_t late = begin > w0 * rows_each ? team : 0;
            total([&](uint32_t j) { return parts.gate + ((uint64_t)(w0 + j) * 2 + (j < late ? 1 : 0)) * C; },
                  w1 - w0 + 1, grad_gate + (uint64_t)group * C);
        }
    }
}

}  // namespace tahq
