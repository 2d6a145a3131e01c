// The norms before and after a block with its gate and residual scale (include/tahq_norm.h), forward and backward.
//
// Bound by memory: four tensors forward (two and 17/32 of a byte an element where h leaves in mx4), six backward, each once.  A
// workgroup takes a row at a time, so that both of its row sums come from registers.
#pragma once
#include "tahq_mx4_common.hpp"

namespace tahq {

struct NormShape {
    uint32_t rows, cols, gate_rows;
    float eps, alpha;
};

// How many of the eight channels from c on a row has, as far as load8 and store8 care; rows of whole eights need no code for others.
template <bool EIGHTS>
__device__ __forceinline__ int64_t valid8(uint32_t C, uint32_t c)
{
    if constexpr (EIGHTS) return c < C ? 8 : 0;
    else return (int64_t)C - c;
}

// Sum over a workgroup, the same in every lane: a butterfly in each wavefront, then the wavefronts' sums from LDS in order.  `turn`
// alternates between two places, so that one barrier per sum is enough: nobody writes a place again before all have passed the
// barrier of the sum in between.
template <int NT>
__device__ __forceinline__ float group_sum(float v, float (*places)[NT / 64], uint32_t &turn)
{
    float (*slot)[NT / 64] = places + turn;
    turn ^= 1;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) v += __shfl_xor(v, d, 64);
    if constexpr (NT == 64) {
        return v;
    } else {
        if (threadIdx.x % 64 == 0) (*slot)[threadIdx.x / 64] = v;
        __syncthreads();
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < NT / 64; ++i) s += (*slot)[i];
        return s;
    }
}

template <bool BF16, bool EIGHTS, int NT, int V>
__global__ __launch_bounds__(NT)
void k_norm_forward(const void *residual, const void *block, const void *w_post, const void *gate, const void *w_pre,
                    void *residual_out, void *h, uint8_t *h_mx4, float *stats, NormShape s, uint32_t cover, uint32_t rotate,
                    uint32_t rows_each)
{
    __shared__ float sums[2][NT / 64];
    uint32_t turn = 0;
    const uint32_t tid = threadIdx.x, C = s.cols;
    auto valid = [&](uint32_t c) { return valid8<EIGHTS>(C, c); };
    const Mx4Layout L(s.rows, C);
    const uint32_t end = h_mx4 ? 32 * L.rb : s.rows;
    const uint32_t first = blockIdx.x * rows_each, last = min(first + rows_each, end);
    for (uint32_t row = first; row < last; ++row) {
        const bool there = row < s.rows;                                   // rows behind fill up the packed matrix with zeros
        const uint64_t base = (uint64_t)row * C;
        float x[V][8];
        float rstd_b = 0.0f, rstd_r = 0.0f;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const uint32_t c = 8 * (v * NT + tid);
            load8<BF16, EIGHTS>(residual, base + c, there ? valid(c) : 0, x[v]);
#pragma unroll
            for (int i = 0; i < 8; ++i) x[v][i] *= s.alpha;
        }
        if (block && there) {
            float b[V][8], sum = 0.0f;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const uint32_t c = 8 * (v * NT + tid);
                load8<BF16, EIGHTS>(block, base + c, valid(c), b[v]);
#pragma unroll
                for (int i = 0; i < 8; ++i) sum = __builtin_fmaf(b[v][i], b[v][i], sum);
            }
            rstd_b = 1.0f / __builtin_sqrtf(group_sum<NT>(sum, sums, turn) / (float)C + s.eps);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const uint32_t c = 8 * (v * NT + tid);
                float w[8];
                load8<BF16, EIGHTS>(w_post, c, valid(c), w);
                if (gate) {
                    float g[8];
                    load8<BF16, EIGHTS>(gate, (uint64_t)(row / s.gate_rows) * C + c, valid(c), g);
#pragma unroll
                    for (int i = 0; i < 8; ++i) b[v][i] *= g[i];
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) x[v][i] = __builtin_fmaf(b[v][i] * rstd_b, w[i], x[v][i]);
            }
        }
        if (residual_out && there) {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const uint32_t c = 8 * (v * NT + tid);
                store8<BF16, EIGHTS>(residual_out, base + c, valid(c), x[v]);
            }
        }
        if (w_pre) {
            float sum = 0.0f;
#pragma unroll
            for (int v = 0; v < V; ++v)
#pragma unroll
                for (int i = 0; i < 8; ++i) sum = __builtin_fmaf(x[v][i], x[v][i], sum);
            rstd_r = 1.0f / __builtin_sqrtf(group_sum<NT>(sum, sums, turn) / (float)C + s.eps);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const uint32_t c = 8 * (v * NT + tid);
                float w[8];
                load8<BF16, EIGHTS>(w_pre, c, valid(c), w);
#pragma unroll
                for (int i = 0; i < 8; ++i) x[v][i] = x[v][i] * rstd_r * w[i];
                if (h && there) store8<BF16, EIGHTS>(h, base + c, valid(c), x[v]);
                if (h_mx4) {
                    uint32_t e;
                    const uint32_t codes = rotate ? quantize_quad<true>(x[v], cover, e) : quantize_quad<false>(x[v], cover, e);
                    const uint32_t blk = c / 32;
                    if (blk / 2 < L.kb) *reinterpret_cast<uint32_t *>(h_mx4 + L.code(row, blk) + tid % 4 * 4) = codes;
                    if (tid % 4 == 0 && blk / 8 < L.kc) h_mx4[L.scale(row, blk)] = (uint8_t)e;
                }
            }
        }
        if (stats && there && tid == 0) {
            stats[row] = rstd_b;
            stats[(uint64_t)s.rows + row] = rstd_r;
        }
    }
}

// Column sums of a workgroup's rows, in the workspace: post [W][C], pre [W][C], gate [W][2][C].  A group of rows that share a row of
// the gate and lie in one workgroup has its sum written at once; of a group that several workgroups have rows of, each keeps its part: in slot 0
// if the workgroup's first row is in the group, in slot 1 otherwise.
struct NormPartials {
    float *post, *pre, *gate;
};

__device__ __forceinline__ void put(float *to, uint32_t c, uint32_t C, const float (&v)[8], bool add)
{
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (c + i < C) to[c + i] = add ? to[c + i] + v[i] : v[i];
}

template <bool BF16, bool EIGHTS, int NT, int V>
__global__ __launch_bounds__(NT)
void k_norm_backward(const void *grad_out, const void *grad_h, const void *block, const void *w_post, const void *gate,
                     const void *residual_out, const void *w_pre, const float *stats, void *grad_residual, void *grad_block,
                     float *grad_gate, NormPartials parts, NormShape s, uint32_t rows_each, uint32_t accumulate)
{
    __shared__ float sums[2][NT / 64];
    uint32_t turn = 0;
    const uint32_t tid = threadIdx.x, C = s.cols;
    auto valid = [&](uint32_t c) { return valid8<EIGHTS>(C, c); };
    const uint32_t first = blockIdx.x * rows_each, last = min(first + rows_each, s.rows);
    const float inv_c = 1.0f / (float)C;
    float post[V][8] = {}, pre[V][8] = {}, gates[V][8] = {};
    for (uint32_t row = first; row < last; ++row) {
        const uint64_t base = (uint64_t)row * C;
        float g[V][8];
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const uint32_t c = 8 * (v * NT + tid);
            load8<BF16, EIGHTS>(grad_out, base + c, grad_out ? valid(c) : 0, g[v]);
        }
        if (grad_h) {
            const float rstd = stats[(uint64_t)s.rows + row];
            float x2[V][8], t[V][8], sum = 0.0f;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const uint32_t c = 8 * (v * NT + tid);
                float w[8];
                load8<BF16, EIGHTS>(grad_h, base + c, valid(c), t[v]);
                load8<BF16, EIGHTS>(residual_out, base + c, valid(c), x2[v]);
                load8<BF16, EIGHTS>(w_pre, c, valid(c), w);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    x2[v][i] *= rstd;
                    pre[v][i] = __builtin_fmaf(t[v][i], x2[v][i], pre[v][i]);
                    t[v][i] *= w[i];
                    sum = __builtin_fmaf(t[v][i], x2[v][i], sum);
                }
            }
            const float mean = group_sum<NT>(sum, sums, turn) * inv_c;
#pragma unroll
            for (int v = 0; v < V; ++v)
#pragma unroll
                for (int i = 0; i < 8; ++i) g[v][i] = __builtin_fmaf(rstd, __builtin_fmaf(-x2[v][i], mean, t[v][i]), g[v][i]);
        }
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const uint32_t c = 8 * (v * NT + tid);
            float d[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) d[i] = s.alpha * g[v][i];
            store8<BF16, EIGHTS>(grad_residual, base + c, valid(c), d);
        }
        if (block) {
            const float rstd = stats[row];
            float x1[V][8], sum = 0.0f;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const uint32_t c = 8 * (v * NT + tid);
                float w[8];
                load8<BF16, EIGHTS>(block, base + c, valid(c), x1[v]);
                load8<BF16, EIGHTS>(w_post, c, valid(c), w);
#pragma unroll
                for (int i = 0; i < 8; ++i) x1[v][i] *= rstd;
                if (gate) {
                    float k[8];
                    load8<BF16, EIGHTS>(gate, (uint64_t)(row / s.gate_rows) * C + c, valid(c), k);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        gates[v][i] = __builtin_fmaf(g[v][i] * x1[v][i], w[i], gates[v][i]);
                        g[v][i] *= k[i];
                    }
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    post[v][i] = __builtin_fmaf(g[v][i], x1[v][i], post[v][i]);
                    g[v][i] *= w[i];
                    sum = __builtin_fmaf(g[v][i], x1[v][i], sum);
                }
            }
            const float mean = group_sum<NT>(sum, sums, turn) * inv_c;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const uint32_t c = 8 * (v * NT + tid);
                float d[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) d[i] = rstd * __builtin_fmaf(-x1[v][i], mean, g[v][i]);
                store8<BF16, EIGHTS>(grad_block, base + c, valid(c), d);
            }
            if (gate) {
                const uint32_t group = row / s.gate_rows;
                if (row + 1 == last || (row + 1) / s.gate_rows != group) {
                    const uint32_t begin = group * s.gate_rows;
                    const uint32_t stop = (uint32_t)min((uint64_t)begin + s.gate_rows, (uint64_t)s.rows);
                    const bool whole = begin >= first && stop <= last;
                    float *to = whole ? grad_gate + (uint64_t)group * C
                                      : parts.gate + ((uint64_t)blockIdx.x * 2 + (begin <= first ? 0 : 1)) * C;
#pragma unroll
                    for (int v = 0; v < V; ++v) {
                        put(to, 8 * (v * NT + tid), C, gates[v], whole && accumulate);
#pragma unroll
                        for (int i = 0; i < 8; ++i) gates[v][i] = 0.0f;
                    }
                }
            }
        }
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const uint32_t c = 8 * (v * NT + tid);
        if (block) put(parts.post + (uint64_t)blockIdx.x * C, c, C, post[v], false);
        if (grad_h) put(parts.pre + (uint64_t)blockIdx.x * C, c, C, pre[v], false);
    }
}

// The workgroups' column sums, added in order: 64 columns x 4 runs of workgroups.  blockIdx.y: 0 post, 1 pre, then the groups of the gate.
__global__ __launch_bounds__(256)
void k_norm_reduce(NormPartials parts, float *grad_w_post, float *grad_w_pre, float *grad_gate, uint32_t C, uint32_t W,
                   uint32_t rows, uint32_t gate_rows, uint32_t rows_each, uint32_t groups, uint32_t accumulate)
{
    __shared__ float runs[4][64];
    const uint32_t lane = threadIdx.x % 64, run = threadIdx.x / 64, c = blockIdx.x * 64 + lane;
    auto total = [&](auto part, uint32_t n, float *to) {
        const uint32_t each = (n + 3) / 4, from = min(run * each, n), till = min(from + each, n);
        float sum = 0.0f;
        if (c < C)
            for (uint32_t i = from; i < till; ++i) sum += part(i)[c];
        runs[run][lane] = sum;
        __syncthreads();
        if (run == 0 && c < C) {
            const float t = ((runs[0][lane] + runs[1][lane]) + runs[2][lane]) + runs[3][lane];
            to[c] = accumulate ? to[c] + t : t;
        }
        __syncthreads();
    };
    if (blockIdx.y == 0) {
        if (grad_w_post) total([&](uint32_t i) { return parts.post + (uint64_t)i * C; }, W, grad_w_post);
    } else if (blockIdx.y == 1) {
        if (grad_w_pre) total([&](uint32_t i) { return parts.pre + (uint64_t)i * C; }, W, grad_w_pre);
    } else {
        // groups in more than one workgroup: each of them holds the last row in front of some workgroup's first
        const uint32_t stride = gridDim.y - 2;
        const bool by_group = groups <= W;
        const uint32_t count = by_group ? groups : W - 1;
        for (uint32_t i = blockIdx.y - 2; i < count; i += stride) {
            const uint32_t group = by_group ? i : ((i + 1) * rows_each - 1) / gate_rows;
            const uint32_t begin = group * gate_rows, stop = (uint32_t)min((uint64_t)begin + gate_rows, (uint64_t)rows);
            const uint32_t w0 = begin / rows_each, w1 = (stop - 1) / rows_each;
            if (w0 == w1 || (!by_group && w0 != i)) continue;
            total([&](uint32_t j) { return parts.gate + ((uint64_t)(w0 + j) * 2 + (j == 0 && begin > w0 * rows_each ? 1 : 0)) * C; },
                  w1 - w0 + 1, grad_gate + (uint64_t)group * C);
        }
    }
}

}  // namespace tahq
