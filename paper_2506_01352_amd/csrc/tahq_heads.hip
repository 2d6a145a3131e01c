// Entry points of the heads' norms and rotation (include/tahq_heads.h): validation, plan, launches.
#include <math.h>

#include <type_traits>

#include "tahq_enqueue.hpp"
#include "tahq_heads.h"
#include "tahq_heads_kernels.hpp"

using namespace tahq;

namespace {

tahq_status check(const tahq_heads_config *c)
{
    if (!c) return TAHQ_ERR_NULL;
    if (c->struct_size != sizeof *c) return TAHQ_ERR_INVALID_ARG;
    if (c->tokens == 0 || c->tokens >= 0x80000000u || c->q_heads == 0 || c->head == 0 || c->dtype > TAHQ_BF16) return TAHQ_ERR_INVALID_ARG;
    if (c->q_heads >= 0x10000u || c->k_heads >= 0x10000u || c->q_heads + c->k_heads >= 0x10000u) return TAHQ_ERR_INVALID_ARG;
    if (c->rotated % 2 || c->rotated > c->head || c->layout > TAHQ_HEADS_PAIRS || c->norm > 1 || c->accumulate > 1) return TAHQ_ERR_INVALID_ARG;
    if (!(c->eps > 0.0f) || !(c->eps <= 3.4028234663852886e38f)) return TAHQ_ERR_INVALID_ARG;
    if (!(__builtin_fabsf(c->magnitude) <= 3.4028234663852886e38f)) return TAHQ_ERR_INVALID_ARG;
    if (c->head > TAHQ_HEADS_MAX) return TAHQ_ERR_UNSUPPORTED;
    for (const uint32_t ld : {c->ldq, c->ldq_out})
        if (ld && ld < c->q_heads * c->head) return TAHQ_ERR_INVALID_ARG;
    for (const uint32_t ld : {c->ldk, c->ldk_out})
        if (ld && ld < c->k_heads * c->head) return TAHQ_ERR_INVALID_ARG;
    return TAHQ_OK;
}

uint32_t esize(const tahq_heads_config *c) { return c->dtype == TAHQ_BF16 ? 2 : 4; }

HeadShape shape_of(const tahq_heads_config *c)
{
    HeadShape s = {};
    s.tokens = c->tokens;
    s.heads[0] = c->q_heads;
    s.heads[1] = c->k_heads;
    s.head = c->head;
    s.rotated = c->rotated;
    s.ld[0] = c->ldq ? c->ldq : c->q_heads * c->head;
    s.ld[1] = c->ldk ? c->ldk : c->k_heads * c->head;
    s.ld_out[0] = c->ldq_out ? c->ldq_out : c->q_heads * c->head;
    s.ld_out[1] = c->ldk_out ? c->ldk_out : c->k_heads * c->head;
    s.eps = c->eps;
    s.magnitude = c->magnitude;
    return s;
}

// Whether heads go by chunks of 16 bytes: halves of whole chunks, or rotated channels of whole chunks, and everything aligned.
bool wide(const tahq_heads_config *c, const HeadShape &s, std::initializer_list<const void *> tensors)
{
    const uint32_t chunk = 16 / esize(c);
    if (c->head % chunk || c->rotated % (c->layout == TAHQ_HEADS_PAIRS ? chunk : 2 * chunk)) return false;
    for (int i = 0; i < (c->k_heads ? 2 : 1); ++i)
        if (s.ld[i] % chunk || s.ld_out[i] % chunk) return false;
    for (const void *p : tensors)
        if (misaligned(p)) return false;
    return true;
}

// lanes to a head: two chunks, or four pairs, to each
uint32_t lanes_of(const tahq_heads_config *c, bool wide)
{
    const uint32_t chunk = 16 / esize(c), need = wide ? (c->head / chunk + 1) / 2 : ((c->head + 1) / 2 + 3) / 4;
    uint32_t lanes = 1;
    while (lanes < need) lanes *= 2;
    return lanes;
}

// Where tokens alone would leave vector units idle, each of a token's groups of heads has a wavefront of its own, which works out the token's angles again.
// bf16, 40 + 8 heads of 128: 512 tokens split 6.8 us forward and 12.6 backward, not split 8.1 and 13.5; 1024 8.4 and 15.4, 8.6 and 14.2; 2048 13.0 and 21.4, 11.7
// and 18.1; 4096 22.2 and 32.3, 18.5 and 26.6.
constexpr uint32_t kSplitBelow = 1024;

// groups of queries' (0) and of keys' heads (1) that a wavefront takes side by side
uint32_t groups_of(const HeadShape &s, int which)
{
    const uint32_t each = 64 / s.lanes;
    return (s.heads[which] + each - 1) / each;
}
// workgroups that give every wavefront one token, or one group, but so few that queries' and keys' together are a launch of less than 2^32 lanes
uint32_t workgroups_of(const HeadShape &s, uint32_t groups)
{
    const uint64_t all = ((uint64_t)s.tokens * (s.split ? groups : 1) + kHeadWaves - 1) / kHeadWaves;
    return (uint32_t)(all < (1u << 22) ? all : 1u << 22);
}

// Workgroups of the backward pass, queries' and keys'.  With norms each leaves a part of a weight's gradient, so there are no more than are at work at
// once: three to a compute unit of bf16 in chunks of 16 bytes, which has up to 144 registers (32768 x 48 x 128: 768 workgroups 250 us, 1024 311, and with 128
// registers, some of them in memory, 367), five of the others with up to 105 (fp32 2331 x 25 x 80: 768 17.6 us, 1280 16.1).
// They are shared as the work is, a token's angles counting as a group.
constexpr uint32_t kBackwardMost = 1280;
struct BackwardGroups {
    uint32_t queries, keys;
};
BackwardGroups backward_groups(const tahq_heads_config *c, const HeadShape &s, bool by_chunks)
{
    const uint32_t at_once = by_chunks && c->dtype == TAHQ_BF16 ? 768 : kBackwardMost;
    const uint32_t gq = groups_of(s, 0), gk = groups_of(s, 1);
    BackwardGroups g = {workgroups_of(s, gq), gk ? workgroups_of(s, gk) : 0};
    if (!c->norm || g.queries + g.keys <= at_once) return g;
    const uint32_t angles = s.split ? 0 : 1, all = gq + gk + 2 * angles;
    const uint32_t keys = gk ? (at_once * (gk + angles) + all / 2) / all : 0;
    const uint32_t least = keys < 1 && gk ? 1 : keys, most = least < at_once ? least : at_once - 1;
    if (g.keys > most) g.keys = most;
    if (g.queries > at_once - g.keys) g.queries = at_once - g.keys;
    return g;
}

// what a configuration's kernel is compiled for
template <typename Run>
void with_kind(const tahq_heads_config *c, bool wide, Run run)
{
    auto norm = [&](auto b, auto w, auto p) {
        if (c->norm) run(b, w, p, std::true_type{});
        else run(b, w, p, std::false_type{});
    };
    auto pairs = [&](auto b, auto w) {
        if (c->layout == TAHQ_HEADS_PAIRS) norm(b, w, std::true_type{});
        else norm(b, w, std::false_type{});
    };
    auto by = [&](auto b) {
        if (wide) pairs(b, std::true_type{});
        else pairs(b, std::false_type{});
    };
    if (c->dtype == TAHQ_BF16) by(std::true_type{});
    else by(std::false_type{});
}

// Elements' alignment for queries, keys and their like and for positions, 16 bytes for the rest
bool misplaced(const tahq_heads_config *c, const int64_t *positions, std::initializer_list<const void *> heads, std::initializer_list<const void *> others)
{
    if (reinterpret_cast<uintptr_t>(positions) % sizeof *positions) return true;
    for (const void *p : heads)
        if (reinterpret_cast<uintptr_t>(p) % esize(c)) return true;
    for (const void *p : others)
        if (misaligned(p)) return true;
    return false;
}

// NULL where a tensor is needed, a tensor where there is none
tahq_status given(const void *p, bool needed) { return needed == (p != nullptr) ? TAHQ_OK : needed ? TAHQ_ERR_NULL : TAHQ_ERR_INVALID_ARG; }
tahq_status all_given(std::initializer_list<std::pair<const void *, bool>> tensors)
{
    for (const auto &t : tensors)
        if (given(t.first, t.second) == TAHQ_ERR_NULL) return TAHQ_ERR_NULL;
    for (const auto &t : tensors)
        if (given(t.first, t.second) != TAHQ_OK) return TAHQ_ERR_INVALID_ARG;
    return TAHQ_OK;
}

}  // namespace

extern "C" {

void tahq_heads_config_default(tahq_heads_config *cfg)
{
    if (!cfg) return;
    *cfg = tahq_heads_config{};
    cfg->struct_size = (uint32_t)sizeof *cfg;
    cfg->dtype = TAHQ_BF16;
    cfg->norm = 1;
    cfg->eps = 1e-6f;
    cfg->magnitude = 1.0f;
}

void tahq_rotary_config_default(tahq_rotary_config *cfg)
{
    if (!cfg) return;
    *cfg = tahq_rotary_config{};
    cfg->struct_size = (uint32_t)sizeof *cfg;
    cfg->original = 4096;
    cfg->base = 10000.0;
    cfg->factor = 1.0;
    cfg->low = 1.0;
    cfg->high = 32.0;
}

tahq_status tahq_rotary_frequencies(const tahq_rotary_config *c, uint64_t *frequencies)
{
    if (!c || !frequencies) return TAHQ_ERR_NULL;
    if (c->struct_size != sizeof *c || c->rotated == 0 || c->rotated % 2 || c->scaling > TAHQ_ROTARY_PARTS) return TAHQ_ERR_INVALID_ARG;
    if (!(c->base > 0.0 && c->base < INFINITY) || !(c->factor > 0.0 && c->factor < INFINITY)) return TAHQ_ERR_INVALID_ARG;
    if (c->scaling == TAHQ_ROTARY_PARTS && (c->original == 0 || !(c->low < c->high) || !(c->low > -INFINITY) || !(c->high < INFINITY))) return TAHQ_ERR_INVALID_ARG;
    if (c->rotated > TAHQ_HEADS_MAX) return TAHQ_ERR_UNSUPPORTED;
    const long double turn = 6.283185307179586476925286766559005768L, all = 18446744073709551616.0L;
    const long double n = (long double)c->rotated, factor = (long double)c->factor;
    // a single pair's frequency is 1, whatever the base
    const long double base = c->scaling == TAHQ_ROTARY_STRETCHED && c->rotated > 2 ? (long double)c->base * powl(factor, n / (n - 2.0L)) : (long double)c->base;
    for (uint32_t i = 0; i < c->rotated / 2; ++i) {
        long double f = powl(base, -2.0L * (long double)i / n);
        if (c->scaling == TAHQ_ROTARY_LINEAR) f /= factor;
        if (c->scaling == TAHQ_ROTARY_PARTS) {
            long double k = ((long double)c->original * f / turn - (long double)c->low) / ((long double)c->high - (long double)c->low);
            k = k < 0.0L ? 0.0L : k > 1.0L ? 1.0L : k;
            f = k * f + (1.0L - k) * f / factor;
        }
        long double t = f / turn;
        if (!(t < INFINITY)) return TAHQ_ERR_INVALID_ARG;
        t -= floorl(t);
        const long double units = floorl(t * all + 0.5L);
        frequencies[i] = units >= all ? 0 : (uint64_t)units;
    }
    return TAHQ_OK;
}

tahq_status tahq_heads_forward(const tahq_heads_config *cfg, const void *d_q, const void *d_k, const void *d_w_q, const void *d_w_k,
                               const int64_t *d_positions, const uint64_t *d_frequencies, void *d_q_out, void *d_k_out, tahq_stream stream)
{
    tahq_status rc = check(cfg);
    if (rc != TAHQ_OK) return rc;
    const bool keys = cfg->k_heads != 0, norm = cfg->norm != 0, turned = cfg->rotated != 0;
    rc = all_given({{d_q, true}, {d_k, keys}, {d_w_q, norm}, {d_w_k, norm && keys}, {d_positions, turned}, {d_frequencies, turned},
                    {d_q_out, true}, {d_k_out, keys}});
    if (rc != TAHQ_OK) return rc;
    if (misplaced(cfg, d_positions, {d_q, d_k, d_q_out, d_k_out}, {d_w_q, d_w_k, d_frequencies})) return TAHQ_ERR_MISALIGNED;
    HeadShape s = shape_of(cfg);
    const bool by_chunks = wide(cfg, s, {d_q, d_k, d_q_out, d_k_out});
    s.lanes = lanes_of(cfg, by_chunks);
    s.split = cfg->tokens < kSplitBelow;
    Enqueue q{(hipStream_t)stream};
    with_kind(cfg, by_chunks, [&](auto bf16, auto w, auto pairs, auto normed) {
        q(k_heads_forward<bf16, w, pairs, normed>, dim3(workgroups_of(s, groups_of(s, 0) + groups_of(s, 1))), dim3(64 * kHeadWaves), HeadTensors{{d_q, d_k}}, HeadTensors{{d_w_q, d_w_k}}, d_positions,
          d_frequencies, HeadOutputs{{d_q_out, d_k_out}}, s);
    });
    return q.result();
}

size_t tahq_heads_workspace_size(const tahq_heads_config *cfg)
{
    return check(cfg) == TAHQ_OK && cfg->norm ? (size_t)kBackwardMost * cfg->head * sizeof(float) : 0;
}

tahq_status tahq_heads_backward(const tahq_heads_config *cfg, const void *d_grad_q_out, const void *d_grad_k_out, const void *d_q,
                                const void *d_k, const void *d_w_q, const void *d_w_k, const int64_t *d_positions,
                                const uint64_t *d_frequencies, void *d_grad_q, void *d_grad_k, float *d_grad_w_q, float *d_grad_w_k,
                                void *d_workspace, size_t workspace_capacity, tahq_stream stream)
{
    tahq_status rc = check(cfg);
    if (rc != TAHQ_OK) return rc;
    const bool keys = cfg->k_heads != 0, norm = cfg->norm != 0, turned = cfg->rotated != 0;
    rc = all_given({{d_grad_q_out, true}, {d_grad_k_out, keys}, {d_q, norm}, {d_k, norm && keys}, {d_w_q, norm}, {d_w_k, norm && keys},
                    {d_positions, turned}, {d_frequencies, turned}, {d_grad_q, true}, {d_grad_k, keys}, {d_grad_w_q, norm}, {d_grad_w_k, norm && keys}});
    if (rc != TAHQ_OK) return rc;
    if (norm && !d_workspace) return TAHQ_ERR_NULL;
    if (workspace_capacity < tahq_heads_workspace_size(cfg)) return TAHQ_ERR_WORKSPACE_TOO_SMALL;
    if (misplaced(cfg, d_positions, {d_grad_q_out, d_grad_k_out, d_q, d_k, d_grad_q, d_grad_k},
                  {d_w_q, d_w_k, d_frequencies, d_grad_w_q, d_grad_w_k, norm ? d_workspace : nullptr}))
        return TAHQ_ERR_MISALIGNED;
    HeadShape s = shape_of(cfg);
    const bool by_chunks = wide(cfg, s, {d_grad_q_out, d_grad_k_out, d_q, d_k, d_grad_q, d_grad_k});
    s.lanes = lanes_of(cfg, by_chunks);
    s.split = cfg->tokens < kSplitBelow;
    const BackwardGroups g = backward_groups(cfg, s, by_chunks);
    float *parts = static_cast<float *>(d_workspace);
    Enqueue q{(hipStream_t)stream};
    with_kind(cfg, by_chunks, [&](auto bf16, auto w, auto pairs, auto normed) {
        q(k_heads_backward<bf16, w, pairs, normed>, dim3(g.queries + g.keys), dim3(64 * kHeadWaves), HeadTensors{{d_grad_q_out, d_grad_k_out}}, HeadTensors{{d_q, d_k}},
          HeadTensors{{d_w_q, d_w_k}}, d_positions, d_frequencies, HeadOutputs{{d_grad_q, d_grad_k}}, parts, g.queries, s);
    });
    if (norm) q(k_heads_reduce, dim3((cfg->head + 15) / 16, keys ? 2 : 1), dim3(1024), parts, d_grad_w_q, d_grad_w_k, cfg->head, g.queries, g.queries + g.keys, cfg->accumulate);
    return q.result();
}

}  // extern "C"
