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

// Channels of a chunk: the most, up to 16 bytes, that halves, or pairs, are whole ones of; 1 where there are none.  Alignment does not matter for that.
int chunk_of(const tahq_heads_config *c)
{
    for (uint32_t chunk = 16 / esize(c); chunk > 1; chunk /= 2)
        if (c->head % chunk == 0 && c->rotated % (c->layout == TAHQ_HEADS_PAIRS ? chunk : 2 * chunk) == 0 && c->head <= 128 * chunk) return (int)chunk;
    return 1;
}

// lanes to a head: two chunks, or four pairs, to each
uint32_t lanes_of(const tahq_heads_config *c, uint32_t chunk)
{
    const uint32_t need = chunk > 1 ? (c->head / chunk + 1) / 2 : ((c->head + 1) / 2 + 3) / 4;
    uint32_t lanes = 1;
    while (lanes < need) lanes *= 2;
    return lanes;
}

// Where tokens alone would leave vector units idle, each of a token's groups of heads has a wavefront of its own, which works out the token's angles again.
// bf16, 40 + 8 heads of 128: 512 tokens split 6.8 us forward and 12.6 backward, not split 8.1 and 13.5; 1024 8.4 and 15.4, 8.6 and 14.2; 2048 13.0 and
// 21.4, 11.7 and 18.1; 4096 22.2 and 32.3, 18.5 and 26.6.
constexpr uint32_t kSplitBelow = 1024;

// groups of `heads` heads that a wavefront takes side by side
uint32_t groups_of(const HeadShape &s, uint32_t heads)
{
    const uint32_t each = 64 / s.lanes;
    return (heads + each - 1) / each;
}
// tokens whose heads a wavefront takes side by side
uint32_t side_of(const HeadShape &s, uint32_t heads) { return 64 / s.lanes / heads > 1 ? 64 / s.lanes / heads : 1; }
// workgroups that give every wavefront one token, or one group, or a group of several tokens, but so few that queries' and keys' together are a launch
// of less than 2^32 lanes
uint32_t workgroups_of(const HeadShape &s, uint32_t heads)
{
    if (heads == 0) return 0;
    const uint32_t side = side_of(s, heads), groups = groups_of(s, heads);
    const uint64_t all = (((uint64_t)s.tokens + side - 1) / side * (s.split ? groups : 1) + kHeadWaves - 1) / kHeadWaves;
    return (uint32_t)(all < (1u << 22) ? all : 1u << 22);
}

// Workgroups of the backward pass, queries' and keys'.  With norms each leaves a part of a weight's gradient, so there are no more than are at work at once
// (bf16 32768 x 48 x 128, three to a compute unit: 768 245 us, 1024 311; fp32 2331 x 25 x 80, five: 768 17.6 us, 1024 16.4, 1280 16.1; bf16 7432 x 40 x 58,
// four: 1024 72 us, 1280 85).  They are shared as the work is, a token's angles counting as a group.
constexpr uint32_t kBackwardMost = 1280;
struct BackwardGroups {
    uint32_t queries, keys;
};
BackwardGroups backward_groups(const tahq_heads_config *c, const HeadShape &s, int chunk)
{
    const uint32_t at_once = 256 * backward_per_cu(c->dtype == TAHQ_BF16, chunk, c->layout == TAHQ_HEADS_PAIRS);
    const uint32_t gq = groups_of(s, c->q_heads), gk = groups_of(s, c->k_heads);
    BackwardGroups g = {workgroups_of(s, c->q_heads), workgroups_of(s, c->k_heads)};
    if (!c->norm || g.queries + g.keys <= at_once) return g;
    // of a token, in fractions of a group where a group has several tokens
    auto work = [&](uint32_t heads, uint32_t groups) { return heads ? (groups + (s.split ? 0.0 : 1.0)) / side_of(s, heads) : 0.0; };
    const double wq = work(c->q_heads, gq), wk = work(c->k_heads, gk);
    const uint32_t keys = (uint32_t)(at_once * wk / (wq + wk) + 0.5);
    const uint32_t least = keys < 1 && gk ? 1 : keys, most = least < at_once ? least : at_once - 1;
    if (g.keys > most) g.keys = most;
    if (g.queries > at_once - g.keys) g.queries = at_once - g.keys;
    return g;
}

// what a configuration's kernel is compiled for
template <typename Run>
void with_kind(const tahq_heads_config *c, int chunk, Run run)
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
        if (chunk == 4) pairs(b, std::integral_constant<int, 4>{});
        else if (chunk == 2) pairs(b, std::integral_constant<int, 2>{});
        else pairs(b, std::integral_constant<int, 1>{});
    };
    if (c->dtype != TAHQ_BF16) by(std::false_type{});
    else if (chunk == 8) pairs(std::true_type{}, std::integral_constant<int, 8>{});
    else by(std::true_type{});
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
    const int chunk = chunk_of(cfg);
    s.lanes = lanes_of(cfg, chunk);
    s.split = cfg->tokens < kSplitBelow;
    Enqueue q{(hipStream_t)stream};
    with_kind(cfg, chunk, [&](auto bf16, auto w, auto pairs, auto normed) {
        q(k_heads_forward<bf16, w, pairs, normed>, dim3(workgroups_of(s, cfg->q_heads + cfg->k_heads)), dim3(64 * kHeadWaves), HeadTensors{{d_q, d_k}}, HeadTensors{{d_w_q, d_w_k}}, d_positions,
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
    const int chunk = chunk_of(cfg);
    s.lanes = lanes_of(cfg, chunk);
    s.split = cfg->tokens < kSplitBelow;
    const BackwardGroups g = backward_groups(cfg, s, chunk);
    float *parts = static_cast<float *>(d_workspace);
    Enqueue q{(hipStream_t)stream};
    with_kind(cfg, chunk, [&](auto bf16, auto w, auto pairs, auto normed) {
        q(k_heads_backward<bf16, w, pairs, normed>, dim3(g.queries + g.keys), dim3(64 * kHeadWaves), HeadTensors{{d_grad_q_out, d_grad_k_out}}, HeadTensors{{d_q, d_k}},
          HeadTensors{{d_w_q, d_w_k}}, d_positions, d_frequencies, HeadOutputs{{d_grad_q, d_grad_k}}, parts, g.queries, s);
    });
    if (norm) q(k_heads_reduce, dim3((cfg->head + 15) / 16, keys ? 2 : 1), dim3(1024), parts, d_grad_w_q, d_grad_w_k, cfg->head, g.queries, g.queries + g.keys, cfg->accumulate);
    return q.result();
}

}  // extern "C"
