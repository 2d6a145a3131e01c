// Entry points of the block norms (include/tahq_norm.h): validation, plan, launches.
#include <type_traits>

#include "tahq_enqueue.hpp"
#include "tahq_norm.h"
#include "tahq_norm_kernels.hpp"

using namespace tahq;

namespace {

tahq_status check(const tahq_norm_config *c)
{
    if (!c) return TAHQ_ERR_NULL;
    if (c->struct_size != sizeof *c) return TAHQ_ERR_INVALID_ARG;
    if (c->rows == 0 || c->rows >= 0x80000000u || c->cols == 0 || c->dtype > TAHQ_BF16) return TAHQ_ERR_INVALID_ARG;
    if (!(c->eps > 0.0f) || !(c->eps <= 3.4028234663852886e38f)) return TAHQ_ERR_INVALID_ARG;
    if (!(__builtin_fabsf(c->residual_scale) <= 3.4028234663852886e38f)) return TAHQ_ERR_INVALID_ARG;
    if (c->accumulate > 1 || c->transform > 1 || c->scale_rule > TAHQ_MX4_COVER) return TAHQ_ERR_INVALID_ARG;
    if (c->cols > TAHQ_NORM_MAX_COLS) return TAHQ_ERR_UNSUPPORTED;
    return TAHQ_OK;
}

// wavefronts of a row: eight channels to a lane
uint32_t waves_of(const tahq_norm_config *c) { return (c->cols + 511) / 512; }

NormShape shape_of(const tahq_norm_config *c)
{
    // a gate row for more tokens than there are is one for all of them
    return {c->rows, c->cols, c->gate_rows < c->rows ? c->gate_rows : c->rows, waves_of(c), c->eps, c->residual_scale};
}

// the kernels' template parameters from a configuration and the halves that there are
template <bool BF16, bool EIGHTS, typename Run>
void with_halves(bool post, bool pre, Run run)
{
    const std::bool_constant<BF16> b;
    const std::bool_constant<EIGHTS> e;
    if (post && pre) run(b, e, std::true_type{}, std::true_type{});
    else if (post) run(b, e, std::true_type{}, std::false_type{});
    else if (pre) run(b, e, std::false_type{}, std::true_type{});
    else run(b, e, std::false_type{}, std::false_type{});
}
template <typename Run>
void with_kind(const tahq_norm_config *c, bool post, bool pre, Run run)
{
    const bool eights = c->cols % 8 == 0;
    if (c->dtype == TAHQ_BF16) eights ? with_halves<true, true>(post, pre, run) : with_halves<true, false>(post, pre, run);
    else eights ? with_halves<false, true>(post, pre, run) : with_halves<false, false>(post, pre, run);
}

// Forward: rows that a workgroup takes one after another.  Two where there are many (8192 x 4096, one row: 45 us, two: 42.7, eight:
// 47); eight where a workgroup of more than twelve wavefronts has a compute unit to itself and only the next row on its way keeps
// memory busy (2048 x 8192: one 36, two 31, eight 28); one where there are few.  From 2^27 rows on (of few channels) as many more as a
// launch's 2^32 lanes ask for.
uint32_t forward_rows(const tahq_norm_config *c, uint32_t rows)
{
    uint32_t each = waves_of(c) > 12 ? (rows >= 2048 ? 8 : 1) : rows >= 4096 ? 2 : 1;
    while (!launchable((rows - 1) / each + 1, 64 * waves_of(c))) each *= 2;
    return each;
}

// Backward: the workgroups that share the rows.  A compute unit holds sixteen wavefronts of up to 128 registers, so `most` workgroups
// at once; more than one round of workgroups of unlike length costs more than it gives (rows side by side: 32768 x 5120, ten
// wavefronts: 256 workgroups 455 us, 409 534, 512 458; 32768 x 1024, two: 512 152, 1024 111, 2048 101).  What counts below that, in
// rows of a compute unit: the rows of the unit with most of them, a third of a workgroup's rows, which nobody hides, and a row for
// every 256 workgroups, whose column sums are added afterwards.  Both kernels, fp32 with one row of a gate, by a workgroup's rows: 777
// x 1600 one 20.7 us, four 15.3; 4096 x 1600 four 35.6, eight 31.2, sixteen 33.3; 2331 x 1600 five 22.3, ten 23.7.
struct BackwardPlan {
    uint32_t rows_each, workgroups;
    uint64_t workspace;
};
BackwardPlan plan_backward(const tahq_norm_config *c)
{
    BackwardPlan p;
    const uint32_t most = waves_of(c) > 1 ? 16 / waves_of(c) : 8;          // of one wavefront eight: 32768 x 512, 2048 in all 47 us, 4096 71
    float least = 0.0f;
    p.rows_each = 0;
    for (uint32_t k = most; k > 0; --k) {
        const uint32_t each = (uint32_t)(((uint64_t)c->rows + 256 * k - 1) / (256 * k)), workgroups = (uint32_t)(((uint64_t)c->rows + each - 1) / each);
        const float cost = (float)each * ((float)((workgroups + 255) / 256) + 0.3f) + (float)workgroups / 256;
        if (!p.rows_each || cost < least) {
            least = cost;
            p.rows_each = each;
        }
    }
    p.workgroups = (c->rows + p.rows_each - 1) / p.rows_each;
    p.workspace = (uint64_t)p.workgroups * c->cols * 4 * (c->gate_rows ? 4 : 2);
    return p;
}
// Workgroups that take the rows of a span in turn: where the six tensors are larger than the last cache, as many as the gate allows.  In turn and
// side by side: 32768 x 5120 bf16 378 us and 441, 16384 x 1600 57 and 67, 8192 x 4096 fp32 147 and 160 (but 2048 x 8192 with four rows of a gate 95
// and 87); of 100 MB, 8192 x 1024 bf16, 20.6 and 18.9, with four rows of a gate 24.6 and 20.2.
uint32_t backward_team(const tahq_norm_config *c, const BackwardPlan &p, uint32_t gate_rows)
{
    if ((uint64_t)c->rows * c->cols * (c->dtype == TAHQ_BF16 ? 12 : 24) < (256u << 20)) return 1;
    const uint32_t most = gate_rows / p.rows_each;
    return gate_rows == c->rows || most > p.workgroups ? p.workgroups : most ? most : 1;
}

}  // namespace

extern "C" {

void tahq_norm_config_default(tahq_norm_config *cfg)
{
    if (!cfg) return;
    *cfg = tahq_norm_config{};
    cfg->struct_size = (uint32_t)sizeof *cfg;
    cfg->dtype = TAHQ_BF16;
    cfg->eps = 1e-6f;
    cfg->residual_scale = 1.0f;
}

tahq_status tahq_norm_forward(const tahq_norm_config *cfg, const void *d_residual, const void *d_block, const void *d_w_post,
                              const void *d_gate, const void *d_w_pre, void *d_residual_out, void *d_h, void *d_h_mx4,
                              size_t h_mx4_capacity, float *d_stats, tahq_stream stream)
{
    const tahq_status rc = check(cfg);
    if (rc != TAHQ_OK) return rc;
    if (!d_residual) return TAHQ_ERR_NULL;
    if (d_block) {
        if (!d_w_post || !d_residual_out || (cfg->gate_rows && !d_gate)) return TAHQ_ERR_NULL;
        if (!cfg->gate_rows && d_gate) return TAHQ_ERR_INVALID_ARG;
    } else if (d_w_post || d_gate) {
        return TAHQ_ERR_INVALID_ARG;
    }
    if (d_w_pre) {
        if (!d_h && !d_h_mx4) return TAHQ_ERR_NULL;
    } else {
        if (d_h || d_h_mx4) return TAHQ_ERR_INVALID_ARG;
        if (!d_residual_out) return TAHQ_ERR_NULL;
    }
    if (d_h_mx4 && h_mx4_capacity < tahq_mx4_packed_size(cfg->rows, cfg->cols)) return TAHQ_ERR_BUFFER_TOO_SMALL;
    for (const void *p : {d_residual, d_block, d_w_post, d_gate, d_w_pre, (const void *)d_residual_out, (const void *)d_h, (const void *)d_h_mx4, (const void *)d_stats})
        if (misaligned(p)) return TAHQ_ERR_MISALIGNED;
    const NormShape s = shape_of(cfg);
    const uint32_t cover = cfg->scale_rule == TAHQ_MX4_COVER ? kCover : 0u;
    const uint32_t total = d_h_mx4 ? 32 * ((cfg->rows + 31) / 32) : cfg->rows;
    const uint32_t rows_each = forward_rows(cfg, total), together = rows_each <= 32 ? 256 / rows_each : 1;
    const dim3 grid((total - 1) / rows_each + 1);
    Enqueue q{(hipStream_t)stream};
    with_kind(cfg, d_block, d_w_pre, [&](auto bf16, auto eights, auto post, auto pre) {
        q(k_norm_forward<bf16, eights, post, pre>, grid, dim3(64 * waves_of(cfg)), d_residual, d_block, d_w_post, d_block ? d_gate : nullptr, d_w_pre, d_residual_out, d_h,
          static_cast<uint8_t *>(d_h_mx4), d_stats, s, cover, cfg->transform, rows_each, together);
    });
    return q.result();
}

size_t tahq_norm_workspace_size(const tahq_norm_config *cfg)
{
    return check(cfg) == TAHQ_OK ? (size_t)plan_backward(cfg).workspace : 0;
}

tahq_status tahq_norm_backward(const tahq_norm_config *cfg, const void *d_grad_residual_out, const void *d_grad_h,
                               const void *d_block, const void *d_w_post, const void *d_gate, const void *d_residual_out,
                               const void *d_w_pre, const float *d_stats, void *d_grad_residual, void *d_grad_block,
                               float *d_grad_w_post, float *d_grad_gate, float *d_grad_w_pre, void *d_workspace,
                               size_t workspace_capacity, tahq_stream stream)
{
    const tahq_status rc = check(cfg);
    if (rc != TAHQ_OK) return rc;
    if (!d_grad_residual || !d_workspace || (!d_grad_residual_out && !d_grad_h)) return TAHQ_ERR_NULL;
    if ((d_block || d_grad_h) && !d_stats) return TAHQ_ERR_NULL;
    if (d_block) {
        if (!d_w_post || !d_grad_block || !d_grad_w_post) return TAHQ_ERR_NULL;
        if (cfg->gate_rows ? !d_gate || !d_grad_gate : false) return TAHQ_ERR_NULL;
        if (!cfg->gate_rows && (d_gate || d_grad_gate)) return TAHQ_ERR_INVALID_ARG;
    } else if (d_w_post || d_gate || d_grad_block || d_grad_w_post || d_grad_gate) {
        return TAHQ_ERR_INVALID_ARG;
    }
    if (d_grad_h) {
        if (!d_w_pre || !d_residual_out || !d_grad_w_pre) return TAHQ_ERR_NULL;
    } else if (d_w_pre || d_grad_w_pre) {
        return TAHQ_ERR_INVALID_ARG;
    }
    const BackwardPlan p = plan_backward(cfg);
    if (workspace_capacity < p.workspace) return TAHQ_ERR_WORKSPACE_TOO_SMALL;
    for (const void *x : {d_grad_residual_out, d_grad_h, d_block, d_w_post, d_gate, d_residual_out, d_w_pre, (const void *)d_stats,
                          (const void *)d_grad_residual, (const void *)d_grad_block, (const void *)d_grad_w_post,
                          (const void *)d_grad_gate, (const void *)d_grad_w_pre, (const void *)d_workspace})
        if (misaligned(x)) return TAHQ_ERR_MISALIGNED;
    const NormShape s = shape_of(cfg);
    const uint64_t each = (uint64_t)p.workgroups * cfg->cols;
    float *ws = static_cast<float *>(d_workspace);
    const NormPartials parts = {ws, ws + each, ws + 2 * each};
    const void *gate = d_block ? d_gate : nullptr;
    const uint32_t team = backward_team(cfg, p, gate ? s.gate_rows : cfg->rows);
    Enqueue q{(hipStream_t)stream};
    with_kind(cfg, d_block, d_grad_h, [&](auto bf16, auto eights, auto post, auto pre) {
        q(k_norm_backward<bf16, eights, post, pre>, dim3(p.workgroups), dim3(64 * waves_of(cfg)), d_grad_residual_out, d_grad_h, d_block, d_w_post, gate, d_residual_out, d_w_pre,
          d_stats, d_grad_residual, d_grad_block, d_grad_gate, parts, s, p.rows_each, team, cfg->accumulate);
    });
    const uint32_t groups = gate ? (cfg->rows + s.gate_rows - 1) / s.gate_rows : 0;
    if (d_block || d_grad_h) {
        const uint32_t slots = groups < 64 ? groups : 64;
        const uint32_t width = cfg->cols <= 2048 ? 16 : 64;
        q(k_norm_reduce, dim3((cfg->cols + width - 1) / width, 2 + slots), dim3(kReduceLanes), parts, d_grad_w_post, d_grad_w_pre, d_grad_gate, cfg->cols,
          p.workgroups, cfg->rows, s.gate_rows, p.rows_each, team, groups, cfg->accumulate, width);
    }
    return q.result();
}

}  // extern "C"
