// Entry points of the loss over a vocabulary (include/tahq_loss.h): validation, plan, launches.
#include "tahq_enqueue.hpp"
#include "tahq_loss.h"
#include "tahq_loss_kernels.hpp"
#include "tahq_loss_plan.hpp"

using namespace tahq;

namespace {

tahq_status check(const tahq_loss_config *c)
{
    if (!c) return TAHQ_ERR_NULL;
    if (c->struct_size != sizeof *c) return TAHQ_ERR_INVALID_ARG;
    if (c->rows == 0 || c->rows >= 0x80000000u || c->vocab == 0 || c->vocab >= 0x80000000u || c->cols == 0) return TAHQ_ERR_INVALID_ARG;
    if (c->dtype > TAHQ_BF16 || c->weight_dtype > TAHQ_BF16 || c->reduction > TAHQ_LOSS_MEAN || c->accumulate > 1) return TAHQ_ERR_INVALID_ARG;
    if (c->cols > TAHQ_LOSS_MAX_COLS || c->rows > TAHQ_LOSS_MAX_ROWS) return TAHQ_ERR_UNSUPPORTED;
    for (const bool backward : {false, true}) {
        const LossPlan p = plan_loss(c, backward);
        if (!launchable(loss_tiles(p.kind, c->rows, p.piece), 256) || !launchable(p.x_groups, 256) || !launchable(loss_tiles(kLossMiddle, p.piece, c->cols), 256))
            return TAHQ_ERR_UNSUPPORTED;
    }
    return TAHQ_OK;
}

struct Call {
    const tahq_loss_config *cfg;
    LossPlan p;
    uint8_t *ws;
    Enqueue q;
    LossTokens tokens;

    Call(const tahq_loss_config *c, bool backward, void *workspace, tahq_stream stream)
        : cfg(c), p(plan_loss(c, backward)), ws(static_cast<uint8_t *>(workspace)), q{(hipStream_t)stream},
          tokens{at<uint32_t>(p.rows), at<uint32_t>(p.targets), at<uint32_t>(0)} {}
    template <typename T>
    T *at(uint64_t place) const { return reinterpret_cast<T *>(ws + place); }

    void gather(const void *d_x, const int64_t *d_target, float *zero, float *zero_also, void *grad_x)
    {
        uint32_t *counts = p.spans > 1 ? at<uint32_t>(p.counts) : nullptr;
        if (counts) q(k_loss_count, dim3(p.spans), dim3(1024), d_target, cfg->ignore, cfg->rows, counts);
        q(p.bf16 ? k_loss_gather<true, 1> : p.planes ? k_loss_gather<false, 3> : k_loss_gather<false, 1>, dim3((uint32_t)loss_ceil(cfg->rows, kGatherRows)), dim3(256), d_x, d_target,
          counts, cfg->rows, cfg->cols, cfg->vocab, cfg->ignore, at<uint8_t>(p.x), p.blocks, p.padded, tokens, zero, zero_also, grad_x);
    }
    // Rows of the weight as the tiles take them: the first one's address, bytes from row to row or from block to block, and from plane to plane
    struct Weight {
        const uint8_t *from;
        uint64_t ld, plane;
    };
    Weight weight(const void *d_weight, uint32_t first, uint32_t rows)
    {
        const uint64_t row = (uint64_t)cfg->cols * (p.bf16 ? 2 : 4);
        const uint8_t *from = static_cast<const uint8_t *>(d_weight) + first * row;
        if (!p.copy) return {from, row, 0};
        const uint32_t padded = (uint32_t)loss_ceil(rows, p.whole) * p.whole, sixteens = (uint32_t)loss_ceil(padded, 16);
        // few rows: several workgroups to sixteen of them, up to 2048 in all (1699 x 3070 x 2157 forward 55 -> 50 us, 21 x 7999 x 50257 637 -> 604)
        const uint32_t most = (uint32_t)loss_ceil(p.blocks, 4), share = sixteens < 2048 ? 2048 / sixteens : 1;
        q(p.bf16 ? k_loss_blocks<true, 1> : p.planes ? k_loss_blocks<false, 3> : k_loss_blocks<false, 1>, dim3(sixteens, share < most ? share : most), dim3(256), from, at<uint8_t>(p.weight),
          rows, cfg->cols, padded);
        return {at<uint8_t>(p.weight), (uint64_t)padded * 64, (uint64_t)padded * 64 * p.blocks};
    }
    template <int MODE, Lies LIES>
    void logits_of(const LogitArgs &g)
    {
        const dim3 grid((uint32_t)(loss_ceil(cfg->rows, kLossTiles[p.kind].tm) * g.tiles_n)), block(256);
        if (p.kind == kLossLarge) q(k_loss_logits<true, 1, 2, 2, 4, 4, 1, LIES, MODE>, grid, block, g);
        else if (p.kind == kLossMiddle) p.bf16 ? q(k_loss_logits<true, 1, 2, 2, 2, 2, 2, LIES, MODE>, grid, block, g) : q(k_loss_logits<false, 1, 2, 2, 2, 2, 2, LIES, MODE>, grid, block, g);
        else if (!p.bf16) q(k_loss_logits<false, 1, 1, 4, 1, 1, 2, LIES, MODE>, grid, block, g);
        else if constexpr (MODE == kGrads || LIES == kRows) q(k_loss_logits<true, 1, 1, 4, 1, 1, 2, LIES, MODE>, grid, block, g);       // otherwise: few
    }
    template <int MODE>
    void logits(const LogitArgs &g)
    {
        if (p.planes) {
            const dim3 grid((uint32_t)(loss_ceil(cfg->rows, kLossTiles[p.kind].tm) * g.tiles_n)), block(256);
            if (p.kind == kLossLarge) q(k_loss_logits<true, 3, 2, 2, 4, 4, 1, kBlocks, MODE>, grid, block, g);
            else q(k_loss_logits<true, 3, 2, 2, 2, 2, 2, kBlocks, MODE>, grid, block, g);
        } else if (p.copy) {
            logits_of<MODE, kBlocks>(g);
        } else {
            logits_of<MODE, kRows>(g);
        }
    }
    void few(const FewArgs &g)
    {
        const dim3 grid((uint32_t)loss_ceil(g.end - g.first, 32));
        if (p.split) q(p.bf16 ? k_loss_few<true, kFewWaves> : k_loss_few<false, kFewWaves>, grid, dim3(64 * kFewWaves), g);
        else q(p.bf16 ? k_loss_few<true, 1> : k_loss_few<false, 1>, grid, dim3(64), g);
    }
    LogitArgs logit_args(const Weight &w, uint32_t first, uint32_t rows) const
    {
        LogitArgs g = {};
        g.x = at<uint8_t>(p.x);
        g.weight = w.from;
        g.ldw = w.ld;
        g.x_plane = p.x_plane;
        g.w_plane = w.plane;
        g.g_plane = p.g_plane;
        g.tokens = tokens;
        g.stages = p.blocks;
        g.first = first;
        g.vocab = first + rows;
        g.tiles_n = (uint32_t)loss_ceil(rows, kLossTiles[p.kind].tn);
        g.padded = p.padded;
        return g;
    }
    template <Lies LIES>
    void grad_x_of(const GradXArgs &g)
    {
        const dim3 grid((uint32_t)p.x_groups), block(256);
        if (p.x_kind == kLossLarge) q(k_loss_grad_x<true, 1, 2, 2, 4, 4, 1, LIES>, grid, block, g);
        else if (p.x_kind == kLossMiddle) p.bf16 ? q(k_loss_grad_x<true, 1, 2, 2, 2, 2, 2, LIES>, grid, block, g) : q(k_loss_grad_x<false, 1, 2, 2, 2, 2, 2, LIES>, grid, block, g);
        else p.bf16 ? q(k_loss_grad_x<true, 1, 1, 4, 1, 1, 3, LIES>, grid, block, g) : q(k_loss_grad_x<false, 1, 1, 4, 1, 1, 3, LIES>, grid, block, g);
    }
    void grad_x(const GradXArgs &g)
    {
        const dim3 grid((uint32_t)p.x_groups), block(256);
        if (p.planes) p.x_kind == kLossLarge ? q(k_loss_grad_x<true, 3, 2, 2, 4, 4, 1, kBlocksTurned>, grid, block, g) : q(k_loss_grad_x<true, 3, 2, 2, 2, 2, 2, kBlocksTurned>, grid, block, g);
        else if (p.copy) grad_x_of<kBlocksTurned>(g);
        else grad_x_of<kTurned>(g);
    }
    void grad_w(GradWArgs g)
    {
        // sums run after run are added up in the gradient itself, if that is of fp32
        const bool chain = p.planes && g.out_bf16 && cfg->rows > kPlanesChain * p.whole;
        const int kind = p.es == 2 && !chain && loss_large(g.rows, g.cols) ? kLossLarge : kLossMiddle;
        g.tiles_m = (uint32_t)loss_ceil(g.rows, kLossTiles[kind].tm);
        g.tiles_n = (uint32_t)loss_ceil(g.cols, kLossTiles[kind].tn);
        const dim3 grid(g.tiles_m * g.tiles_n), block(256);
        if (p.planes) kind == kLossLarge ? q(k_loss_grad_w<true, 3, 2, 2, 4, 4, 1>, grid, block, g) : q(k_loss_grad_w<true, 3, 2, 2, 2, 2, 2>, grid, block, g);
        else if (kind == kLossLarge) q(k_loss_grad_w<true, 1, 2, 2, 4, 4, 1>, grid, block, g);
        else p.bf16 ? q(k_loss_grad_w<true, 1, 2, 2, 2, 2, 2>, grid, block, g) : q(k_loss_grad_w<false, 1, 2, 2, 2, 2, 2>, grid, block, g);
    }
};

}  // namespace

extern "C" {

void tahq_loss_config_default(tahq_loss_config *cfg)
{
    if (!cfg) return;
    *cfg = tahq_loss_config{};
    cfg->struct_size = (uint32_t)sizeof *cfg;
    cfg->dtype = cfg->weight_dtype = TAHQ_BF16;
    cfg->reduction = TAHQ_LOSS_MEAN;
    cfg->ignore = -100;
}

size_t tahq_loss_forward_workspace_size(const tahq_loss_config *cfg) { return check(cfg) == TAHQ_OK ? (size_t)plan_loss(cfg, false).total : 0; }
size_t tahq_loss_backward_workspace_size(const tahq_loss_config *cfg) { return check(cfg) == TAHQ_OK ? (size_t)plan_loss(cfg, true).total : 0; }

tahq_status tahq_loss_forward(const tahq_loss_config *cfg, const void *d_x, const void *d_weight, const int64_t *d_target, float *d_losses,
                              float *d_lse, float *d_total, void *d_workspace, size_t workspace_capacity, tahq_stream stream)
{
    const tahq_status rc = check(cfg);
    if (rc != TAHQ_OK) return rc;
    for (const void *p : {d_x, d_weight, (const void *)d_target, (const void *)d_losses, (const void *)d_lse, (const void *)d_total, (const void *)d_workspace})
        if (!p) return TAHQ_ERR_NULL;
    Call call(cfg, false, d_workspace, stream);
    const LossPlan &p = call.p;
    if (workspace_capacity < p.total) return TAHQ_ERR_WORKSPACE_TOO_SMALL;
    for (const void *x : {d_x, d_weight, (const void *)d_losses, (const void *)d_lse, (const void *)d_total, (const void *)d_workspace})
        if (misaligned(x)) return TAHQ_ERR_MISALIGNED;
    if (reinterpret_cast<uintptr_t>(d_target) % sizeof *d_target) return TAHQ_ERR_MISALIGNED;
    if (!p.few) call.gather(d_x, d_target, d_losses, d_lse, nullptr);
    // Tokens of a workgroup that joins statistics: up to 32 in one, then 64 workgroups and more, as a workgroup reads lines of 32 bytes of 4 tokens, and
    // each compute unit works on two (vocabulary of 50257: 256 workgroups and more, 500 tokens 37 us, 64 34; 1024 workgroups, 2048 tokens 91 us, 64 and 256
    // 83).
    uint32_t width = 32;
    while (width > 1 && (cfg->rows <= 32 ? cfg->rows <= width / 2 : cfg->rows < 64 * width)) width /= 2;
    const bool alone = cfg->rows <= width;
    for (uint32_t first = 0; first < cfg->vocab; first += p.piece) {
        const uint32_t rows = cfg->vocab - first < p.piece ? cfg->vocab - first : p.piece;
        float2 *const parts = call.at<float2>(p.stats);
        float *const at_target = call.at<float>(p.at_target);
        if (p.few) {
            call.few({d_x, static_cast<const uint8_t *>(d_weight) + (uint64_t)first * cfg->cols * p.es, d_target, cfg->ignore, cfg->rows, cfg->cols, first, first + rows, cfg->vocab,
                      p.padded, call.tokens, parts, at_target, d_losses, d_lse});
        } else {
            LogitArgs g = call.logit_args(call.weight(d_weight, first, rows), first, rows);
            g.parts = parts;
            g.at_target = at_target;
            call.logits<kStats>(g);
        }
        const uint32_t count = (uint32_t)loss_ceil(rows, kLossTiles[p.kind].tn) * kLossTiles[p.kind].along;
        call.q(k_loss_join, dim3((uint32_t)loss_ceil(cfg->rows, width)), dim3(kJoinLanes), parts, p.few ? (uint32_t)loss_ceil(rows, 32) : count, p.padded, call.tokens, at_target,
               call.at<float2>(p.running), first != 0, first + rows == cfg->vocab, width, d_losses, d_lse, cfg->reduction == TAHQ_LOSS_MEAN,
               alone && first + rows == cfg->vocab ? d_total : nullptr);
    }
    if (!alone) call.q(k_loss_total, dim3(1), dim3(kJoinLanes), d_losses, cfg->rows, call.tokens, cfg->reduction == TAHQ_LOSS_MEAN, d_total);
    return call.q.result();
}

tahq_status tahq_loss_backward(const tahq_loss_config *cfg, const void *d_x, const void *d_weight, const int64_t *d_target, const float *d_lse,
                               const float *d_grad_loss, void *d_grad_x, void *d_grad_weight, void *d_workspace, size_t workspace_capacity,
                               tahq_stream stream)
{
    const tahq_status rc = check(cfg);
    if (rc != TAHQ_OK) return rc;
    if (!d_grad_x && !d_grad_weight) return TAHQ_ERR_NULL;
    for (const void *p : {d_x, d_weight, (const void *)d_target, (const void *)d_lse, (const void *)d_workspace})
        if (!p) return TAHQ_ERR_NULL;
    Call call(cfg, true, d_workspace, stream);
    const LossPlan &p = call.p;
    if (workspace_capacity < p.total) return TAHQ_ERR_WORKSPACE_TOO_SMALL;
    for (const void *x : {d_x, d_weight, (const void *)d_lse, (const void *)d_grad_x, (const void *)d_grad_weight, (const void *)d_workspace})
        if (misaligned(x)) return TAHQ_ERR_MISALIGNED;
    if (reinterpret_cast<uintptr_t>(d_target) % sizeof *d_target || reinterpret_cast<uintptr_t>(d_grad_loss) % sizeof *d_grad_loss) return TAHQ_ERR_MISALIGNED;
    const bool each = cfg->reduction == TAHQ_LOSS_NONE;
    const uint32_t mean = cfg->reduction == TAHQ_LOSS_MEAN;
    const float *whole = each ? nullptr : d_grad_loss;
    call.gather(d_x, d_target, nullptr, nullptr, d_grad_x);
    for (uint32_t first = 0; first < cfg->vocab; first += p.piece) {
        const uint32_t rows = cfg->vocab - first < p.piece ? cfg->vocab - first : p.piece;
        const Call::Weight w = call.weight(d_weight, first, rows);
        LogitArgs g = call.logit_args(w, first, rows);
        g.lse = d_lse;
        g.grad_loss = each ? d_grad_loss : nullptr;
        g.grads = call.at<uint8_t>(p.grads);
        call.logits<kGrads>(g);
        if (d_grad_x)
            call.grad_x({g.grads, w.from, w.ld, p.g_plane, w.plane, call.tokens, rows, cfg->cols, (uint32_t)loss_ceil(rows, p.whole), p.x_stages, p.x_slots,
                         (uint32_t)loss_ceil(cfg->cols, kLossTiles[p.x_kind].tn), p.padded, first != 0, call.at<float4>(p.sums)});
        if (d_grad_weight)
            call.grad_w({g.grads, g.x, p.g_plane, p.x_plane, call.tokens, rows, cfg->cols, 0, 0, p.padded, whole, mean, cfg->weight_dtype == TAHQ_BF16, cfg->accumulate,
                         static_cast<uint8_t *>(d_grad_weight) + (uint64_t)first * cfg->cols * (cfg->weight_dtype == TAHQ_BF16 ? 2 : 4)});
    }
    if (d_grad_x) {
        const LossTile &t = kLossTiles[p.x_kind];
        const uint32_t eights = (uint32_t)loss_ceil(cfg->rows, 8), columns = (uint32_t)loss_ceil(cfg->cols, 128);
        call.q(p.bf16 ? k_loss_scatter<true> : k_loss_scatter<false>, dim3(eights, columns < 8 ? columns : 8), dim3(256), call.at<float4>(p.sums), p.x_stages, p.x_slots,
               (uint32_t)loss_ceil(cfg->cols, t.tn), SumsLayout{t.tm, t.tn, t.wm, t.wn}, call.tokens, cfg->cols, whole, mean, d_grad_x);
    }
    return call.q.result();
}

}  // extern "C"
