// Entry points of the mx4 matrices (include/tahq_mx4.h): validation, size arithmetic, launches.
#include <type_traits>

#include "tahq_enqueue.hpp"
#include "tahq_mx4_plan.hpp"
#include "tahq_mx4_product.hpp"
#include "tahq_mx4_quant.hpp"

using namespace tahq;

namespace {

bool dimension(uint32_t n) { return n > 0 && n < 0x80000000u; }

tahq_status check(const tahq_mx4_config *c)
{
    if (!c) return TAHQ_ERR_NULL;
    if (c->struct_size != sizeof *c) return TAHQ_ERR_INVALID_ARG;
    if (!dimension(c->rows) || !dimension(c->cols) || (c->ld && c->ld < c->cols)) return TAHQ_ERR_INVALID_ARG;
    if (c->dtype > TAHQ_BF16 || c->transform > 1 || c->scale_rule > TAHQ_MX4_COVER) return TAHQ_ERR_INVALID_ARG;
    return TAHQ_OK;
}
tahq_status check(const tahq_mx4_matmul_config *c)
{
    if (!c) return TAHQ_ERR_NULL;
    if (c->struct_size != sizeof *c) return TAHQ_ERR_INVALID_ARG;
    if (!dimension(c->m) || !dimension(c->n) || !dimension(c->k) || (c->ldc && c->ldc < c->n)) return TAHQ_ERR_INVALID_ARG;
    if (c->out_dtype > TAHQ_BF16 || c->accumulate > 1) return TAHQ_ERR_INVALID_ARG;
    return TAHQ_OK;
}

uint32_t cover_of(const tahq_mx4_config *c) { return c->scale_rule == TAHQ_MX4_COVER ? kCover : 0u; }
uint64_t ld_of(const tahq_mx4_config *c) { return c->ld ? c->ld : c->cols; }

template <bool BF16, bool ROTATE>
void launch_quantize(const tahq_mx4_config *c, const void *d_in, uint8_t *p, uint8_t *pt, uint32_t grid, uint32_t tiles_x, Enqueue *q)
{
    auto run = [&](auto kernel) {
        (*q)(kernel, dim3(grid), dim3(kQuantThreads), d_in, p, pt, c->rows, c->cols, ld_of(c), cover_of(c), tiles_x);
    };
    if (p && pt) run(k_mx4_quantize<BF16, true, true, ROTATE>);
    else if (p) run(k_mx4_quantize<BF16, true, false, ROTATE>);
    else run(k_mx4_quantize<BF16, false, true, ROTATE>);
}

struct QuantGrid {
    uint64_t tiles_x, tiles_y;
    bool fits() const { return launchable(tiles_x * tiles_y, kQuantThreads); }
};
QuantGrid quant_grid(const tahq_mx4_config *c, bool transposed)
{
    // along columns the last four units of 64 rows are filled up: their scale bytes are written, too
    return {ceil_div(c->cols, kQuantCols), transposed ? ceil_div(c->rows, 256) * (256 / kQuantRows) : ceil_div(c->rows, kQuantRows)};
}

tahq_status enqueue_quantize(const tahq_mx4_config *c, const void *d_in, void *d_packed, void *d_packed_t, Enqueue *q)
{
    const QuantGrid tiles = quant_grid(c, d_packed_t != nullptr);
    if (!tiles.fits()) return TAHQ_ERR_UNSUPPORTED;
    uint8_t *p = static_cast<uint8_t *>(d_packed), *pt = static_cast<uint8_t *>(d_packed_t);
    const uint32_t grid = (uint32_t)(tiles.tiles_x * tiles.tiles_y), tiles_x = (uint32_t)tiles.tiles_x;
    if (c->dtype == TAHQ_BF16) {
        if (c->transform) launch_quantize<true, true>(c, d_in, p, pt, grid, tiles_x, q);
        else launch_quantize<true, false>(c, d_in, p, pt, grid, tiles_x, q);
    } else {
        if (c->transform) launch_quantize<false, true>(c, d_in, p, pt, grid, tiles_x, q);
        else launch_quantize<false, false>(c, d_in, p, pt, grid, tiles_x, q);
    }
    return q->result();
}

bool product_fits(const tahq_mx4_matmul_config *c)
{
    const ProductPlan p = plan_product(c);
    if (p.kind < 0) return launchable(ceil_div(c->n, c->m <= 16 ? 16 : 32), 64 * kFewWaves);
    return launchable(tiles_of(kTiles[p.kind], c), p.kind == 5 ? 512 : 256);
}

uint64_t ldc_of(const tahq_mx4_matmul_config *c) { return c->ldc ? c->ldc : c->n; }

template <int WM, int WN, int MF, int NF, int NB, int KS, int PER_CU>
void launch_tiles(const tahq_mx4_matmul_config *c, const ProductPlan &p, const uint8_t *a, const uint8_t *b, void *d_c, void *d_workspace, Enqueue *q)
{
    const uint32_t tiles_m = (uint32_t)ceil_div(c->m, 32 * WM * MF), tiles_n = (uint32_t)ceil_div(c->n, 32 * WN * NF);
    auto run = [&](auto kernel, void *to) {
        (*q)(kernel, dim3(tiles_m * tiles_n, p.parts), dim3(64 * WM * WN * KS), a, b, to, c->m, c->n, c->k, ldc_of(c), c->accumulate, tiles_m, tiles_n, p.run);
    };
    if constexpr (MF == 1 && NF == 1 && KS == 1) {
        if (p.parts > 1) {
            run(k_mx4_tiles<WM, WN, MF, NF, NB, KS, PER_CU, 2>, d_workspace);
            const dim3 grid((uint32_t)ceil_div((uint64_t)c->m * c->n, 1024));
            (*q)(c->out_dtype == TAHQ_BF16 ? k_mx4_sum_parts<true> : k_mx4_sum_parts<false>, grid, dim3(256), static_cast<const float *>(d_workspace),
                 d_c, c->m, c->n, ldc_of(c), c->accumulate, p.parts);
            return;
        }
    }
    if (c->out_dtype == TAHQ_BF16) run(k_mx4_tiles<WM, WN, MF, NF, NB, KS, PER_CU, 1>, d_c);
    else run(k_mx4_tiles<WM, WN, MF, NF, NB, KS, PER_CU, 0>, d_c);
}

template <int MT, int NT, int QUANT, bool ROTATE, int PAIRS>
void launch_few(const tahq_mx4_matmul_config *c, const FewInput &in, const uint8_t *b, void *d_c, Enqueue *q)
{
    (*q)(k_mx4_few<MT, NT, QUANT, ROTATE, PAIRS>, dim3((uint32_t)ceil_div(c->n, 16 * NT)), dim3(64 * kFewWaves), b, in, d_c, c->m, c->n, c->k, ldc_of(c),
         c->accumulate, (uint32_t)(c->out_dtype == TAHQ_BF16));
}
template <int QUANT, bool ROTATE>
void launch_few_quant(const tahq_mx4_matmul_config *c, const FewInput &in, const uint8_t *b, void *d_c, Enqueue *q)
{
    if (c->m <= 2) launch_few<1, 1, QUANT, ROTATE, 1>(c, in, b, d_c, q);
    else if (c->m <= 4) launch_few<1, 1, QUANT, ROTATE, 2>(c, in, b, d_c, q);
    else launch_few<1, 1, QUANT, ROTATE, 4>(c, in, b, d_c, q);
}

tahq_status enqueue_product(const tahq_mx4_matmul_config *c, const void *d_a, const void *d_b, void *d_c, void *d_workspace, Enqueue *q)
{
    const ProductPlan p = plan_product(c);
    const uint8_t *a = static_cast<const uint8_t *>(d_a), *b = static_cast<const uint8_t *>(d_b);
    if (!product_fits(c)) return TAHQ_ERR_UNSUPPORTED;
    switch (p.kind) {
    case 0: launch_tiles<2, 2, 4, 4, 4, 1, 1>(c, p, a, b, d_c, d_workspace, q); break;
    case 1: launch_tiles<2, 2, 4, 2, 3, 1, 2>(c, p, a, b, d_c, d_workspace, q); break;
    case 2: launch_tiles<2, 2, 2, 2, 4, 1, 2>(c, p, a, b, d_c, d_workspace, q); break;
    case 3: launch_tiles<2, 2, 1, 2, 4, 1, 3>(c, p, a, b, d_c, d_workspace, q); break;
    case 4: launch_tiles<2, 2, 1, 1, 4, 1, 4>(c, p, a, b, d_c, d_workspace, q); break;
    case 5: launch_tiles<2, 2, 1, 1, 4, 2, 2>(c, p, a, b, d_c, d_workspace, q); break;
    default:
        if (c->m <= 16) launch_few<1, 1, 0, false, 1>(c, {a, 0, 0}, b, d_c, q);
        else launch_few<2, 2, 0, false, 1>(c, {a, 0, 0}, b, d_c, q);
    }
    return q->result();
}

tahq_status enqueue_few(const tahq_mx4_config *x, const tahq_mx4_matmul_config *c, const void *d_x, const uint8_t *b, void *d_c, Enqueue *q)
{
    const FewInput in{d_x, ld_of(x), cover_of(x)};
    if (x->dtype == TAHQ_BF16) x->transform ? launch_few_quant<1, true>(c, in, b, d_c, q) : launch_few_quant<1, false>(c, in, b, d_c, q);
    else x->transform ? launch_few_quant<2, true>(c, in, b, d_c, q) : launch_few_quant<2, false>(c, in, b, d_c, q);
    return q->result();
}

}  // namespace

extern "C" {

void tahq_mx4_config_default(tahq_mx4_config *cfg)
{
    if (!cfg) return;
    *cfg = tahq_mx4_config{};
    cfg->struct_size = (uint32_t)sizeof *cfg;
    cfg->dtype = TAHQ_BF16;
}

void tahq_mx4_matmul_config_default(tahq_mx4_matmul_config *cfg)
{
    if (!cfg) return;
    *cfg = tahq_mx4_matmul_config{};
    cfg->struct_size = (uint32_t)sizeof *cfg;
    cfg->out_dtype = TAHQ_BF16;
}

size_t tahq_mx4_packed_size(uint32_t rows, uint32_t cols)
{
    return dimension(rows) && dimension(cols) ? (size_t)Mx4Layout(rows, cols).total() : 0;
}

tahq_status tahq_mx4_quantize(const tahq_mx4_config *cfg, const void *d_in, void *d_packed, size_t packed_capacity,
                              void *d_packed_t, size_t packed_t_capacity, tahq_stream stream)
{
    const tahq_status rc = check(cfg);
    if (rc != TAHQ_OK) return rc;
    if (!d_in || (!d_packed && !d_packed_t)) return TAHQ_ERR_NULL;
    if (d_packed && packed_capacity < tahq_mx4_packed_size(cfg->rows, cfg->cols)) return TAHQ_ERR_BUFFER_TOO_SMALL;
    if (d_packed_t && packed_t_capacity < tahq_mx4_packed_size(cfg->cols, cfg->rows)) return TAHQ_ERR_BUFFER_TOO_SMALL;
    if (misaligned(d_in) || misaligned(d_packed) || misaligned(d_packed_t)) return TAHQ_ERR_MISALIGNED;
    Enqueue q{(hipStream_t)stream};
    return enqueue_quantize(cfg, d_in, d_packed, d_packed_t, &q);
}

tahq_status tahq_mx4_dequantize(const tahq_mx4_config *cfg, const void *d_packed, size_t packed_bytes, void *d_out, tahq_stream stream)
{
    const tahq_status rc = check(cfg);
    if (rc != TAHQ_OK) return rc;
    if (!d_packed || !d_out) return TAHQ_ERR_NULL;
    if (packed_bytes < tahq_mx4_packed_size(cfg->rows, cfg->cols)) return TAHQ_ERR_BUFFER_TOO_SMALL;
    if (misaligned(d_packed) || misaligned(d_out)) return TAHQ_ERR_MISALIGNED;
    const QuantGrid tiles = quant_grid(cfg, false);
    if (!tiles.fits()) return TAHQ_ERR_UNSUPPORTED;
    Enqueue q{(hipStream_t)stream};
    auto run = [&](auto kernel) {
        q(kernel, dim3((uint32_t)(tiles.tiles_x * tiles.tiles_y)), dim3(kQuantThreads), static_cast<const uint8_t *>(d_packed), d_out, cfg->rows,
          cfg->cols, ld_of(cfg), (uint32_t)tiles.tiles_x);
    };
    if (cfg->dtype == TAHQ_BF16) {
        if (cfg->transform) run(k_mx4_dequantize<true, true>);
        else run(k_mx4_dequantize<true, false>);
    } else {
        if (cfg->transform) run(k_mx4_dequantize<false, true>);
        else run(k_mx4_dequantize<false, false>);
    }
    return q.result();
}

size_t tahq_mx4_matmul_workspace_size(const tahq_mx4_matmul_config *cfg)
{
    return check(cfg) == TAHQ_OK ? (size_t)product_workspace(cfg) : 0;
}

tahq_status tahq_mx4_matmul(const tahq_mx4_matmul_config *cfg, const void *d_a, size_t a_bytes, const void *d_b, size_t b_bytes,
                            void *d_c, void *d_workspace, size_t workspace_capacity, tahq_stream stream)
{
    const tahq_status rc = check(cfg);
    if (rc != TAHQ_OK) return rc;
    const uint64_t need = product_workspace(cfg);
    if (!d_a || !d_b || !d_c || (need && !d_workspace)) return TAHQ_ERR_NULL;
    if (a_bytes < tahq_mx4_packed_size(cfg->m, cfg->k) || b_bytes < tahq_mx4_packed_size(cfg->n, cfg->k)) return TAHQ_ERR_BUFFER_TOO_SMALL;
    if (workspace_capacity < need) return TAHQ_ERR_WORKSPACE_TOO_SMALL;
    if (misaligned(d_a) || misaligned(d_b) || misaligned(d_c) || (need && misaligned(d_workspace))) return TAHQ_ERR_MISALIGNED;
    Enqueue q{(hipStream_t)stream};
    return enqueue_product(cfg, d_a, d_b, d_c, d_workspace, &q);
}

size_t tahq_mx4_linear_workspace_size(const tahq_mx4_config *x, const tahq_mx4_matmul_config *cfg)
{
    if (check(x) != TAHQ_OK || check(cfg) != TAHQ_OK || x->rows != cfg->m || x->cols != cfg->k) return 0;
    return (size_t)(Mx4Layout(x->rows, x->cols).total() + product_workspace(cfg));
}

tahq_status tahq_mx4_linear(const tahq_mx4_config *x, const tahq_mx4_matmul_config *cfg, const void *d_x, const void *d_b,
                            size_t b_bytes, void *d_y, void *d_workspace, size_t workspace_capacity, tahq_stream stream)
{
    tahq_status rc = check(x);
    if (rc == TAHQ_OK) rc = check(cfg);
    if (rc != TAHQ_OK) return rc;
    if (x->rows != cfg->m || x->cols != cfg->k) return TAHQ_ERR_INVALID_ARG;
    const uint64_t need = tahq_mx4_linear_workspace_size(x, cfg);
    if (!d_x || !d_b || !d_y || !d_workspace) return TAHQ_ERR_NULL;
    if (b_bytes < tahq_mx4_packed_size(cfg->n, cfg->k)) return TAHQ_ERR_BUFFER_TOO_SMALL;
    if (workspace_capacity < need) return TAHQ_ERR_WORKSPACE_TOO_SMALL;
    if (misaligned(d_x) || misaligned(d_b) || misaligned(d_y) || misaligned(d_workspace)) return TAHQ_ERR_MISALIGNED;
    if (!product_fits(cfg)) return TAHQ_ERR_UNSUPPORTED;
    Enqueue q{(hipStream_t)stream};
    if (quantizes_itself(cfg)) return enqueue_few(x, cfg, d_x, static_cast<const uint8_t *>(d_b), d_y, &q);
    uint8_t *packed = static_cast<uint8_t *>(d_workspace);
    rc = enqueue_quantize(x, d_x, packed, nullptr, &q);
    if (rc != TAHQ_OK) return rc;
    return enqueue_product(cfg, packed, d_b, d_y, packed + Mx4Layout(x->rows, x->cols).total(), &q);
}

}  // extern "C"
