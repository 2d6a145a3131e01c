// Entry points of the mx4 matrices (include/tahq_mx4.h): validation, size arithmetic, launches.
#include <type_traits>

#include "tahq_enqueue.hpp"
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

constexpr uint64_t kMaxGrid = 0x7fffffffu;
uint64_t ceil_div(uint64_t a, uint64_t b) { return (a + b - 1) / b; }
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

tahq_status enqueue_quantize(const tahq_mx4_config *c, const void *d_in, void *d_packed, void *d_packed_t, Enqueue *q)
{
    // along columns the last four units of 64 rows are filled up: their scale bytes are written, too
    const uint64_t tiles_y = d_packed_t ? ceil_div(c->rows, 256) * 4 : ceil_div(c->rows, kQuantRows);
    const uint64_t tiles_x = ceil_div(c->cols, kQuantCols);
    if (tiles_x * tiles_y > kMaxGrid) return TAHQ_ERR_UNSUPPORTED;
    uint8_t *p = static_cast<uint8_t *>(d_packed), *pt = static_cast<uint8_t *>(d_packed_t);
    const uint32_t grid = (uint32_t)(tiles_x * tiles_y);
    if (c->dtype == TAHQ_BF16) {
        if (c->transform) launch_quantize<true, true>(c, d_in, p, pt, grid, (uint32_t)tiles_x, q);
        else launch_quantize<true, false>(c, d_in, p, pt, grid, (uint32_t)tiles_x, q);
    } else {
        if (c->transform) launch_quantize<false, true>(c, d_in, p, pt, grid, (uint32_t)tiles_x, q);
        else launch_quantize<false, false>(c, d_in, p, pt, grid, (uint32_t)tiles_x, q);
    }
    return q->result();
}

tahq_status enqueue_product(const tahq_mx4_matmul_config *c, const void *d_a, const void *d_b, void *d_c, void *, Enqueue *q)
{
    const uint64_t tiles_n = ceil_div(c->n, 64), tiles = tiles_n * ceil_div(c->m, 64);
    if (tiles > kMaxGrid) return TAHQ_ERR_UNSUPPORTED;
    const uint64_t ldc = c->ldc ? c->ldc : c->n;
    const uint8_t *a = static_cast<const uint8_t *>(d_a), *b = static_cast<const uint8_t *>(d_b);
    (*q)(c->out_dtype == TAHQ_BF16 ? k_mx4_product<true> : k_mx4_product<false>, dim3((uint32_t)tiles), dim3(64), a, b, d_c,
         c->m, c->n, c->k, ldc, c->accumulate, (uint32_t)tiles_n);
    return q->result();
}

uint64_t product_workspace(const tahq_mx4_matmul_config *) { return 0; }

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
    const uint64_t tiles_x = ceil_div(cfg->cols, kQuantCols), tiles = tiles_x * ceil_div(cfg->rows, 32);
    if (tiles > kMaxGrid) return TAHQ_ERR_UNSUPPORTED;
    Enqueue q{(hipStream_t)stream};
    auto run = [&](auto kernel) {
        q(kernel, dim3((uint32_t)tiles), dim3(kQuantThreads), static_cast<const uint8_t *>(d_packed), d_out, cfg->rows, cfg->cols,
          ld_of(cfg), (uint32_t)tiles_x);
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
    Enqueue q{(hipStream_t)stream};
    uint8_t *packed = static_cast<uint8_t *>(d_workspace);
    rc = enqueue_quantize(x, d_x, packed, nullptr, &q);
    if (rc != TAHQ_OK) return rc;
    return enqueue_product(cfg, packed, d_b, d_y, packed + Mx4Layout(x->rows, x->cols).total(), &q);
}

}  // extern "C"
