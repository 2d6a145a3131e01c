// The plan of a product of mx4 matrices, from its sizes and the type of its result: host code alone.
#pragma once
#include <stdint.h>

#include "tahq_mx4.h"

namespace tahq {

inline uint64_t ceil_div(uint64_t a, uint64_t b) { return (a + b - 1) / b; }

// How a product is cut.  Up to kFewRows rows of A: k_mx4_few.  More: tiles, of the kind that the estimate below takes least time with, and for few
// tiles and a long k several runs of it, whose sums are added afterwards.
constexpr uint32_t kFewRows = 32, kFewQuantRows = 8;

// Time of a product on 256 compute units, in us, with tiles of tm x tn of which `per_cu` are on a compute unit at once: `start` for
// each that one takes after another, `each` byte of results, and for 256 columns `alone` while a unit has one tile and not all units
// have one, `loaded` for each tile of a unit's once they have.  (All units at work slow down: 256 x 256 tiles 1.37 -> 1.77 us; the
// clock gives way.)  Fitted to 166 shapes from 33 x 512 x 512 to 8192^3, of a part of them both types of C: what it chooses takes 0.4 %
// longer on average than the best of the six.  The last kind has two teams to a tile: 64 x 8192 x 8192 11.4 -> 9.6 us, 512 x 2048 x
// 8192 11.1 -> 10.1; two teams for larger tiles and four for these gained nothing more.
struct TileKind {
    uint32_t tm, tn, per_cu;
    float start, alone, loaded;
};
constexpr TileKind kTiles[] = {
    {256, 256, 1, 5.6f, 1.37f, 1.77f},  {256, 128, 2, 4.18f, 0.687f, 1.08f}, {128, 128, 2, 2.68f, 0.43f, 0.584f},
    {64, 128, 3, 2.75f, 0.32f, 0.36f}, {64, 64, 4, 2.84f, 0.275f, 0.248f},  {64, 64, 2, 3.3f, 0.22f, 0.24f}};
constexpr float kEachByte = 4e-5f;

inline uint64_t tiles_of(const TileKind &t, const tahq_mx4_matmul_config *c) { return ceil_div(c->m, t.tm) * ceil_div(c->n, t.tn); }

inline float estimate(const TileKind &t, const tahq_mx4_matmul_config *c)
{
    const float tiles = (float)tiles_of(t, c), groups = (float)ceil_div(c->k, 256), share = tiles / 256.0f;
    const float out = (float)t.tm * t.tn * (c->out_dtype == TAHQ_BF16 ? 2 : 4) * kEachByte;
    if (share <= 1.0f) {
        const float more = t.loaded > t.alone ? (t.loaded - t.alone) * share : 0.0f;
        return t.start + out * share + groups * (t.alone + more);
    }
    const float most = __builtin_ceilf(share), rounds = __builtin_ceilf(most / t.per_cu);
    const float busy = t.loaded * most > t.alone ? t.loaded * most : t.alone;
    return (t.start + out) * rounds + groups * busy;
}

struct ProductPlan {
    int kind;              // of kTiles; -1: few rows
    uint32_t run, parts;   // groups of 256 columns in a run, runs
};
inline ProductPlan plan_product(const tahq_mx4_matmul_config *c)
{
    const uint32_t groups = (uint32_t)ceil_div(c->k, 256);
    ProductPlan p{-1, groups, 1};
    // a half unit of B's rows to a workgroup reads A too often where B is long: 32 rows, 28672 x 8192: 31 us, 64 x 64 tiles 23
    if (c->m <= 16 || (c->m <= kFewRows && c->n <= 16384)) return p;
    float best = 0.0f;
    for (int i = 0; i < (int)(sizeof kTiles / sizeof *kTiles); ++i) {
        const float t = estimate(kTiles[i], c);
        if (p.kind < 0 || t < best) {
            p.kind = i;
            best = t;
        }
    }
    // A long sum in few of the smallest tiles: runs of 16 groups and more, as many as there are compute units for.  512 x 512 x 16384: 15.8 us
    // in one run of two teams, 13.9 in four; with 32 groups, x 8192, 9.0 and 11.1.
    const uint64_t tiles = tiles_of(kTiles[p.kind], c);
    if (p.kind >= 4 && groups >= 48 && tiles <= 64) {
        const uint32_t by_units = (uint32_t)(256 / tiles), by_length = groups / 16;
        p.kind = 4;
        p.run = (uint32_t)ceil_div(groups, by_units < by_length ? by_units : by_length);
        p.parts = (uint32_t)ceil_div(groups, p.run);
    }
    return p;
}
inline uint64_t product_workspace(const tahq_mx4_matmul_config *c)
{
    const ProductPlan p = plan_product(c);
    return p.parts > 1 ? (uint64_t)p.parts * c->m * c->n * 4 : 0;
}

// Few rows in fp32 or bf16 are quantized in the product's launch, by every workgroup anew, where that is less than a launch of its own: up to two
// rows (8192 x 8192: 9.0 us, apart 7.6 + 4.6), up to eight if B is small (4 rows, 4096 x 4096: 5.2, 3.7 + 4.5; 8192 x 8192: 13.9, 7.6 + 4.6).
inline bool quantizes_itself(const tahq_mx4_matmul_config *c)
{
    return c->m <= 2 || (c->m <= kFewQuantRows && (uint64_t)c->n * c->k <= (1u << 24));
}

}  // namespace tahq
