// How a loss over a vocabulary is cut, from its sizes alone: host code, but for Shares.
#pragma once
#include <stdint.h>

#include "tahq_loss.h"

#ifdef __HIP__
#define TAHQ_LOSS_BOTH __host__ __device__
#else
#define TAHQ_LOSS_BOTH
#endif

namespace tahq {

constexpr uint32_t kLossSpan = 4096;         // tokens that are counted together
constexpr uint64_t kLossBudget = 256u << 20; // bytes of a piece, where the hidden states have no more
constexpr uint64_t kLossMostRows = 1u << 22; // rows of the vocabulary in a piece

// fp32 is multiplied as such (v_mfma_f32_32x32x2_f32, 110 to 135 TFLOP/s here), or as three bf16 whose sum it is, six products of bf16 for one (at the
// tiles; 155 to 200 TFLOP/s of fp32), for which the weight is copied into planes first.  So many tokens pay for that, as such and in planes: forward (2048
// x 32000: 260 tokens 328 and 402 us, 400 500 and 476), with rows of no whole stages, which are copied in any case (2047: 100 tokens 264 and 263, 200 378
// and 329); backward, where three products share a copy (160 637 and 650, 200 743 and 694, 400 1382 and 1136).  And so many tiles of 128 x 128: six
// products take six times the stages, one after another (400 x 5120 x 2000, 64 tiles: 116 and 290 forward, 284 and 422 backward; 400 x 2048 x 32000 has
// 1000).
constexpr uint64_t kPlanesTiles = 256;
constexpr uint32_t kPlanesPadded = 112, kPlanesForward = 384, kPlanesBackward = 224;

// Large tiles of fp32 in planes have no registers for sums in parts: they sum so many stages of 32 columns one after another, 384 instructions as in a
// part of fp32 as such.  Longer sums of logits go in middle tiles (2048 x 1600 x 32000 forward 1.06 and 1.28 ms, losses off by 8.8e-7 and 6.9e-7; 4194 x
// 4096 x 32000 5.7 and 6.5 ms, 1.13e-6 and 6.3e-7), those of gradients run after run, which are added up in memory (hidden states' gradients of these
// two off by 1.06e-6 and 3.6e-7, 1.59e-6 and 4.0e-7; backward in all 3.4 and 3.9 ms, 20.2 and 22.5).
constexpr uint32_t kPlanesChain = 32;

// Up to 32 tokens forward go by tiles of 128 rows of the vocabulary through LDS, or, against so many rows, by 32 rows from registers with eight wavefronts
// to the channels, as there are few tiles of one stage after another (5 x 8192 x n: fp32 n 2345 173 and 68 us, 8192 180 and 99, 16384 183 and 200; bf16 51
// and 29, 67 and 36, 86 and 71; 30 x 1600 x 16384 20 and 32).
constexpr uint32_t kFewSplit = 8192;

// Tiles, and what a wavefront has of one; `along`: wavefronts side by side along the second
struct LossTile {
    uint32_t tm, tn, wm, wn, along;
};
constexpr LossTile kLossTiles[] = {{256, 256, 128, 128, 2}, {128, 128, 64, 64, 2}, {32, 128, 32, 32, 4}};
enum { kLossLarge = 0, kLossMiddle = 1, kLossFew = 2 };

inline uint64_t loss_ceil(uint64_t a, uint64_t b) { return (a + b - 1) / b; }
inline uint64_t loss_tiles(int kind, uint64_t m, uint64_t n) { return loss_ceil(m, kLossTiles[kind].tm) * loss_ceil(n, kLossTiles[kind].tn); }

// Whether a product [m, n] of bf16 goes in large tiles, 256 at a time, or middle ones, 512 in three fifths of the time.  Forward, 1024 x 4096 x n in tiles
// of 256 x 256 and of 128 x 128: 128 large tiles 94 and 76 us, 192 105 and 107, 256 120 and 135, 320 191 and 165, 512 226 and 273.
inline bool loss_large(uint64_t m, uint64_t n)
{
    const uint64_t tiles = loss_tiles(kLossLarge, m, n), middle = loss_tiles(kLossMiddle, m, n);
    return tiles >= 256 && 5 * loss_ceil(tiles, 256) <= 3 * loss_ceil(middle, 512);
}

// The kind of tile of logits; `wide`: of bf16.  Products of fp32 as such keep the matrix cores busy whatever the tile, so smaller tiles, a quarter of a
// middle one each, pay where they spread better over 256 compute units (forward in middle and in small ones: 163 x 5120 x 1355 339 and 117 us, 200 x 1600 x
// 9000 115 and 70, 200 x 1600 x 50257 391 and 327; but 220 x 4096 x 32000, seven rounds in the place of eight, 517 and 542).
inline int loss_kind(bool wide, uint64_t m, uint64_t n)
{
    const uint64_t few = loss_tiles(kLossFew, m, n), middle = loss_tiles(kLossMiddle, m, n);
    if (m <= 32 || (!wide && 5 * loss_ceil(few, 256) <= 16 * loss_ceil(middle, 256))) return kLossFew;
    return wide && loss_large(m, n) ? kLossLarge : kLossMiddle;
}

// How sums over a piece's `stages` are shared: `parts` of `run` stages, so many that `slots` workgroups, what the device holds at once, have one each of
// the tiles of the tokens that count; sixteen stages and more to a part of the first piece.  Later pieces, which are no longer, are added to the first
// one's parts, to no more of them than there are.
struct Shares {
    uint32_t tiles, parts, run;
    TAHQ_LOSS_BOTH Shares(uint32_t tiles_, uint32_t first_stages, uint32_t stages, uint32_t slots) : tiles(tiles_)
    {
        const uint32_t fit = slots / (tiles ? tiles : 1), most = first_stages / 16;
        const uint32_t want = fit < most ? (fit ? fit : 1) : (most ? most : 1);
        const uint32_t each = (first_stages + want - 1) / want, first = (first_stages + each - 1) / each;
        run = (stages + first - 1) / first;
        parts = (stages + run - 1) / run;
    }
};

// The plan of one direction.
struct LossPlan {
    bool bf16, planes;                       // the tensors' type; fp32 as three planes of bf16
    bool copy;                               // the weight is copied into blocks of whole stages
    bool few;                                // forward, up to 32 tokens: instead of that the weight as it lies, and hidden states are not gathered either
    bool split;                              // with several wavefronts to the channels
    uint32_t es, whole, blocks, padded;      // bytes of an element in a tile; columns of a stage; stages of a row of x; tokens up to whole stages
    uint32_t spans;                          // of kLossSpan tokens
    uint32_t piece;                          // rows of the vocabulary
    int kind, x_kind;                        // tiles of logits, of the hidden states' gradient
    uint32_t parts;                          // of a forward piece's statistics
    uint32_t x_stages, x_slots;              // sums for the hidden states' gradient: stages of the first piece, Shares
    uint64_t x_groups;                       // workgroups for them
    uint64_t x_plane, g_plane;               // bytes of a plane
    // places in the workspace
    uint64_t rows, targets, counts, x, at_target, running, stats, grads, sums, weight, total;
};

inline LossPlan plan_loss(const tahq_loss_config *c, bool backward)
{
    LossPlan p = {};
    p.bf16 = c->dtype == TAHQ_BF16;
    const bool odd = c->cols % (p.bf16 ? 32 : 16) != 0;
    p.planes = !p.bf16 && c->rows >= (odd ? kPlanesPadded : backward ? kPlanesBackward : kPlanesForward) && loss_tiles(kLossMiddle, c->rows, c->vocab) >= kPlanesTiles;
    p.split = !backward && c->rows <= 32 && c->vocab <= kFewSplit;
    p.few = !backward && c->rows <= 32 && (odd || p.split);
    p.copy = (odd || p.planes) && !p.few;
    p.es = p.bf16 || p.planes ? 2 : 4;
    p.whole = 64 / p.es;
    p.blocks = (uint32_t)loss_ceil(c->cols, p.whole);
    p.padded = (uint32_t)loss_ceil(c->rows, p.whole) * p.whole;
    p.spans = (uint32_t)loss_ceil(c->rows, kLossSpan);
    const uint32_t n = p.planes ? 3 : 1;
    uint64_t at = 256;
    auto place = [&](uint64_t bytes) {
        const uint64_t here = at;
        at += loss_ceil(bytes, 256) * 256;
        return here;
    };
    p.rows = place((uint64_t)p.padded * 4);
    p.targets = place((uint64_t)p.padded * 4);
    p.counts = place((uint64_t)p.spans * 4);
    p.x_plane = (uint64_t)p.padded * p.blocks * 64;
    p.x = place(n * p.x_plane);
    const uint64_t x_bytes = n * p.x_plane, least = p.planes ? 2 * kLossBudget : kLossBudget, budget = x_bytes > least ? x_bytes : least;
    const uint64_t vocab = loss_ceil(c->vocab, 256) * 256;
    // rows of the vocabulary for which `each` bytes are kept: multiples of 256, and so few that eight blocks of them are less than 2^32 bytes apart
    auto piece = [&](uint64_t each) {
        uint64_t rows = budget / each / 256 * 256;
        rows = rows < kLossMostRows ? rows : kLossMostRows;
        return (uint32_t)(rows < 256 ? 256 : rows < vocab ? rows : vocab);
    };
    // Pieces of at most `most` rows, so long that their tiles make whole rounds of the compute units where that is possible: launches take a round for
    // every 256 tiles, begun or not, of as many stages as `logits` and `weights` say and a start as long as twenty more.  (Tiles of 256 x 256; fp32 4319 x
    // 1024 x 50257, pieces of 20480 rows, 320 tiles of the weight's gradient: 9.99 ms, chosen so 9.87, sums of gradients in one run.)
    const uint64_t factor = p.planes ? 6 : 1, tiles_m = loss_tiles(kLossLarge, c->rows, 1), tiles_c = loss_tiles(kLossLarge, c->cols, 1);
    auto even = [&](uint32_t most, uint64_t logits, uint64_t weights) {
        if (p.es != 2 || c->rows <= 32 || most >= vocab) return most;
        auto cost = [&](uint64_t t) {
            return t ? loss_ceil(tiles_m * t, 256) * (logits + 20) + (weights ? loss_ceil(t * tiles_c, 256) * (weights + 20) : 0) + 30 : 0;
        };
        uint64_t best = most / 256, least_cost = ~0ull;
        for (uint64_t t = most / 256, end = t > 64 ? t - 64 : 0; t > end; --t) {
            const uint64_t all = vocab / 256, here = all / t * cost(t) + cost(all % t);
            if (here < least_cost) {
                least_cost = here;
                best = t;
            }
        }
        return (uint32_t)(best * 256);
    };
    auto kind_of = [&](uint64_t vocab_rows) {
        const int kind = loss_kind(p.es == 2, c->rows, vocab_rows);
        return p.planes && kind == kLossLarge && p.blocks > kPlanesChain ? (int)kLossMiddle : kind;
    };
    const uint32_t copied = p.copy ? piece((uint64_t)n * p.blocks * 64) : ~0u;
    if (!backward) {
        // 8 bytes of statistics of every token and 32 rows of the vocabulary at least
        p.kind = kind_of(c->vocab);
        const LossTile &t = kLossTiles[p.kind];
        p.piece = piece((uint64_t)p.padded * 8 * t.along / t.tn + 1);
        if (copied < p.piece) p.piece = even(copied, factor * p.blocks, 0);
        p.parts = p.piece / t.tn * t.along;
        p.at_target = place((uint64_t)p.padded * 4);
        p.running = place((uint64_t)p.padded * 8);
        p.stats = place((uint64_t)p.parts * p.padded * 8);
    } else {
        p.piece = piece((uint64_t)n * p.padded * p.es);
        p.piece = even(copied < p.piece ? copied : p.piece, factor * p.blocks, factor * loss_ceil(c->rows, p.whole));
        const uint64_t widest = p.piece < c->vocab ? p.piece : c->vocab;
        p.kind = kind_of(widest);
        // Few tiles: several workgroups share the sums of one over the vocabulary (Shares), as many as the device holds at once.  Then large tiles are as
        // good where there are few, but for what hangs over the edges (2048 x 1600, of which 1448 tokens count, x 50257: 365 us in tiles of 128 x 128, 245
        // in 256 x 256).
        const uint64_t stages = loss_ceil(widest, p.whole), large = loss_tiles(kLossLarge, c->rows, c->cols), middle = loss_tiles(kLossMiddle, c->rows, c->cols);
        p.x_kind = c->rows <= 32 ? kLossFew : p.es == 2 && 3 * large <= middle && large * stages >= 256 * 16 ? kLossLarge : kLossMiddle;
        p.x_stages = (uint32_t)stages;
        p.x_slots = p.x_kind == kLossLarge ? 256 : 512;
        const uint64_t tiles = loss_tiles(p.x_kind, c->rows, c->cols);
        p.x_groups = tiles > p.x_slots ? tiles : p.x_slots;
        p.g_plane = (uint64_t)p.padded * stages * 64;
        p.grads = place(n * p.g_plane);
        p.sums = place(p.x_groups * kLossTiles[p.x_kind].tm * kLossTiles[p.x_kind].tn * 4);
    }
    p.weight = place(p.copy ? (uint64_t)n * p.piece * p.blocks * 64 : 0);
    p.total = at;
    return p;
}

}  // namespace tahq
