// How a loss over a vocabulary is cut, from its sizes alone: host code.
#pragma once
#include <stdint.h>

#include "tahq_loss.h"

namespace tahq {

constexpr uint32_t kLossSpan = 4096;         // tokens that are counted together
constexpr uint64_t kLossBudget = 256u << 20; // bytes of a piece, where the hidden states have no more
constexpr uint64_t kLossMostRows = 1u << 22; // rows of the vocabulary in a piece

// Tiles, and what a wavefront has of one; `along`: wavefronts side by side along the second
struct LossTile {
    uint32_t tm, tn, wm, wn, along;
};
constexpr LossTile kLossTiles[] = {{256, 256, 128, 128, 2}, {128, 128, 64, 64, 2}, {32, 128, 32, 32, 4}};
enum { kLossLarge = 0, kLossMiddle = 1, kLossFew = 2 };

inline uint64_t loss_ceil(uint64_t a, uint64_t b) { return (a + b - 1) / b; }
inline uint64_t loss_tiles(int kind, uint64_t m, uint64_t n) { return loss_ceil(m, kLossTiles[kind].tm) * loss_ceil(n, kLossTiles[kind].tn); }

// The kind of tile of a product [m, n]
inline int loss_kind(bool bf16, uint64_t m, uint64_t n)
{
    if (m <= 32) return kLossFew;
    return bf16 && loss_tiles(kLossLarge, m, n) >= 256 ? kLossLarge : kLossMiddle;
}

struct LossPlan {
    bool bf16, pad;                          // pad: the weight is copied into blocks of whole stages
    uint32_t es, whole, ldx, padded;         // bytes of an element; columns of a stage; elements of a gathered row; tokens up to whole stages
    uint32_t spans;                          // of kLossSpan tokens
    uint32_t forward_piece, backward_piece;  // rows of the vocabulary
    int forward_kind, grads_kind, x_kind;
    uint32_t parts, x_stages, x_slots;       // of a forward piece's statistics; of the sums for the hidden states' gradient: stages of the first piece, Shares
    uint64_t x_groups;                       // workgroups for them
    // places in the workspace
    uint64_t rows, targets, counts, x, at_target, running, stats, forward_weight, forward_total;
    uint64_t grads, sums, backward_weight, backward_total;
};

inline LossPlan plan_loss(const tahq_loss_config *c)
{
    LossPlan p = {};
    p.bf16 = c->dtype == TAHQ_BF16;
    p.es = p.bf16 ? 2 : 4;
    p.whole = 64 / p.es;
    p.ldx = (uint32_t)loss_ceil(c->cols, p.whole) * p.whole;
    p.pad = p.ldx != c->cols;
    p.padded = (uint32_t)loss_ceil(c->rows, p.whole) * p.whole;
    p.spans = (uint32_t)loss_ceil(c->rows, kLossSpan);
    uint64_t at = 256;
    auto place = [&](uint64_t bytes) {
        const uint64_t here = at;
        at += loss_ceil(bytes, 256) * 256;
        return here;
    };
    p.rows = place((uint64_t)p.padded * 4);
    p.targets = place((uint64_t)p.padded * 4);
    p.counts = place((uint64_t)p.spans * 4);
    p.x = place((uint64_t)p.padded * p.ldx * p.es);
    const uint64_t common = at, x_bytes = (uint64_t)p.padded * p.ldx * p.es, budget = x_bytes > kLossBudget ? x_bytes : kLossBudget;
    const uint64_t vocab = loss_ceil(c->vocab, 256) * 256;
    // rows of the vocabulary for which `each` bytes are kept: multiples of 256, and so few that eight blocks of them are less than 2^32 bytes apart
    auto piece = [&](uint64_t each) {
        uint64_t n = budget / each / 256 * 256;
        n = n < kLossMostRows ? n : kLossMostRows;
        return (uint32_t)(n < 256 ? 256 : n < vocab ? n : vocab);
    };
    // forward: 8 bytes of statistics of every token and 32 rows of the vocabulary at least; the copy of the weight
    p.forward_kind = loss_kind(p.bf16, c->rows, c->vocab);
    const LossTile &f = kLossTiles[p.forward_kind];
    p.forward_piece = piece((uint64_t)p.padded * 8 * f.along / f.tn + 1);
    if (p.pad && piece((uint64_t)p.ldx * p.es) < p.forward_piece) p.forward_piece = piece((uint64_t)p.ldx * p.es);
    p.parts = p.forward_piece / f.tn * f.along;
    p.at_target = place((uint64_t)p.padded * 4);
    p.running = place((uint64_t)p.padded * 8);
    p.stats = place((uint64_t)p.parts * p.padded * 8);
    p.forward_weight = place(p.pad ? (uint64_t)p.forward_piece * p.ldx * p.es : 0);
    p.forward_total = at;
    // backward
    at = common;
    p.backward_piece = piece((uint64_t)p.padded * p.es);
    if (p.pad && piece((uint64_t)p.ldx * p.es) < p.backward_piece) p.backward_piece = piece((uint64_t)p.ldx * p.es);
    const uint64_t widest = p.backward_piece < c->vocab ? p.backward_piece : c->vocab;
    p.grads_kind = loss_kind(p.bf16, c->rows, widest);
    // Few tiles: several workgroups share the sums of one over the vocabulary (Shares), as many as the device holds at once.  Then large tiles are as good
    // where there are few, but for what hangs over the edges (2048 x 1600, of which 1448 tokens count, x 50257: 365 us in tiles of 128 x 128, 245 in 256 x 256).
    const uint64_t stages = loss_ceil(widest, p.whole), large = loss_tiles(kLossLarge, c->rows, c->cols), middle = loss_tiles(kLossMiddle, c->rows, c->cols);
    p.x_kind = c->rows <= 32 ? kLossFew : p.bf16 && 3 * large <= middle && large * stages >= 256 * 16 ? kLossLarge : kLossMiddle;
    p.x_stages = (uint32_t)stages;
    p.x_slots = p.x_kind == kLossLarge ? 256 : 512;
    const uint64_t tiles = loss_tiles(p.x_kind, c->rows, c->cols);
    p.x_groups = tiles > p.x_slots ? tiles : p.x_slots;
    p.grads = place((uint64_t)p.padded * loss_ceil(widest, p.whole) * 64);
    p.sums = place(p.x_groups * kLossTiles[p.x_kind].tm * kLossTiles[p.x_kind].tn * 4);
    p.backward_weight = place(p.pad ? (uint64_t)p.backward_piece * p.ldx * p.es : 0);
    p.backward_total = at;
    return p;
}

}  // namespace tahq
