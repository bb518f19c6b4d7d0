// How the head loss (dv_head.hip) cuts its work: the pieces of the vocabulary, the products'
// tiles and splits, and the workspaces.  Host code only.
#pragma once

#include "dv_train.h"

namespace dv {

constexpr int64_t kPieceElements = (int64_t)1 << 27;
constexpr int kPieceTokens = 1 << 18;
constexpr int64_t kPackedPerRow = (int64_t)1 << 19;

// The tile side and the splits of k for a product of `i` x `j` over `stages` of
// k (64 of bf16, 32 of fp32), by the time that each choice would take.  Up to
// per_unit blocks share a compute unit: a stage of all of them takes `us` (PFLOP/s
// at 8192 x 8192 x 4096, bf16 and fp32: side 256 1.17 and 0.205, 128 1.09 and 0.181, 64
// 0.66 and 0.122), one alone two fifths of that and more; a tile takes some stages
// more to start and end; its results (out_bytes an element; 0: what little the
// logits' kernels write does not count) leave at the unit's share of the memory,
// hidden behind another block's work where units have several.  Splits write and
// read their sums.  Against all choices of side and splits, timed at nine shapes of
// 8 to 8,192 rows in both types, it picks one within 5 % of the fastest.
//
// fp32 products of at most 32 rows j may take tiles of 64 x 32: each part of A is
// split for fewer columns that nobody asked for (8 x 4096 x 128,256 forward: 455 us, in 64 x 64 ones 637).
constexpr int kNarrow = 32;

struct Plan {
    int side, splits, stages;  // stages of a split; no split is empty
};

inline Plan plan_product(int64_t i, int64_t j, int64_t stages, int most_splits, bool bf16, int out_bytes, bool narrow)
{
    struct Side {
        int side, other, per_unit, around;  // around: stages that a tile's start and end cost
        double us[2];
    };
    constexpr Side kSides[] = {{256, 256, 1, 3, {1.72, 5.2}},
                               {128, 128, 2, 5, {1.03, 3.1}},
                               {64, 64, 4, 5, {0.80, 2.3}},
                               {kNarrow, 64, 6, 5, {0, 2.3}}};
    constexpr int kUnits = 256;
    constexpr double kBytesPerUs = 19500;  // of a unit
    Plan best{64, 1, (int)stages};
    double least = 1e30;
    for (const Side &s : kSides) {
        if (s.side == kNarrow && (!narrow || bf16 || j > kNarrow))
            continue;
        const int64_t tiles = ((i + s.other - 1) / s.other) * ((j + s.side - 1) / s.side);
        for (int64_t want = 1; want <= most_splits; ++want) {
            const int64_t per = (stages + want - 1) / want;
            const int64_t used = (stages + per - 1) / per;
            const int64_t blocks = tiles * used, slots = (int64_t)kUnits * s.per_unit;
            const double tile_bytes = (double)s.side * s.other * (used > 1 ? 4 : out_bytes);
            const auto round = [&](int64_t per_unit) {
                const double work = (double)(per + s.around) * s.us[bf16 ? 0 : 1] * (0.4 + 0.6 * (double)per_unit / s.per_unit);
                const double store = (double)per_unit * tile_bytes / kBytesPerUs;
                return per_unit > 1 ? (work > store ? work : store) : work + store;
            };
            const int64_t rest = blocks % slots;
            const double us = (double)(blocks / slots) * round(s.per_unit) +
                              (rest ? round((rest + kUnits - 1) / kUnits) : 0) +
                              (used > 1 ? (double)(used * i * j) * 2e-6 + 5 : 0);
            if (us < least) {
                least = us;
                best = {s.side, (int)used, (int)per};
            }
        }
    }
    return best;
}

inline int64_t up64(int64_t n) { return (n + 63) / 64 * 64; }

// Which operands are used where they lie, the others packed: rows of whole stages from
// 16-byte boundaries, not too far apart for the loads' 32-bit offsets.
struct InPlace {
    bool x, w;
};

inline bool in_place(const void *p, int64_t ld, int dtype, int hidden)
{
    return hidden % 64 == 0 && ld % (dtype == 1 ? 8 : 4) == 0 && reinterpret_cast<uintptr_t>(p) % 16 == 0 &&
           ld <= ((int64_t)1 << 20);
}

inline InPlace in_place(const HeadArgs &a)
{
    return {in_place(a.x, a.ld_x, a.dtype, a.hidden), in_place(a.weight, a.ld_w, a.dtype, a.hidden)};
}

// The workspace: packed operands where they are not in place, and what the call itself needs.
struct HeadLayout {
    InPlace here;
    int64_t k;        // hidden size as the products see it
    int stage_k;
    int piece;        // tokens of a piece, a multiple of 256 (or all)
    int pieces;
    size_t x, w;
    size_t bytes;

    size_t take(size_t n)
    {
        const size_t at = bytes;
        bytes += align_up(n, 256);
        return at;
    }
};

// A piece has at most kPieceElements of G, and of packed weights that many and more with the
// rows, whose products lose by a cut (the loss of 300 rows x 4100 x 50,257 bf16 in one piece
// and two: 384 and 413 us; 8 x 4096 x 128,256 in one and four: 655 and 630, backward 1111 and
// 1049); or the least number of tokens that keeps the products' tiles busy.
inline HeadLayout head_layout(int rows, int hidden, int V, int dtype, InPlace here)
{
    HeadLayout l{};
    const size_t elt = dtype == 1 ? 2 : 4;
    l.here = here;
    l.k = up64(hidden);
    l.stage_k = 128 / (int)elt;
    const int64_t r64 = up64(rows > 0 ? rows : 1);
    const auto tokens = [](int64_t elements, int64_t least) {
        const int64_t n = elements / 256 * 256;
        return n < least ? least : n > kPieceTokens ? kPieceTokens : n;
    };
    int64_t piece = tokens(kPieceElements / r64, 4096);
    if (!here.w) {
        const int64_t packed = tokens((kPieceElements + rows * kPackedPerRow) / l.k, 8192);
        piece = packed < piece ? packed : piece;
    }
    l.pieces = (int)((V + piece - 1) / piece);
    // pieces of about the same size
    piece = ((V + l.pieces - 1) / l.pieces + 255) / 256 * 256;
    l.piece = (int)(piece < V ? piece : V);
    l.pieces = (int)((V + l.piece - 1) / l.piece);
    l.x = l.take(here.x ? 0 : r64 * l.k * elt);
    l.w = l.take(here.w ? 0 : up64(l.piece) * l.k * elt);
    return l;
}

// The tile side for the logits of n tokens.
inline int logits_side(const HeadLayout &l, int rows, int64_t n, bool bf16)
{
    return plan_product(n, rows, l.k / l.stage_k, 1, bf16, 0, true).side;
}

// Tokens of one launch of the loss at most: tiles of any side, 512 threads each, stay below
// the 2^32 threads of a grid.
inline int64_t launch_tokens(int rows)
{
    constexpr int64_t kMostTiles = (int64_t)1 << 22;
    return kMostTiles / (((int64_t)rows + 63) / 64) * 64 / 256 * 256;
}

struct ForwardLayout : HeadLayout {
    int step;    // tokens of a launch
    int side;
    int nparts;  // softmax states of a row
    size_t parts, target_logit;
};

inline ForwardLayout forward_layout(int rows, int hidden, int V, int dtype, InPlace here)
{
    ForwardLayout l{head_layout(rows, hidden, V, dtype, here)};
    l.step = here.w ? V : l.piece;
    if (rows > 0 && l.step > launch_tokens(rows))
        l.step = (int)launch_tokens(rows);
    l.side = logits_side(l, rows, l.step, dtype == 1);
    const int tile_tokens = l.side == kNarrow ? 64 : l.side;
    l.nparts = (V + tile_tokens - 1) / tile_tokens * 2;
    l.parts = l.take((size_t)l.nparts * rows * sizeof(Softmax));
    l.target_logit = l.take((size_t)rows * 4);
    return l;
}

// A stage of the gradients' products takes 32 rows or tokens of G: in fp32, or in two bf16
// parts (a stage of 64 k).
constexpr int kGradientStage = 32;
__host__ __device__ constexpr int gradient_rows(int rows) { return (rows + kGradientStage - 1) / kGradientStage * kGradientStage; }

struct BackwardLayout : HeadLayout {
    Plan dx_plan;
    size_t g, weight, dx, dw;
};

inline Plan dw_plan(const HeadLayout &l, int rows, int64_t n, bool bf16)
{
    const int64_t stages = rows > 0 ? gradient_rows(rows) / kGradientStage : 1;
    return plan_product(l.k, n, stages, 8, bf16, bf16 ? 2 : 4, false);
}

inline BackwardLayout backward_layout(int rows, int hidden, int V, int dtype, InPlace here)
{
    BackwardLayout l{head_layout(rows, hidden, V, dtype, here)};
    const int64_t p64 = up64(l.piece);
    l.g = l.take((size_t)gradient_rows(rows) * p64 * 4);  // an fp32 element or both parts
    l.weight = l.take((size_t)rows * 4);
    // dx over a piece: few tiles and a long k
    l.dx_plan = plan_product(l.k, rows, p64 / kGradientStage, 16, dtype == 1, 4, true);
    l.dx = l.take((size_t)l.dx_plan.splits * rows * hidden * 4);
    // dw over a piece, and over the last one: split where hidden and tokens make few tiles
    const auto dw_sums = [&](int64_t n) {
        const Plan p = dw_plan(l, rows, n, dtype == 1);
        return p.splits > 1 ? (size_t)p.splits * n * hidden * 4 : 0;
    };
    const size_t whole = dw_sums(l.piece), last = dw_sums(V - (int64_t)(l.pieces - 1) * l.piece);
    l.dw = l.take(whole > last ? whole : last);
    return l;
}

}  // namespace dv
