// How the embedding and the cross entropy over a vocabulary are cut into launches, tiles and layers, and what their
// workspaces hold, from their sizes alone (host code; no GPU types, so that the rules can be compiled and checked
// without one).
#pragma once

#include <stdint.h>

#include <algorithm>

#include "mesa_dtypes.hpp"

namespace mesa {
namespace vocab {

inline int64_t ceil_to(int64_t x, int64_t n) { return (x + n - 1) / n * n; }
inline int64_t ceil_div(int64_t x, int64_t n) { return (x + n - 1) / n; }

struct Carve {      // the workspace, piece after piece of 256 bytes
    int64_t at = 0;
    int64_t take(int64_t bytes)
    {
        const int64_t p = at;
        at += ceil_to(bytes, 256);
        return p;
    }
};

// ------------------------------------------------------------------ sums over sorted tokens
constexpr int kTile = 1024;            // tokens a workgroup sorts
constexpr int kDigitBits = 9, kBins = 1 << kDigitBits;
constexpr int kRun = 32;               // pieces of a run

// Sorted positions of a piece: short ones make more waves of few rows, long ones fewer sums to join.  777 rows of 321
// fp32 channels take 14.6 us by 8, 17.6 by 16 and 23.7 by 32, 4096 of 1024 bf16 ones 27.9, 30.1 and 35.8, 16384 of
// 2048 60.0, 55.0 and 57.2 (and all of them one token 204, 126 and 86).
constexpr int kFewPiece = 8, kManyPiece = 16;
constexpr int64_t kFewRows = 8192;
inline int64_t piece_of(int64_t rows) { return rows <= kFewRows ? kFewPiece : kManyPiece; }

// Past so many rows there are runs of pieces.  Up to there a token that is everywhere has 1024 pieces at most: 16384
// rows of 2048 bf16 channels take 55 us, 126 if they are one token, with runs 60 and 55.  65536 of 512 take 77 and
// 333 without runs, 69 and 84 with them.
constexpr int64_t kRunRows = 16384;

struct TokenSumLayout {
    int64_t tiles, ld, hist, keys[2], places[2], entered, left, runs, bytes;
    TokenSumLayout(int64_t rows, int64_t width)
    {
        tiles = (rows + kTile - 1) / kTile;
        ld = ceil_to(width, 8);
        Carve c;
        hist = c.take(tiles * kBins * 4);
        for (int k = 0; k < 2; ++k) keys[k] = c.take(rows * 4), places[k] = c.take(rows * 4);
        // no fewer for more rows: a workspace for many serves fewer
        const int64_t few = std::min(rows, kFewRows), pieces = std::max((rows + piece_of(rows) - 1) / piece_of(rows), (few + kFewPiece - 1) / kFewPiece);
        entered = c.take(pieces * ld * 4);
        left = c.take(pieces * ld * 4);
        runs = rows <= kRunRows ? 0 : c.take(pieces / kRun * ld * 4);
        bytes = c.at;
    }
};

// ------------------------------------------------------------------ the cross entropy's products
constexpr int kStepK = 64;      // rows that the products read are filled up to a multiple of this

constexpr int64_t kUnits = 256;      // compute units of the card
constexpr int64_t kMostTiles = int64_t(UINT32_MAX) / 512;      // of a launch, whose threads are counted in 32 bits

enum Shape { kWide, kMiddle, kNarrow, kThin };
inline int logit_planes(int dtype) { return dtype == kBf16 ? 1 : 2; }
inline int grad_planes(int dtype) { return dtype == kBf16 ? 1 : 3; }
// Rows of the tile (of the table, or channels) and columns (of h, or of the table).  There is a thin one of bf16 and of
// fp32 logits.
constexpr int kTileRows[3][4] = {{256, 128, 64, 64}, {128, 128, 64, 64}, {128, 128, 64, 0}};
constexpr int kTileColumns[3][4] = {{256, 128, 64, 32}, {256, 128, 64, 32}, {256, 128, 64, 0}};
inline int64_t shape_m(Shape s, int planes) { return kTileRows[planes - 1][s]; }
inline int64_t shape_n(Shape s, int planes) { return kTileColumns[planes - 1][s]; }
constexpr int step_of(int planes) { return planes == 1 ? 64 : 32; }      // of k

// What a product takes with each tile shape, in us, fitted to 261 sizes of each type (48 to 4000 rows, 1000 to
// 50257 of the table, 128 to 2048 channels), half of them within 5 to 8 percent.  A tile alone on its compute unit
// takes `alone` + `alone_step` a step of k; where more share a unit they take `shared` + `shared_step` of
// its time each.  The shape of the least cost is 0.4 to 1.1 percent slower than the fastest on average, and more than
// a tenth in 0 to 4 percent of the sizes.  What it decides, in us (256 or 128 x 256, 128, 64 wide): 777 rows by 5003
// of 768, bf16 27, 19, 22 a call, fp32 47, 49, 54; 2000 by 32003 of 768 bf16 108, 125, 180; 300 by 5003 of 768 fp32
// 48, 39, 34.
struct Cost {
    float alone, alone_step, shared, shared_step;
    int per_unit;
};
constexpr Cost kCost[3][3] = {
    {{11.6f, 1.29f, 11.6f, 1.29f, 1}, {6.5f, 0.69f, 3.35f, 0.47f, 2}, {4.4f, 0.44f, 0.84f, 0.196f, 5}},
    {{11.2f, 1.00f, 11.2f, 1.00f, 1}, {9.5f, 0.67f, 4.2f, 0.64f, 2}, {5.8f, 0.375f, 0.92f, 0.307f, 5}},
    {{9.2f, 1.91f, 9.2f, 1.91f, 1}, {5.7f, 1.22f, 5.7f, 1.22f, 1}, {4.3f, 0.62f, 0.90f, 0.40f, 3}}};
constexpr Cost kThinCost = {4.0f, 0.40f, 0.6f, 0.12f, 6};      // of bf16

inline float cost_of(Shape s, int planes, int64_t tiles, int64_t k)
{
    const Cost& c = s == kThin ? kThinCost : kCost[planes - 1][s];
    const float steps = float(ceil_div(k, step_of(planes))), alone = c.alone + c.alone_step * steps, shared = c.shared + c.shared_step * steps;
    const int64_t each = ceil_div(tiles, kUnits), rounds = each / c.per_unit, rest = each % c.per_unit;
    return float(rounds) * std::max(alone, shared * float(c.per_unit)) + (rest > 0 ? std::max(alone, shared * float(rest)) : 0.0f);
}

// How a product of m by n over k is cut: into tiles of a shape and, up to `most`, layers of k whose sums a
// further launch adds up.
struct Cut {
    Shape shape;
    int64_t layers;
};
// Whether a product of fp32 logits, of n rows, takes the table as it lies.
constexpr int kStreamRows = 32;
inline bool streams(int64_t n, int planes) { return planes == 2 && n <= kStreamRows; }
inline Cut cut_of(int64_t m, int64_t n, int64_t k, int planes, int64_t most)
{
    Cut best{kThin, 1};
    if (streams(n, planes)) return best;
    float least = 0.0f;
    for (Shape s : {kWide, kMiddle, kNarrow, kThin}) {
        if (s == kThin && (planes != 1 || n > 32)) continue;      // it reads the table's rows once for 32 of the others
        const int64_t tiles = ceil_div(m, shape_m(s, planes)) * ceil_div(n, shape_n(s, planes));
        for (int64_t l = 1; l <= most; l += l < 4 ? 1 : l / 2) {
            const float sum = l > 1 ? 5.0f + float(l) * float(m) * float(n) * 1e-6f : 0.0f;
            const float t = cost_of(s, planes, tiles * l, ceil_div(k, l)) + sum;
            if (least == 0.0f || t < least) least = t, best = {s, l};
        }
    }
    return best;
}
inline Shape shape_of(int64_t m, int64_t n, int64_t k, int planes) { return cut_of(m, n, k, planes, 1).shape; }

// Of the table's rows that are copied at a time, forward: each time costs two launches whose ends leave the card
// part empty.  One row by 50257 of 1000 bf16 channels, 103 MB of them: 62 us at 64 MiB, 51 in one; 2000 rows by 50257
// of 768 fp32 channels 566, 547 (128 MiB), 527 (256), 524 (in one).
constexpr int64_t kCopyBytes = int64_t(256) << 20;
// And for the gradients, which take a piece of the vocabulary at a time for that too: 64 rows by 128000 of 4096 fp32
// channels, 5.2 GB of planes, 3.65 ms in one piece, 4.16 by 1 GiB, 5.65 by 256 MiB; 256 rows by 50257 of 2048, 1.03 GB, 1.20
// and (256 MiB) 1.48.
constexpr int64_t kGradCopyBytes = int64_t(1) << 30;
// Elements of dz at a time.  16384 rows by 50257 of 2048 bf16 channels: backward 9.41 ms with half as many, 8.60 with
// these, 8.58 with twice, 9.01 with four times; 4096 rows of 768 fp32 channels 4.88, 4.57, 4.53, 4.47.
constexpr int64_t kPieceElements = int64_t(1) << 27;
// What rounding takes off bf16 rows' dz does not even out in sums of few rows.  Up to so many rows, or products, dz has its
// rounding's rest behind it as rows of their own, and h once more, for the table's gradient: its error is its own
// rounding's, 0.0017 of its norm, for 0.0027 at 3 rows by 20000 of 768 to 1024 channels, 0.0025 at 100, 0.0024 at 1000.  That
// doubles the product: the backward call takes 40 us for 36.5 at 256 rows by 5003 of 768, 368 for 308 by 50257 of 2048.
// Of more the target's element alone, which is most of it, gets its rest back, summed over the sorted rows of each target:
// 0.0017 as well where the probabilities are spread (0.0020 without at 3997 rows by 32003 of 1000), at most 0.0024 where other
// elements of dz are as large.  Sorting and summing are launches: a training pass over 1500 rows by 1000 of 128
// takes 47 us with all of the rest, 60 with the target's, over 1100 by 5003 of 768 106 and 110, 2048 by 5003 of 768 161
// and 159, backward over 2000 by 32003 of 1000 609 and 475, 2048 by 50257 of 2048 1742 and 1285.
constexpr int64_t kTwiceRows = 1024;
constexpr float kTwiceProducts = 4.3e9f;
inline bool keeps_all_rest(int64_t rows, int64_t vocab, int64_t width)
{
    return rows <= kTwiceRows || float(rows) * float(vocab) * float(width) <= kTwiceProducts;
}
constexpr int64_t kSlabBytes = int64_t(256) << 20;     // of fp32 layers of one product, at most (or one layer)

// Rows of the table in a piece of the forward, where it has to be copied.
inline int64_t copy_rows(int64_t vocab, int64_t width, int dtype)
{
    const int64_t row = ceil_to(width, kStepK) * 2 * logit_planes(dtype);
    return std::min(ceil_to(vocab, 256), std::max<int64_t>(256, kCopyBytes / row / 256 * 256));
}

// Exponents of n rows, which are read up to the end of the last tile.
inline int64_t exponents_of(int64_t n) { return ceil_to(n, 256) + 256; }

struct ForwardPlan {
    int64_t part, best_z, best_v, at, h, h_parts, table, h_e, table_e, bytes;
    ForwardPlan(int64_t rows, int64_t vocab, int64_t width, int dtype)
    {
        // whether the table is copied hangs on its address, so there is room for either way's tiles
        const int planes = logit_planes(dtype);
        const int64_t copied = streams(rows, planes) ? 0 : copy_rows(vocab, width, dtype);
        auto tiles_of = [&](int64_t m) { return ceil_div(vocab, shape_m(shape_of(m, rows, width, planes), planes)); };
        const int64_t tiles = std::max(tiles_of(vocab), tiles_of(copied));
        Carve c;
        const int64_t row = ceil_to(width, kStepK) * 2 * planes;
        part = c.take(tiles * rows * 8);
        best_z = c.take(tiles * rows * 4);
        best_v = c.take(tiles * rows * 4);
        at = c.take(rows * 4);
        const bool halves = planes > 1 && !streams(rows, planes);
        h = planes == 1 || halves ? c.take(rows * row) : 0;
        h_parts = streams(rows, planes) ? c.take(rows * ceil_to(width, kStepK) * 6) : 0;
        table = c.take(copied * row);
        h_e = halves ? c.take(exponents_of(rows) * 4) : 0;
        table_e = halves ? c.take(exponents_of(copied) * 4) : 0;
        bytes = c.at;
    }
};

// Whether the products may read a table where it lies; whether they do hangs on its address and stride.
inline bool may_lie(int64_t width, int dtype) { return dtype == kBf16 && width % kStepK == 0; }

struct GradPlan {
    // h and the table as the gradients' products read them, and (fp32) as the logits' does, with the exponents
    int64_t piece, dz, dz_rows, deep, dz_ld, h, table, h16, table16, h_e, table_e, rest, slab_h, slab_e, order, sums, at, bytes, ld;
    Shape logits;
    Cut dh, de, de_last;
    bool sorts;      // the table's gradient gets the targets' rests, from sorted targets
    // copied: of a table that the products cannot read where it lies
    GradPlan(int64_t rows, int64_t vocab, int64_t width, int dtype, bool copied)
    {
        const int planes = grad_planes(dtype);
        const bool halves = planes > 1 && !streams(rows, logit_planes(dtype));      // of the table, for the logits
        ld = ceil_to(width, kStepK);
        dz_rows = ceil_to(rows, 64);
        const bool all_rest = keeps_all_rest(rows, vocab, width);
        deep = planes == 1 && all_rest ? 2 * dz_rows : dz_rows;
        piece = std::max<int64_t>(256, kPieceElements / deep / 256 * 256);
        const int64_t row = ld * (2 * planes + (halves ? 4 : 0));
        if (copied) piece = std::min(piece, std::max<int64_t>(256, kGradCopyBytes / row / 256 * 256));
        // pieces of about the same size, and whose part of the table's gradient is whole rounds of wide tiles on all
        // compute units, where they are large enough for that
        const int64_t round = std::max<int64_t>(1, kUnits / ceil_div(width, shape_m(kWide, planes))) * shape_n(kWide, planes);
        if (vocab <= piece)
            piece = ceil_to(vocab, 256);
        else
            piece = piece >= round ? ceil_to(ceil_div(vocab, ceil_div(vocab, piece / round * round)), round)
                                   : ceil_to(ceil_div(vocab, ceil_div(vocab, piece)), 256);
        dz_ld = piece;
        logits = shape_of(piece, rows, width, logit_planes(dtype));
        dh = layers(width, rows, std::min(piece, vocab), planes);
        // the last piece may be much shorter, and is then cut otherwise
        const int64_t ending = vocab - (ceil_div(vocab, piece) - 1) * piece;
        de = layers(width, std::min(piece, vocab), deep, planes);
        de_last = layers(width, ending, deep, planes);
        Carve c;
        h = c.take(deep * ld * 2 * planes);
        table = copied ? c.take(piece * ld * 2 * planes) : 0;
        h16 = halves ? c.take(dz_rows * ld * 4) : h;
        table16 = halves ? c.take(piece * ld * 4) : table;
        h_e = halves ? c.take(exponents_of(dz_rows) * 4) : 0;
        table_e = halves ? c.take(exponents_of(piece) * 4) : 0;
        rest = planes == 1 ? c.take(rows * 4) : 0;
        dz = c.take(deep * dz_ld * 2 * planes);
        slab_h = dh.layers > 1 || piece < vocab ? c.take(dh.layers * rows * ld * 4) : 0;
        const int64_t layered = std::max(de.layers > 1 ? de.layers * std::min(piece, vocab) : 0, de_last.layers > 1 ? de_last.layers * ending : 0);
        slab_e = layered > 0 ? c.take(layered * ld * 4) : 0;
        sorts = planes == 1 && !all_rest;
        order = sorts ? c.take(TokenSumLayout(rows, width).bytes) : 0;
        sums = sorts ? c.take(rows * ld * 4) : 0;
        at = sorts ? c.take(vocab * 4) : 0;
        bytes = c.at;
    }
    // Layers have at least eight steps of 64, and there is room for their sums.
    static Cut layers(int64_t m, int64_t n, int64_t k, int planes)
    {
        return cut_of(m, n, k, planes, std::max<int64_t>(1, std::min(ceil_div(k, kStepK) / 8, kSlabBytes / (ceil_to(m, kStepK) * n * 4))));
    }
};
inline int64_t grad_bytes(int64_t rows, int64_t vocab, int64_t width, int dtype)
{
    const int64_t copied = GradPlan(rows, vocab, width, dtype, true).bytes;
    return may_lie(width, dtype) ? std::max(copied, GradPlan(rows, vocab, width, dtype, false).bytes) : copied;
}

}  // namespace vocab
}  // namespace mesa
