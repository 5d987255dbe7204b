// Which block form a dense product takes (dense.h): the one whose estimated time is least,
//     start + rounds (round + iter * iterations)   [us]
// with rounds = tiles / 256 compute units, rounded up (one block per unit at a time; the fp32 tile
// form, three per unit, not rounded), and iterations = k-tiles / ways, rounded up.  The constants are
// least-squares fits over products of 16 .. 4096 rows, 512 .. 8192 columns and 4 .. 64 k-tiles; the
// times at both sides of the choice, us:
//   512 rows, 2048 columns, int8 k = 2048:  64 x 64 split 7.5, pairs 11.5, turns 26.3;
//   2048 rows: 24.8, 14.1, 28.3;  2048 rows, 8192 columns: 89.8, 52.9, 38.2;
//   64 rows, 2048 columns: 32 x 32 split 4.9, 32 x 64 5.9, 64 x 64 6.8, 16 x 16 (two rounds) 7.6.
//   4096 rows, 2048 columns (128 turns tiles, 512 pairs tiles): bf16 of 128 k-tiles pairs 146,
//   halves 126, of 256 k-tiles 303 and 228; int8 of 64 k-tiles pairs 72, halves 85.
// Halves win over several rounds of the chip too where the contraction is long (us, halves / best other):
// bf16 320 tiles of 256 k-tiles 578 / 690, of 448 970 / 1378, 384 of 256 634 / 679, 640 of 448 1704 /
// 1790; int8 320 of 512 1122 / 1447; near the choice the two are level (384 of 192 491 / 495).
// Over 144 such products the choice (without halves) is 0.3 % slower than the best form on average,
// 13 % at worst, and between pairs and turns over 72 larger ones 0.4 % and 9 %.  fp32: 0.4 % and 10 %
// over 128 products, 1.0 % and 15 % over 54 others (512 rows, 2048 columns, 64 k-tiles: tiles 43.3,
// 64 x 64 split 37.6).  The fp32 tile form's time is met within 10 % at whole rounds of 256 tiles and
// is up to 1.8 times the estimate just above one (272 tiles of 32 k-tiles 38.4, estimated 21.5), where
// the other forms take as long (37 to 41).
// Usable from host code without HIP (for tests).
#pragma once

#include <stddef.h>
#include <stdint.h>

namespace elb {

enum FormId {
    kSplit16x16, kSplit16x32, kSplit16x64, kSplit32x32, kSplit32x64, kSplit64x64,
    kPairs,  // 128 x 128, two groups of waves taking the k-tiles in turn (bf16, int8)
    kTurns,  // 256 x 256, two groups of waves taking turns at the units (bf16, int8)
    kHalves, // the same, two blocks per tile, half of the contraction each (bf16, int8)
    kTiles,  // 64 x 64 (fp32); 128 x 128 for tensors off a 16-byte boundary (bf16, int8)
    kForms
};

struct FormCost {
    int tm, tn, ways;  // ways: k-tiles in work at a time
    float start, round, iter;
    int blocks = 1;    // per tile
};

// bf16 and int8: a k-tile's copies, LDS reads and matrix cycles are the same
constexpr FormCost kFormCosts[kForms] = {
    {16, 16, 8, 1.7f, 2.5f, 0.32f},  {16, 32, 8, 1.55f, 2.5f, 0.46f},
    {16, 64, 4, 1.4f, 2.45f, 0.37f}, {32, 32, 8, 1.4f, 2.4f, 0.60f},
    {32, 64, 4, 1.35f, 2.8f, 0.45f}, {64, 64, 4, 1.25f, 3.3f, 0.59f},
    {128, 128, 2, 0.0f, 5.4f, 0.76f}, {256, 256, 1, 0.0f, 9.2f, 1.05f},
    {256, 256, 2, 0.0f, 30.f, 1.10f, 2}, {0, 0, 0, 0, 0, 0}};
constexpr FormCost kFormCostsF32[kForms] = {
    {16, 16, 8, 1.75f, 2.95f, 0.38f}, {16, 32, 8, 1.7f, 2.95f, 0.65f},
    {16, 64, 4, 1.5f, 2.8f, 0.66f},   {32, 32, 8, 1.55f, 2.85f, 1.17f},
    {32, 64, 4, 1.35f, 3.25f, 1.14f}, {64, 64, 4, 1.15f, 3.65f, 2.09f},
    {0, 0, 0, 0, 0, 0},               {0, 0, 0, 0, 0, 0},
    {0, 0, 0, 0, 0, 0},               {64, 64, 1, 2.6f, 1.15f, 0.52f}};

inline int64_t form_tiles(const FormCost& f, int64_t rows, int64_t cols) {
    return ((rows + f.tm - 1) / f.tm) * ((cols + f.tn - 1) / f.tn);
}

inline float form_time(const FormCost& f, int64_t tiles, int64_t ktiles, bool whole_rounds) {
    const int64_t n = tiles * f.blocks;
    const float r = n <= 256 ? 1.0f : whole_rounds ? (float)((n + 255) / 256) : (float)n / 256.0f;
    return f.start + r * (f.round + f.iter * (float)((ktiles + f.ways - 1) / f.ways));
}

// the form for a rows x cols product (cols: rows of the second operand) of that many k-tiles;
// with fp32 set, of fp32; halves: whether there is scratch for kHalves (halves_bytes)
inline FormId pick_form(int64_t rows, int64_t cols, int64_t ktiles, bool fp32, bool halves) {
    int best = -1;
    float least = 0;
    for (int i = 0; i < kForms; ++i) {
        const FormCost& f = (fp32 ? kFormCostsF32 : kFormCosts)[i];
        if (!f.ways || (i == kHalves && !halves)) continue;
        const float t = form_time(f, form_tiles(f, rows, cols), ktiles, i != kTiles);
        if (best < 0 || t < least) best = i, least = t;
    }
    return (FormId)best;
}

// Two products of one contraction in one launch, both operands down the rows (the weight gradients):
// split 32 x 32 or 64 x 64, or the large forms.  The split forms are for small layers (tiles few,
// contraction long): us, large tiles / split: fp32 256 tokens, d = 128, m = 256 8.4 / 5.2, 2000 tokens,
// d = 128, m = 64 61 / 14, bf16 16384 tokens, d = m = 256 114 / 41.
inline FormId pick_form2(int64_t rows1, int64_t cols1, int64_t rows2, int64_t cols2, int64_t ktiles,
                         bool fp32) {
    auto time = [&](FormId i) {
        const FormCost& f = (fp32 ? kFormCostsF32 : kFormCosts)[i];
        return form_time(f, form_tiles(f, rows1, cols1) + form_tiles(f, rows2, cols2), ktiles,
                         i != kTiles);
    };
    FormId large = kTiles;
    float than;
    if (fp32) {
        // read down the rows, the tiles take 1.0 (many rounds) to 1.8 times (one) their estimate;
        // with 1.35 the choice over 30 products of 256 .. 4096 tokens is 3 % slower than the best on
        // average: 512 tokens, d = m = 512 split 13.8 us, tiles 18.0; 256 tokens, d = 2048, m = 1024
        // 47.3, 35.0; at worst 39 %, 256 tokens, d = m = 1024, split 26.4, tiles 19.1
        than = 1.35f * time(kTiles);
    } else {
        const float pairs = time(kPairs), turns = time(kTurns);
        large = pairs <= turns ? kPairs : kTurns;
        than = pairs < turns ? pairs : turns;
    }
    const float t32 = time(kSplit32x32), t64 = time(kSplit64x64);
    if (t32 >= than && t64 >= than) return large;
    return t32 <= t64 ? kSplit32x32 : kSplit64x64;
}

// Whether an int8 product of float rows of K values quantises them itself, where it takes form f: one
// of few rows, and rows that a wave keeps in registers, several at a time.  (The rows' count is no
// term of it: see the times of both sides at QuantForm.)
constexpr int kFusedK = 2048;
inline bool form_quantises(FormId f, int64_t K) { return f <= kSplit32x32 && K <= kFusedK; }

// scratch of a product that may take kHalves: per tile the two blocks' fp32 (int32) partial tiles,
// then a counter; 0 where another form is picked
constexpr int64_t kPartialBytes = 256 * 256 * 4;
inline size_t halves_bytes(int64_t rows, int64_t cols, int64_t ktiles, bool fp32) {
    if (pick_form(rows, cols, ktiles, fp32, true) != kHalves) return 0;
    return (size_t)form_tiles(kFormCosts[kHalves], rows, cols) * (2 * kPartialBytes + 4);
}

// More tiles than this never take kHalves: over q whole rounds of 256 turns tiles and up to half of
// another, 2 q + 1 half rounds of halves cost less only from (50.8 q + 20.8) / (0.5 - 0.05 q) k-tiles
// on, 42 for q = 0, 159 for 1, 9560 for 9 and nowhere for 10.
constexpr int64_t kHalvesMost = 9 * 256 + 128;

// The most that halves_bytes is for any number of rows up to this one: what a caller reserves for
// batches of up to that size.  Within 256 rows the halves' time stays and the others' do not fall, so
// that the last of them tells.
inline size_t halves_reserve(int64_t rows, int64_t cols, int64_t ktiles, bool fp32) {
    // where one tile is no faster, no number of them is: their rounds are no fewer
    if (fp32 || form_time(kFormCosts[kHalves], 1, ktiles, true) >=
                    form_time(kFormCosts[kTurns], 1, ktiles, true))
        return 0;
    const int64_t nt = (cols + 255) / 256, most = kHalvesMost / nt;
    for (int64_t mt = (rows + 255) / 256 < most ? (rows + 255) / 256 : most; mt > 0; --mt)
        if (size_t n = halves_bytes(rows < 256 * mt ? rows : 256 * mt, cols, ktiles, false))
            return n;
    return 0;
}

}  // namespace elb
