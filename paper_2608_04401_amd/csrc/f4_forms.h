// Which form a product with 4-bit weights takes (f4.hip): streamed as they are, and with which tile, or
// converted for the dense forms.  Usable from host code without HIP (for tests).
#pragma once

#include <utility>

#include "forms.h"

namespace elb {

constexpr int kMostShares = 16, kMostSharing = 512;  // shares of a tile, blocks of tiles with shares
constexpr int64_t kStreamedAlways = 64;
constexpr int64_t most_streamed(bool f32) { return f32 ? 8192 : 2048; }  // tokens

// The tile and waves of a streamed product, in how many shares its contraction is cut, and its
// estimated time: start + rounds (round + iter * units of a wave) [+ share] us, with rounds of `per` blocks
// on each of 256 compute units.  The constants are least-squares fits to 1494 measured products (1 to
// 768 tokens, weights of 1024 to 16384 rows of 512 to 8192 values); over these sizes the choice, with
// that of converting the weights, is 0.3 % slower than the best on average and 18 % at worst (fp32, 384
// tokens, 512 to 4096: 31.9 for 27.1).  bf16, us, at both sides: 48 tokens, 8192 to 2048: 48 x 32 tiles
// in four shares 10.7, whole 15.1, 48 x 64 in four 12.9, whole 21.2; 2048 to 16384: 48 x 64 9.3, 32 x 64
// 13.1, 48 x 32 11.2.
struct StreamForm {
    int tm, nf, nw, per;
    float start, round, iter, share;
    int shares = 1;
    float time = 0;
};
constexpr StreamForm kStreamBf16[] = {
    {8, 1, 16, 1, 1.31f, 2.15f, 1.29f, 3.68f}, {8, 2, 8, 2, 1.75f, 1.75f, 0.91f, 3.12f},
    {16, 1, 8, 1, 1.5f, 1.56f, 0.84f, 3.31f},  {16, 2, 8, 1, 1.34f, 1.87f, 1.08f, 3.32f},
    {16, 4, 8, 1, 1.75f, 1.75f, 1.8f, 3.14f},  {32, 2, 4, 1, 1.53f, 1.43f, 1.2f, 3.5f},
    {32, 4, 4, 1, 1.21f, 2.13f, 1.82f, 4.12f}, {48, 2, 4, 1, 1.39f, 1.65f, 1.57f, 4.31f},
    {48, 4, 4, 1, 0.97f, 2.54f, 2.3f, 5.2f}};
constexpr StreamForm kStreamF32[] = {
    {8, 1, 8, 1, 1.25f, 1.83f, 2.0f, 3.44f},   {8, 2, 8, 1, 1.22f, 2.05f, 2.46f, 3.41f},
    {8, 4, 8, 1, 1.69f, 1.69f, 3.59f, 3.15f},  {16, 1, 4, 1, 1.5f, 1.45f, 1.46f, 3.3f},
    {16, 2, 4, 1, 1.51f, 1.39f, 2.01f, 3.42f}, {16, 4, 4, 1, 1.22f, 1.79f, 2.78f, 3.5f},
    {32, 2, 4, 1, 1.4f, 1.61f, 3.28f, 3.7f}};
// (gate and up rows are two fragments at least, and of fp32 tokens 32 x 32 tiles are the best for none)
constexpr bool pair_takes(const StreamForm& f, bool f32) {
    return f.nf > 1 && !(f32 && f.tm == 32);
}

// Calls call(Tile<tm, nf, nw>) for a form of the table, so that what is planned is what is launched; false
// for a form that is not of it (PAIR: or that gate and up rows do not take).
template <int TM_, int NF_, int NW_>
struct Tile {
    static constexpr int TM = TM_, NF = NF_, NW = NW_;
};
template <bool F32, bool PAIR, size_t I, class Call>
bool call_form(const StreamForm& form, Call&& call) {
    constexpr StreamForm t = (F32 ? kStreamF32 : kStreamBf16)[I];
    if constexpr (!PAIR || pair_takes(t, F32)) {
        if (form.tm == t.tm && form.nf == t.nf && form.nw == t.nw) {
            call(Tile<t.tm, t.nf, t.nw>{});
            return true;
        }
    }
    return false;
}
template <bool F32, bool PAIR, class Call, size_t... I>
bool with_form(const StreamForm& form, Call&& call, std::index_sequence<I...>) {
    return (call_form<F32, PAIR, I>(form, call) || ...);
}
template <bool F32, bool PAIR, class Call>
bool with_form(const StreamForm& form, Call&& call) {
    constexpr size_t n = F32 ? sizeof(kStreamF32) / sizeof(kStreamF32[0])
                             : sizeof(kStreamBf16) / sizeof(kStreamBf16[0]);
    return with_form<F32, PAIR>(form, call, std::make_index_sequence<n>{});
}

inline int stream_tiles(const StreamForm& f, int64_t T, int rows) {
    return (rows + 16 * f.nf - 1) / (16 * f.nf) * (int)((T + f.tm - 1) / f.tm);
}
inline StreamForm stream_form(int64_t T, int cols, int k, bool pair, bool f32) {
    const int rows = pair ? 2 * cols : cols, units = (k + 255) / 256;
    const StreamForm* const table = f32 ? kStreamF32 : kStreamBf16;
    const int n = f32 ? (int)(sizeof(kStreamF32) / sizeof(kStreamF32[0]))
                      : (int)(sizeof(kStreamBf16) / sizeof(kStreamBf16[0]));
    const StreamForm* best = nullptr;
    int best_shares = 1;
    float least = 0;
    for (int i = 0; i < n; ++i) {
        const StreamForm& f = table[i];
        // (where the fits hold)
        if ((f.tm == 8 && T > 8) || (f.tm == 16 && T > 16 && !f32) || (f.tm > 16 && T <= 16) ||
            (pair && !pair_takes(f, f32)))
            continue;
        const int tiles = stream_tiles(f, T, rows);
        for (int z = 1; z <= (pair ? 1 : kMostShares); z *= 2) {
            if (z > 1 && (z * f.nw > units || tiles > kMostSharing / z)) break;
            const unsigned per = 256u * f.per, rounds = ((unsigned)tiles * z + per - 1) / per;
            const unsigned its = (unsigned)(units + f.nw * z - 1) / (unsigned)(f.nw * z);
            const float t = f.start + (float)rounds * (f.round + f.iter * (float)its) +
                            (z > 1 ? f.share : 0.0f);
            if (!best || t < least) best = &f, best_shares = z, least = t;
        }
    }
    StreamForm f = *best;
    f.shares = best_shares;
    f.time = least;
    return f;
}

// Whether the product [T, k] x [n, k] (block: the dense block of width n and h of width k) streams its
// weights, by estimated time, or converts them first (the bytes at 5 TB/s, then the best dense form, and
// 6 us for the launch and the dense form's reads of what was just written).  us, streamed / converted,
// bf16: 256 tokens, 2048 to 8192 22 / 34, 384 29 / 35, 768 58 / 50; 8192 to 2048 384 23 / 38, 512
// 34.3 / 35.9, 2048 118 / 75; fp32, whose three bf16 products take less than one of fp32: 512 tokens,
// 8192 to 2048 96 / 179, 2048 to 8192 4096 918 / 1064, 16384 4101 / 4161, but 512 to 4096 4096 264 / 158.
// Up to kStreamedAlways tokens nothing is converted, so that small batches need no scratch for it.
struct F4Plan {
    bool streams;
    StreamForm up, form;  // of a block's gate and up rows; of the projection, or of its down rows
    int tiles;            // of `form`
    size_t part;          // bytes of its partial sums and, behind them, a counter a tile (shares > 1)
    size_t sums() const { return part - 4 * (size_t)tiles; }
};
inline size_t f4_part(const StreamForm& f, int tiles) {
    if (f.shares == 1) return 0;
    return (size_t)tiles * ((size_t)f.shares * ((f.tm + 15) / 16 * 16) * 16 * f.nf * 4 + 4);
}
inline F4Plan f4_plan(int64_t T, int n, int k, bool block, bool f32) {
    F4Plan p{T <= kStreamedAlways, {}, {}, 0, 0};
    if (T > most_streamed(f32)) return p;
    p.form = stream_form(T, n, k, false, f32);
    if (block) p.up = stream_form(T, k, n, true, f32);
    auto converted = [&](int64_t rows, int64_t deep) {
        const int64_t e = f32 ? 4 : 2, kt = (deep * e + 127) / 128;
        const FormId f = pick_form(T, rows, kt, f32, true);
        const FormCost& c = (f32 ? kFormCostsF32 : kFormCosts)[f];
        return 6.0f + (float)(rows * deep) * (0.53f + (float)e) / 5e6f +
               form_time(c, form_tiles(c, T, rows), kt, f != kTiles);
    };
    if (!p.streams) {
        const float c = converted(n, k) + (block ? converted(2 * (int64_t)k, n) : 0.0f);
        p.streams = p.form.time + (block ? p.up.time : 0.0f) < c;
    }
    if (p.streams) {
        p.tiles = stream_tiles(p.form, T, n);
        p.part = f4_part(p.form, p.tiles);
    }
    return p;
}

// The most partial sums that any batch of up to T tokens needs: the form is the same within every 16
// tokens but the first, whose halves differ.
inline size_t f4_part_reserve(int64_t T, int n, int k, bool f32) {
    size_t most = 0;
    for (int64_t t = 8; t < T + 16 && t <= most_streamed(f32); t += t == 8 ? 8 : 16) {
        const int64_t at = t < T ? t : T;
        if (at < 1) break;
        const StreamForm f = stream_form(at, n, k, false, f32);
        const size_t b = f4_part(f, stream_tiles(f, at, n));
        most = b > most ? b : most;
    }
    return most;
}

}  // namespace elb
