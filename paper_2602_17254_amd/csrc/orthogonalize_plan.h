// Which kernels a call of trivance_orthogonalize takes, by its sizes alone: host code without HIP, so that it can
// be looked over without a GPU.
#pragma once

#include <cmath>
#include <cstdint>
#include <initializer_list>

namespace trivance {

constexpr int kSmallSide = 64, kSmallLong = 256;  // X of one workgroup, or of one strip
constexpr int kMostStrips = 32;
constexpr int kMostWorkers = 256;  // that share a symmetric product

// The tiles of a call: of the symmetric products and of the others. Sides are padded to the larger.
struct Tiles {
    int symmetric, update;
    int pad() const { return symmetric > update ? symmetric : update; }
};

inline int64_t padded(int64_t side, int tile) { return (side + tile - 1) / tile * tile; }

// Over how many workgroups a symmetric product's stages are shared out; 0: a workgroup takes a tile. It leaves
// no CU idle, and costs a launch and the parts' way through memory, 6 to 14 us. With tiles of 128 the
// idle CUs of the last round decide: a round takes 30 us for 1000 values of the summed index. 136 tiles from
// 2048 measured 60 us as they are and 53 shared out, from 8192 200 and 130. Tiles of 64 take 0.4 us for 64
// values; a worker has 128 or more.
inline int workers_of(int tile, int64_t tiles, int64_t depth) {
    const int64_t all = tiles * (depth / 64);
    if (all > INT32_MAX / 2) return 0;
    const double rounds = tiles / 256.0;
    if (tile == 128) return all >= kMostWorkers && (std::ceil(rounds) - rounds) * depth >= 512.0 ? kMostWorkers : 0;
    if (tile != 64 || all < 4) return 0;
    const int64_t w = all / 2 < kMostWorkers ? all / 2 : kMostWorkers;
    return 0.4 * all / w + 6.0 < 0.4 * std::ceil(rounds) * (depth / 64) ? (int)w : 0;
}

// The pair that takes the least time by the measured rates, counting whole rounds of the 256 CUs and the
// padding.
inline Tiles tiles_of(int64_t batch, int64_t m, int64_t n) {
    const auto cost = [&](int tile, int64_t tiles, int64_t depth, bool symmetric) {
        const double rate = tile == 256 ? 1.0 : tile == 128 ? 0.76 : 0.5;
        const bool share = symmetric && workers_of(tile, batch * tiles, depth);
        const double rounds = share ? batch * tiles / 256.0 : (double)((batch * tiles + 255) / 256);
        // in units of 1/720000 us; the second launch of shared products takes 10 us
        return rounds * tile * tile * depth / rate + (share ? 7.2e6 : 0.0);
    };
    Tiles best{64, 64};
    double least = INFINITY;
    for (const int s : {64, 128})
        for (const int u : {64, 128, 256}) {
            if (u == 256 && m <= 128) continue;  // half of every tile and more would be padding
            const Tiles t{s, u};
            const int64_t pm = padded(m, t.pad()), pn = padded(n, t.pad());
            const int64_t ms = pm / s, half = ms * (ms + 1) / 2;
            const double c = cost(s, half, pn, true) + cost(s, half, pm, true) + cost(u, pm / u * (pn / u), pm, false);
            if (c < least) {
                least = c;
                best = t;
            }
        }
    return best;
}

// How a product runs.
struct ProductForm {
    int tile;
    bool few;       // tiles of 64, at most one for each CU: with 16 waves
    int64_t tiles;
    int workers;    // that share its stages; 0: a workgroup takes a tile
};

// Of a product over all matrices: rows x cols of C (whole tiles) summed over `depth` values.
inline ProductForm form_of(int64_t batch, int64_t rows, int64_t cols, int64_t depth, int tile, bool symmetric) {
    const int64_t r = rows / tile, c = cols / tile, tiles = batch * (symmetric ? r * (r + 1) / 2 : r * c);
    return {tile, tile == 64 && tiles <= 256, tiles, symmetric ? workers_of(tile, tiles, depth) : 0};
}

}  // namespace trivance
