// How a linear layer with block scales is laid out on the SMs: host code without CUDA, so that it can be tested anywhere.
#pragma once

#include <stdint.h>

namespace w4a8 {

constexpr int kBlocksSmemMax = 232448;

struct BlocksPlan {
    bool pair;     // CTA pairs: tiles of 256 tokens x 256 channels
    int tmax;      // tokens that the kernel's registers are laid out for: 16, 32, 64, 128
    int tokens;    // tokens of a tile at most
    int cut;       // CTAs that share a tile's K
};

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// rows of x8, over `experts` (1: a single layer, whose rows all use it).  The loads of the experts are not known on the host: an
// expert is expected to have up to four times the average.
inline BlocksPlan blocks_plan(int64_t rows, int64_t experts, int64_t N, int64_t K, int sms) {
    BlocksPlan pl;
    const int64_t KB = ceil_div(K, 128), NB = ceil_div(N, 128);
    int64_t load = rows;
    if (experts > 1) {
        load = 4 * ceil_div(rows, experts) + 12;
        if (load > rows) load = rows;
    }
    pl.pair = rows > 128 * experts;
    if (pl.pair) {
        pl.tmax = 0;
        pl.tokens = 256;
        pl.cut = 1;
        return pl;
    }
    pl.tmax = load <= 16 ? 16 : load <= 32 ? 32 : load <= 64 ? 64 : 128;
    pl.tokens = load >= 128 ? 128 : (int)ceil_div(load, 16) * 16;
    int64_t tiles = NB * ceil_div(rows, pl.tokens);
    if (experts > 1) {
        const int64_t full = rows / pl.tokens, with_rows = experts < rows ? experts : rows;
        tiles = NB * (full > with_rows ? full : with_rows);
    }
    // A CTA's time for a tile: its k-blocks at the SM's share of HBM, and a start and an end; the exchange in a cluster.
    pl.cut = 1;
    double best = 1e30;
    for (int cut = 1; cut <= 8 && cut <= KB; ++cut) {
        const int64_t clusters = sms / cut;
        if (clusters < 1) break;
        const int64_t rounds = ceil_div(tiles, clusters);
        const double t = (double)rounds * ((double)ceil_div(KB, cut) * 0.35 + (cut > 1 ? 1.0 : 0.3));
        if (t < best * 0.97) {
            best = t;
            pl.cut = cut;
        }
    }
    return pl;
}

}  // namespace w4a8
