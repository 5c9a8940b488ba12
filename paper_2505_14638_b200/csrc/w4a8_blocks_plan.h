// How a linear layer with block scales is laid out on the SMs: host code (and what the kernel shares with it) without CUDA, so that
// it can be tested anywhere.
#pragma once

#include <math.h>
#include <stdint.h>

#ifdef __CUDACC__
#define W4A8_BOTH __host__ __device__
#else
#define W4A8_BOTH
#endif

namespace w4a8 {

constexpr int kBlocksSmemMax = 232448;       // of a block
constexpr int kBlocksSmemHalf = 115712;      // of two blocks on an SM, each
constexpr int kBlocksMaxStages = 16, kBlocksBuffers = 4;
constexpr int kBlocksChunk = 8;              // k-blocks whose activation scales are fetched at a time
constexpr int kBlocksBars = 2 * kBlocksMaxStages + 2 * kBlocksBuffers + 2 + 2 + 1;
constexpr int kBlocksTableBytes = 2 * 513 * 4 + 32;

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Shared memory of linear_blocks_kernel behind a 1024-byte boundary: the ring, and from where on the rest lies.
struct BlocksSmem {
    int bars, scales, table, parts, end;
};
W4A8_BOTH inline BlocksSmem blocks_smem(int tmax, int channels, int tokens, int stages, int cut, int share, int part_buffers, bool grouped) {
    BlocksSmem s;
    const int ring = stages * (channels * 128 + (tokens + 31) / 32 * 4096);
    s.bars = ring;
    s.scales = s.bars + (8 * kBlocksBars + 8 + 15) / 16 * 16;
    s.table = s.scales + 2 * 2 * kBlocksChunk * tmax * 4;
    s.parts = s.table + (grouped ? (kBlocksTableBytes + 15) / 16 * 16 : 0);
    s.end = s.parts + part_buffers * cut * tokens * share * 4;
    // (an MMA reads 128 rows from where a stage's weights begin, the last stage's too)
    const int read = ring - (channels * 128 + (tokens + 31) / 32 * 4096) + 16384;
    if (s.end < read) s.end = read;
    return s;
}

struct BlocksPlan {
    bool wide;         // tiles of 128 tokens x 256 channels
    int tmax;          // tokens that the kernel's registers are laid out for: 16, 32, 64, 128
    int tokens;        // tokens of a tile at most
    int channels;      // channels of a tile
    int cut, share;    // CTAs that share a tile's K, and channels that each of them writes, at most
    int part_buffers;
    int stages, smem;
    int ctas;          // per SM
    int64_t tiles;     // (expected, where there are several experts)
};

// The ring's depth, and the shared memory, for `rounds` tiles per CTA; false where a plan does not fit.
inline bool blocks_fit(BlocksPlan* pl, int64_t rounds, bool grouped) {
    if (pl->channels < 8 * pl->cut) return false;   // (at least eight channels each)
    pl->share = (int)(ceil_div(pl->channels / 8, pl->cut) * 8);
    const int most = pl->ctas == 2 ? kBlocksSmemHalf : kBlocksSmemMax;
    for (pl->part_buffers = rounds > 1 ? 2 : 1; pl->part_buffers >= 1; --pl->part_buffers)
    {
        const int stage = pl->channels * 128 + (pl->tokens + 31) / 32 * 4096;
        const int fixed = 1024 + blocks_smem(pl->tmax, pl->channels, pl->tokens, 4, pl->cut, pl->share, pl->part_buffers, grouped).end - 4 * stage;
        pl->stages = (most - fixed) / stage;   // (at most one too many or too few: the end of a short ring may be further off)
        if (pl->stages > kBlocksMaxStages) pl->stages = kBlocksMaxStages;
        for (; pl->stages >= 4; --pl->stages) {
            pl->smem = 1024 + blocks_smem(pl->tmax, pl->channels, pl->tokens, pl->stages, pl->cut, pl->share, pl->part_buffers, grouped).end;
            if (pl->smem <= most) return true;
        }
    }
    return false;
}

// rows of x8, over `experts` (1: a single layer, whose rows all use it).  The loads of the experts are not known on the host: the plan
// takes each row to go to any of them, and an expert to have up to four times the average.
//
// Costs are in units of an SM's share of HBM for a k-block of 128 channels (16 KB, 0.37 us), without what every launch takes.
// Measured, us, tiles of up to 128 channels / of 256: (128, 4096, 4096) 11.6 / 21.6, (77, 14336, 4096) 19.7 / 22.5, (128, 28672, 8192)
// 78.0 / 50.6, (256, 14336, 4096) 38.1 / 24.0, (512, 4096, 4096) 20.8 / 21.2, (1024, 4096, 4096) 37.5 / 22.0; 64 experts of (4096,
// 2048) with 32, 64, 128 rows each 133 / 98, 166 / 108, 256 / 134; 128 of (6928, 896) with 6 rows each 194 / 143, of (4096, 4096) with 4
// rows each 291 / 309.
inline BlocksPlan blocks_plan(int64_t rows, int64_t experts, int64_t N, int64_t K, int sms, bool grouped) {
    const int64_t KB = ceil_div(K, 128);
    int64_t with_rows = 1, load = rows;
    if (experts > 1) {
        with_rows = (int64_t)((double)experts * -expm1((double)rows * log1p(-1.0 / (double)experts)) + 0.99);
        if (with_rows < 1) with_rows = 1;
        load = 4 * ceil_div(rows, experts) + 12;
        if (load > rows) load = rows;
    }
    const int tmax = load <= 16 ? 16 : load <= 32 ? 32 : load <= 64 ? 64 : 128;
    // (a layer's tokens are dealt out evenly)
    const int tokens = (int)ceil_div(experts > 1 ? (load < 128 ? load : 128) : ceil_div(rows, ceil_div(rows, 128)), 16) * 16;
    auto token_tiles = [&](int per) -> int64_t {
        if (experts == 1) return ceil_div(rows, per);
        const int64_t n = rows / per + with_rows / 2;   // (half a tile of each expert is empty)
        return n > with_rows ? n : with_rows;
    };
    // (tiles of experts are not that many for certain: a last round that may be empty or full counts half)
    auto rounds_of = [&](int64_t tiles, int64_t places) -> double {
        return tiles <= places ? 1.0 : grouped ? (double)tiles / (double)places + 0.5 : (double)ceil_div(tiles, places);
    };

    BlocksPlan best = {};
    double least = 1e30;
    const int ctas = tmax <= 32 ? 2 : 1;
    const double floor = 0.55 + 0.0055 * tokens;   // a k-block's round of waits and additions
    auto consider = [&](int channels, int cut) {   // whether it fits
        BlocksPlan pl = {};
        pl.tmax = tmax;
        pl.tokens = tokens;
        pl.channels = channels;
        pl.cut = cut;
        pl.ctas = ctas;
        pl.tiles = ceil_div(N, channels) * token_tiles(tokens);
        const double rounds = rounds_of(pl.tiles, (int64_t)sms * ctas / cut);
        if (!blocks_fit(&pl, grouped ? 2 : (int64_t)rounds, grouped)) return false;
        double t;
        if (cut == 1) {
            const double kb = channels / 128.0 * (pl.tiles > sms ? ctas : 1);
            t = rounds * ((double)KB * (kb > floor ? kb : floor) + 2.0);
        } else {
            const double stream = (double)pl.tiles * (double)KB / sms, walk = (double)ceil_div(KB, cut) * floor;
            t = (stream > walk ? stream : walk) + 3.5;
        }
        if (t < least) {
            least = t;
            best = pl;
        }
        return true;
    };
    for (int channels = 128; channels >= 64; channels -= 8) consider(channels, 1);
    // K is cut where that fills the SMs in one round, as far as it does: a tenth of the places is left, since a cluster's lie in one
    // group of SMs, and the groups' sizes are no multiples of it.  Measured, us, not cut / cut: (1, 6144, 4096) 13.8 / 8.3, (16, 4096,
    // 14336) 39.5 / 14.7, (64, 4096, 4096) 15.4 / 9.4.
    int64_t cut = (int64_t)(0.9 * sms * ctas) / (ceil_div(N, 128) * token_tiles(tokens));
    if (cut > 8) cut = 8;
    if (cut > KB / 2) cut = KB / 2;
    while (cut >= 2 && !consider(128, (int)cut)) --cut;
    if (tmax >= 64 && rows > 64 && N > 128) {
        const int64_t of_tokens = token_tiles(128), tiles = ceil_div(N, 256) * of_tokens;
        // weights of a k-block: from HBM for one of an expert's (or the layer's) token tiles, from L2 for the others
        const double stream = 2.0 * (double)with_rows / (double)of_tokens * (tiles < sms ? (double)tiles / sms : 1.0);
        const double work = (double)KB * 1.25 + 4.3, wait = (double)KB * stream + 0.8;
        if (rounds_of(tiles, sms) * (work > wait ? work : wait) < least) {
            best = {};
            best.wide = true;
            best.tokens = 128;
            best.tiles = tiles;
        }
    }
    return best;
}

}  // namespace w4a8
