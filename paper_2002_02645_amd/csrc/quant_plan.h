// How the dense layer on 8-bit rows cuts a product, and the memory that takes.  Host code alone: nothing of HIP in it.
#pragma once
#include <algorithm>
#include <cstddef>
#include <cstdint>

namespace fz {

constexpr int kQuantBlock = 128;             // values that share an exponent: one k-step of the product
constexpr int kQuantTile = 256;              // rows of a tile of the weights
constexpr int kQuantMostCuts = 64;           // of a tile along the depth
constexpr int kQuantMostRounds = 4;          // of workgroups, of cut tiles
constexpr int kQuantThreads = 512;           // of a workgroup of the product
constexpr int64_t kQuantMostWorkgroups = 0xffffffffll / kQuantThreads;   // a grid has less than 2^32 threads

// Tiles of the product's kernels.
struct QuantVariant {
    int bm, bn;         // rows of x, rows of w of a tile
    int per_cu;         // workgroups
    float step_us;      // of a k-step of a workgroup where neither memory nor L2 bounds it
};
constexpr QuantVariant kQuantVariants[] = {
    {16, 128, 2, 0.60f}, {32, 128, 2, 0.75f}, {64, 128, 2, 1.00f}, {16, 256, 1, 0.75f}, {32, 256, 1, 0.90f},
    {64, 256, 1, 1.10f}, {128, 256, 1, 1.55f}, {160, 256, 1, 1.80f}, {192, 256, 1, 2.20f}, {256, 256, 1, 2.95f},
};
constexpr int kQuantNumVariants = (int)(sizeof kQuantVariants / sizeof kQuantVariants[0]);

struct QuantPlan {
    int variant;
    int bm, bn;
    int x_tiles, w_tiles, nk;
    int splits;         // cuts of a tile along the depth
    int64_t wgs;
    size_t part;        // floats of the sums of cut tiles
};

inline int64_t quant_tiled_rows(int64_t rows, int64_t tile) { return (rows + tile - 1) / tile * tile; }

// Rows of x that a workspace holds: no tile is higher than 256, and a larger batch never needs fewer.
inline int64_t quant_workspace_rows(int64_t b) { return b + 255; }

// Bytes for the sums of cut tiles: what a plan may use at most.  It never falls as the batch grows, so that a workspace for a batch serves all
// smaller ones too (the plans' own needs go up and down: 33 rows of 4,096 -> 32,768 are cut and want 17 MB, 39 are not).  No plan needs more
// than four rounds of tiles as high as the batch (256 rows at most), or all cuts of the whole output; beyond 64 MiB, what the weights
// or the rows hold is enough: of 100,000 random sizes whose plans cut, 3 take another plan for it, 4 % slower at most by the cost below.
inline size_t quant_room(int64_t b, int64_t m, int64_t d_pad, int num_cus)
{
    int64_t high = 16;
    while (high < b && high < 256) high *= 2;
    const double rounds = 4.0 * kQuantMostRounds * 256.0 * (double)num_cus * (double)high;   // (per_cu * bn is 256 for every tile)
    const int64_t nk = d_pad / kQuantBlock;
    const double cuts = 4.0 * (double)(nk < kQuantMostCuts ? nk : kQuantMostCuts) * (double)quant_workspace_rows(b) * (double)quant_tiled_rows(m, kQuantTile);
    const double held = std::max(67108864.0, (double)std::max(quant_tiled_rows(m, kQuantTile), quant_workspace_rows(b)) * (double)d_pad);
    return (size_t)std::min(std::min(rounds, cuts), held);
}

// wgs 0: more tiles than a launch has workgroups (outputs that no memory holds).
inline QuantPlan plan_quant_product(int64_t b, int64_t m, int64_t d_pad, int num_cus)
{
    QuantPlan pl{};
    pl.nk = (int)(d_pad / kQuantBlock);
    const int64_t room = (int64_t)(quant_room(b, m, d_pad, num_cus) / 4);
    double best = 0;
    for (int i = 0; i < kQuantNumVariants; ++i) {
        const QuantVariant &v = kQuantVariants[i];
        const int64_t xt = (b + v.bm - 1) / v.bm, wt = (m + v.bn - 1) / v.bn, tiles = xt * wt, places = (int64_t)num_cus * v.per_cu;
        // whole tiles, or each cut along the depth so that a quarter or half a round of workgroups, or one to four rounds are full, with the
        // sums through memory (written and read at 2.5 TB/s, and a launch)
        constexpr int kQuarters[] = {0, 1, 2, 4, 8, 12, 4 * kQuantMostRounds};
        for (int r : kQuarters) {
            const int64_t fit = r == 0 ? 1 : std::min<int64_t>(places * r / 4 / tiles, std::min(pl.nk, kQuantMostCuts));
            if (r > 0 && fit < 2) continue;
            const int splits = (int)fit;
            if (tiles * splits > kQuantMostWorkgroups || (splits > 1 && tiles * splits * v.bm * v.bn > room)) continue;
            const double rounds = (double)((tiles * splits + places - 1) / places);
            // Workgroups in rounds; the weights out of memory (6.5 TB/s where one workgroup reads them, else 5.3); what a CU takes in (40 GB/s; all of them 10 TB/s), of which a part shows
            // beside either.
            const double steps = (double)((pl.nk + splits - 1) / splits);
            const double fed = (double)((tiles * splits + num_cus - 1) / num_cus) * steps * (double)(v.bm + v.bn) * 132.0 / 40e3;
            double us = rounds * (steps * v.step_us + 3.0);
            us = std::max(us, (double)wt * v.bn * (double)d_pad / (xt == 1 ? 6.5e6 : 5.3e6));
            us = std::max(us, fed) + 0.15 * fed;
            if (splits > 1) us += 5.0 + 2.0 * 4.0 * (double)wt * v.bn * (double)b * splits / 2.5e6 + 0.1 * splits;
            if (pl.wgs == 0 || us < best) {
                best = us;
                pl.variant = i;
                pl.bm = v.bm;
                pl.bn = v.bn;
                pl.x_tiles = (int)xt;
                pl.w_tiles = (int)wt;
                pl.splits = splits;
                pl.wgs = tiles * splits;
            }
        }
    }
    pl.part = pl.splits > 1 ? (size_t)pl.wgs * pl.bm * pl.bn : 0;
    return pl;
}

}  // namespace fz
