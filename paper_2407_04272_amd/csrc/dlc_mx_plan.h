// Which kernel a product of microscaled operands takes, and how its k is cut.  Host code without any library.
#pragma once
#include <cstddef>
#include <cstdint>

namespace dlc {

constexpr int kMxGroup = 512;  // columns of a group of scales
constexpr int kMxTileM[] = {256, 128, 64}, kMxTileN[] = {256, 128, 128}, kMxSkinny = 3, kMxSkinnyRows = 32;
constexpr int64_t kMxMaxTiles = int64_t(1) << 24;  // a launch's threads, work-groups of 256, are counted in 32 bits

struct MxPlan {
    int tile;               // of kMxTileM and kMxTileN, or kMxSkinny
    int split, kper;        // work-groups along k, k values of each
    int tiles_m, tiles_n;
    int64_t part_ld;
    size_t bytes;           // of the partial sums
};

// What 256 k values cost with 1 and 2 work-groups on a compute unit, in us, what a work-group costs besides, and every
// further one, measured on full cards (0: no second work-group fits; up to half of a card, whose work-groups have more of the
// caches and the power, kMxHalf of it): E2M1, E4M3, E4M3 with results in fp32.  64 x 128 is the best of the tiles until its
// tiles no longer fit the card at once (1024 x 2048 x 2048 of 4 bits 8.1 us for 10.3 and 22; 2048 x 2048 x 2048 12.3, 11.1 and 22.7, of 8 bits 17.3,
// 13.9 and 29.4), 256 x 256 where there are many (2048 x 8192 x 8192 of 4 bits 120, 98 and 66 us).
struct MxTileCost { double tile[2], first, further; };
constexpr MxTileCost kMxCost[3][3] = {{{{1.66, 0}, 12.8, 11.0}, {{0.64, 0}, 5.8, 3.7}, {{0.46, 0.86}, 4.4, 2.0}},
                                  {{{2.42, 0}, 13.6, 8.3}, {{0.89, 0}, 6.6, 4.2}, {{0.6, 0}, 4.6, 2.6}},
                                  {{}, {{2.2, 0}, 5.5, 3.5}, {{1.45, 0}, 4.2, 2.4}}};
constexpr double kMxHalf = 0.85;

// Few rows: a round of work-groups (a band of 32 rows and 16 columns each, one on a compute unit) with 1024 k values, what the
// first round costs besides and every further one; the kinds as above.  64 x 2048 -> 2048 of 4 bits 4.0 us, 7.4 the best of the
// tiles; 64 x 8192 -> 2048 5.8 and 10.4; 128 x 8192 -> 2048 in two rounds 9.7 and 12.0; 64 x 65536 -> 2048 22.9 and 19.8.
struct MxSkinnyCost { double k, first, further; };
constexpr MxSkinnyCost kMxSkinnyCost[3] = {{0.30, 3.4, 1.5}, {0.44, 4.1, 1.9}, {0.50, 4.2, 2.2}};
constexpr int kMxSkinnyRounds = 4;
constexpr int kMxUnits = 256;  // compute units
constexpr int kMxCuts[] = {1, 2, 3, 4, 6, 8, 12, 16};

// The tile and the cut of k with the smallest estimate
inline MxPlan mx_plan(int64_t M, int64_t K, int64_t N, bool e4m3, bool fp32) {
    const auto div_up = [](int64_t a, int64_t b) { return (a + b - 1) / b; };
    MxPlan best{};
    best.split = 1;
    best.tile = kMxSkinny;
    if (M <= kMxSkinnyRows / 2) return best;
    const int64_t groups = div_up(K, kMxGroup);
    const bool exact = e4m3 && fp32;
    const int kind = exact ? 2 : e4m3 ? 1 : 0;
    const MxTileCost* const cost = kMxCost[kind];
    double least = 1e300;
    const int64_t rounds = div_up(div_up(M, kMxSkinnyRows) * div_up(N, 16), kMxUnits);
    if (rounds <= kMxSkinnyRounds) {
        const MxSkinnyCost& c = kMxSkinnyCost[kind];
        least = c.first + (double)rounds * (double)K / 1024.0 * c.k + (double)(rounds - 1) * c.further;
    }
    for (int tile = exact ? 1 : 0; tile < 3; ++tile) {
        const MxTileCost& c = cost[tile];
        const int64_t tm = div_up(M, kMxTileM[tile]), tn = div_up(N, kMxTileN[tile]), tiles = tm * tn;
        if (tiles >= kMxMaxTiles) continue;
        const int fit = c.tile[1] > 0 ? 2 : 1;
        for (const int cut : kMxCuts) {
            if (cut > 1 && (cut > groups || tiles * cut > 2 * kMxUnits)) break;
            const int64_t per = div_up(groups, cut), split = div_up(groups, per), wgs = tiles * split;
            const int64_t full = wgs / (kMxUnits * fit), rest = wgs % (kMxUnits * fit);
            double t = (double)full * (2.0 * (double)per * c.tile[fit - 1] + c.further) + c.first - c.further;
            if (rest) t += 2.0 * (double)per * c.tile[(rest - 1) / kMxUnits] * (wgs <= kMxUnits / 2 ? kMxHalf : 1.0) + c.further;
            if (split > 1) t += 3.8 + (double)split * (double)M * (double)N * 8.0 / 6.2e6;  // (the second launch, the sums out and in)
            if (t < least) {
                least = t;
                best.tile = tile;
                best.split = (int)split;
                best.kper = (int)(per * kMxGroup);
                best.tiles_m = (int)tm;
                best.tiles_n = (int)tn;
            }
        }
    }
    best.part_ld = (N + 7) / 8 * 8;
    best.bytes = best.split > 1 ? (size_t)best.split * (size_t)M * (size_t)best.part_ld * 4 : 0;
    return best;
}

}  // namespace dlc
