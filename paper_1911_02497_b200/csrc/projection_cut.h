// How a product with a projection in 8 bits is cut into tiles and parts. Host code that needs no GPU.
#pragma once
#include <algorithm>

namespace cs {

constexpr int PJ_GROUP = 128;           // of the depth: columns that share a scale
constexpr int PJ_WIDE = 128;            // output columns of a tile
constexpr int PJ_QUAD = 4;              // groups of the depth whose scales share a word
constexpr int PJ_A = PJ_GROUP * PJ_WIDE;        // bytes of a stage's weights
constexpr int PJ_MAX_TILE = 128;        // rows of a tile
constexpr int PP_TILE = 224;            // most rows of a pair's tile: two accumulators and the scales fill tensor memory
constexpr int PJ_MAX_PARTS = 8, PP_MAX_PARTS = 4;

struct ProjectionCut {
    bool pair;              // pairs of CTAs, or single ones
    int tile, parts;        // rows of a tile; CTAs (pairs) that share its depth
    long long clusters;     // CTAs (pairs) launched: one per tile and part, or as many as the device holds at once
};

// The cut that a simple account in microseconds makes cheapest; its figures are measured (the start and end of a launch are left out but for
// what differs). A group of the depth costs a CTA by itself 150 ns and 0.6 for each row of the tile, one of a pair 100 and 1.1, and all
// their codes pass L2 at 13 MB/us. Codes come from memory at 70 KB/us for an SM and at no more than 4.5 MB/us in so short a time.
// A row of sums takes a single CTA 26 ns to write, a pair 4 ns; sums over a cluster cost 0.7 us and its barriers, more for wider tiles.
// Examples (us; chosen first): 1 row 1500 -> 6000: (single, tile 16, 1 part) 5.3, 3 parts 5.8. 128 rows 4096^2: pairs (64, 1) 9.7, single (32, 1)
// 10.2, (64, 2) 10.6. 512 rows: pairs (128, 1) 11.5, (176, 1) 13.4, single (128, 1) 14.1. 2048 rows: pairs (160, 1) 27.9, (176, 1) 29.0. 64 rows
// 9216 -> 4096: single (32, 2) 13.6, (64, 3) 13.4. Over 16 shapes the choice took at most 4 % more than the best of all cuts.
//
// fit(cut, n, count): clusters of n CTAs of the cut's kernel that the device holds at once; what it returns other than 0 is returned.
template <class Fit>
int choose_cut(long long rows, long long width, int groups, int num_sms, Fit fit_of, ProjectionCut &best)
{
    const int quads = (groups + PJ_QUAD - 1) / PJ_QUAD;
    const double sms = num_sms, codes = (double)groups * PJ_GROUP * (double)(width + rows);
    double least = 0.0;
    auto offer = [&](const ProjectionCut &s, long long ctas, double rounds, double group, double bytes, double more) {
        const double depth = (double)((quads + s.parts - 1) / s.parts * PJ_QUAD), busy = std::min((double)ctas, sms);
        const double t = std::max(rounds * depth * std::max(group, bytes * busy / 13e6), codes / std::min(4.5e6, 70e3 * busy)) + more;
        if (least == 0.0 || t < 0.99 * least) {
            least = t;
            best = s;
        }
    };
    const auto cut = [&](int most, int step) {          // rows of equal tiles of at most so many
        const long long n = (rows + most - 1) / most;
        return (int)(((rows + n - 1) / n + step - 1) / step * step);
    };
    int before = 0;
    for (int most = PJ_MAX_TILE; most >= 16; most -= 16) {
        const int tile = cut(most, 16);
        if (tile == before) continue;
        before = tile;
        const long long tiles = (rows + tile - 1) / tile * ((width + PJ_WIDE - 1) / PJ_WIDE);
        for (int parts = 1; parts <= std::min(PJ_MAX_PARTS, quads); ++parts) {
            const ProjectionCut s = {false, tile, parts, tiles * parts};
            const long long ctas = tiles * parts;
            const double rounds = (double)((ctas + num_sms - 1) / num_sms);
            if (parts > 1) {
                int fit = 0;
                const int rc = fit_of(s, parts, fit);
                if (rc) return rc;
                if (tiles > fit) break;
            }
            offer(s, ctas, rounds, 0.15 + 0.0006 * tile, PJ_A + (double)PJ_GROUP * tile, 0.026 * tile * rounds + (parts > 1 ? 0.7 + 0.3 * parts + 0.006 * tile : 0.0));
        }
    }
    before = 0;
    for (int most = PP_TILE; rows > 64 && most >= 64; most -= 16) {
        const int tile = cut(most, 16);
        if (tile == before) continue;
        before = tile;
        const long long tiles = (rows + tile - 1) / tile * ((width + 2 * PJ_WIDE - 1) / (2 * PJ_WIDE));
        for (int parts = 1; parts <= std::min(PP_MAX_PARTS, quads); ++parts) {
            ProjectionCut s = {true, tile, parts, tiles * parts};
            int fit = 0;
            const int rc = fit_of(s, 2 * parts, fit);
            if (rc) return rc;
            if (fit < 1 || (parts > 1 && tiles > fit)) break;
            if (parts == 1) s.clusters = std::min(tiles, (long long)fit);
            const double rounds = (double)((tiles + fit - 1) / fit);
            offer(s, 2 * s.clusters, rounds, 0.1 + 0.0011 * tile, PJ_A + 0.5 * PJ_GROUP * tile, 0.5 + 0.004 * tile * rounds + (parts > 1 ? 2.0 + 0.01 * tile + 0.5 * parts : 0.0));
        }
    }
    return 0;
}

}  // namespace cs
