// How the encoder of rows is cut: runs of neighbouring groups of a row, some of them a half-warp's. Host code that needs no GPU.
#pragma once
#include <cstdint>

#include "pieces.h"

namespace cs {

constexpr int ENC_UNITS = 4;            // groups of a half-warp, all of whose loads leave together

struct RowRuns {
    int groups_of_run;                  // 4, 2 or 1
    uint32_t runs, reciprocal;          // of a row; floor(2^32 / runs), at most 2^32 - 1
    long long grid;                     // CTAs
};

// For rows of `groups` groups, by CTAs of `halves` half-warps. False where the runs are so many that their numbers leave 32 bits.
inline bool plan_row_runs(long long rows, uint32_t groups, int halves, RowRuns &p)
{
    // the longest runs that leave no more than a quarter of their places empty
    const auto empty = [&](uint32_t n) { return (groups + n - 1) / n * n - groups; };
    p.groups_of_run = 4 * empty(4) <= groups ? 4 : 4 * empty(2) <= groups ? 2 : 1;
    p.runs = (groups + (uint32_t)p.groups_of_run - 1) / (uint32_t)p.groups_of_run;
    p.reciprocal = p.runs == 1 ? 0xFFFFFFFFu : (uint32_t)((1ull << 32) / p.runs);
    const long long per = (long long)halves * (ENC_UNITS / p.groups_of_run);
    p.grid = (rows * p.runs + per - 1) / per;
    return p.grid * per <= 0xFFFFFFFFll;
}

// The run `u` of all: its row, and its number in the row. (The estimate by the reciprocal is the quotient or one less.)
template <class High>
CS_BOTH void place_of_run(uint32_t u, uint32_t runs, uint32_t reciprocal, High high_product, uint32_t &row, uint32_t &run)
{
    row = high_product(u, reciprocal);
    run = u - row * runs;
    if (run >= runs) {
        run -= runs;
        row += 1;
    }
}

}  // namespace cs
