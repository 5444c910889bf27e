// Choice of a product's form from its sizes and the type of its result (q8t_fp8_gemm; the forms: fp8_gemm.h).  Plain C++.
#pragma once
#include <stdint.h>

#include "q8t.h"

// Form of a product: which kernel, and into how many slices the reduction is cut (partial sums in the workspace where there are several)
enum Fp8Form { FP8_DIRECT_16, FP8_DIRECT_32, FP8_DIRECT_64, FP8_TILE_64, FP8_TILE_64_128, FP8_TILE_128_DEEP, FP8_TILE_128, FP8_TILE_256 };
struct Fp8Plan {
    Fp8Form form;
    int slices;
};

namespace {

// Estimated microseconds of a form: what it measured at sizes where one thing bounds it.
//   direct   the operands cross the L2 once for every tile of 16 MT x 16 NT results (9 TB/s), or a wavefront's chain of loads:
//            1.3 (2.5, 5) us for every four blocks of its eighth of the reduction
//   tiles    a step of one block takes `alone` where a compute unit has one tile and `full` for each tile where all units hold as many
//            as fit (`fit`); a round of tiles `start` for the first copies and the last stores
// bf16 / fp32 at 4096 x 4096 weights, us, M = 16: direct 16 6.2 / 6.1, tile 64 9.9 / 20; 32: direct 32 8.4 / 8.2; 64: direct 64 10.6 / 10.5,
// tile 64 10.5 / 21; 128: tile 64 10.5 / 21, in four slices - / 15; 512: tile 64 x 128 14.3 / 26, 128 deep 17 / -; 1024: 128 deep 21 / -, 128 27 / 33; 2048: 128 35 / 58,
// 256 41 / 76; 4096: 256 53 / 99, 128 68 / 113.
struct TileCost {
    Fp8Form form;
    int bm, bn, fit;
    double alone, full, start;
};
const TileCost kBf16[] = {{FP8_TILE_64, 64, 64, 2, 0.20, 0.25, 1.2}, {FP8_TILE_64_128, 64, 128, 1, 0.29, 0.37, 1.4}, {FP8_TILE_128_DEEP, 128, 128, 1, 0.40, 0.58, 2.2},
                          {FP8_TILE_128, 128, 128, 2, 0.66, 0.54, 1.0}, {FP8_TILE_256, 256, 256, 1, 1.10, 1.72, 2.0}};
const TileCost kF32[] = {{FP8_TILE_64, 64, 64, 4, 0.53, 0.32, 1.0}, {FP8_TILE_64_128, 64, 128, 2, 0.64, 0.51, 1.8}, {FP8_TILE_128, 128, 128, 2, 0.73, 0.83, 3.0},
                         {FP8_TILE_256, 256, 256, 1, 2.10, 2.95, 4.0}};
constexpr int kUnits = 256;

double tile_us(const TileCost &c, int64_t tiles, int steps)
{
    const int64_t slots = (int64_t)kUnits * c.fit, rounds = tiles / slots, rest = tiles - rounds * slots;
    const double all = c.fit * c.full > c.alone ? c.fit * c.full : c.alone;
    double us = rounds * (steps * all + c.start);
    if (rest) {
        const int64_t one = c.fit > 1 ? kUnits : 0;   // up to one a unit nothing is shared but the L2
        us += steps * (rest <= one ? c.alone : c.alone + (all - c.alone) * (rest - one) / (slots - one)) + c.start;
    }
    return us;
}

Fp8Plan fp8_plan_of(int M, int N, int nk, int type)
{
    Fp8Plan best = {FP8_TILE_256, 1};
    double least = 1e30;
    auto consider = [&](Fp8Form f, int slices, double us) {
        if (us < least) {
            least = us;
            best = {f, slices};
        }
    };
    auto up = [](int64_t v, int m) { return (v + m - 1) / m; };
    if (M <= 64) {
        const struct {
            Fp8Form f;
            int m, n;
            double chain;
        } d[] = {{FP8_DIRECT_16, 16, 16, 1.3}, {FP8_DIRECT_32, 32, 16, 2.5}, {FP8_DIRECT_64, 32, 32, 5.0}};
        for (const auto &x : d) {
            const double rows = (M < x.m ? M : x.m) + (N < x.n ? N : x.n);
            const double bytes = (double)up(M, x.m) * up(N, x.n) * rows * nk * 128.0, chain = 1.0 + x.chain * up(nk, 32);
            consider(x.f, 1, bytes / 9e6 > chain ? bytes / 9e6 : chain);
        }
    }
    // Tiles sum a bf16 result less exactly than the direct forms; where those take all weights from memory once or run in one round, the
    // estimates differ by less than they are off (a call in a graph, us, direct and tile 64: 1 x 100 x 300 2.6 and 2.9, 2 x 6122 x 421 3.1 and 3.3,
    // 58 x 318 x 418 3.1 and 3.6, but 54 x 3217 x 1003 6.3 and 4.5).
    const double worth = type == Q8T_BF16 && (M <= 16 || (M <= 64 && up(M, 16) * up(N, 16) <= kUnits)) ? 1.0 : 0.0;
    const TileCost *cost = type == Q8T_F32 ? kF32 : kBf16;
    const int n = type == Q8T_F32 ? (int)(sizeof(kF32) / sizeof(kF32[0])) : (int)(sizeof(kBf16) / sizeof(kBf16[0]));
    for (int i = 0; i < n; ++i) {
        const int64_t tiles = up(M, cost[i].bm) * up(N, cost[i].bn);
        if (tiles > 1 << 22) continue;   // a launch holds fewer than 2^32 threads
        consider(cost[i].form, 1, tile_us(cost[i], tiles, nk) + worth);
        // Few small tiles under a long reduction: slices of it fill the chip; their sums cost a launch and cross memory twice (512 x 512
        // x 8192 to fp32 37 us in one slice, 17 in four).
        if (cost[i].form != FP8_TILE_64 || tiles > kUnits) continue;
        for (int z = 2; z <= 16 && z * 8 <= nk; z *= 2)
            consider(cost[i].form, z, worth + tile_us(cost[i], tiles * z, (int)up(up(nk, z), 4) * 4) + 2.5 + (double)M * N * 4.0 * (2 * z + 1) / 4e6);
    }
    return best;
}

}  // namespace
