// Sizes and launch shapes of the microscaled 4-bit matrices' products and gradients: arithmetic on sizes only, kept apart from the
// device code so that a host compiler can walk it.
#pragma once

#include <algorithm>

#include "apb.h"

namespace apb {

constexpr int kMxBlock = 32;                  // values that share a scale
constexpr int kMxSeg = 256;                   // a row is padded to whole segments of 256 values: one 128-byte line of
                                              // codes, 8 scale bytes
constexpr int kMxSegBytes = kMxSeg / 2;

inline int mx_segs(int K) { return (int)(((long long)K + kMxSeg - 1) / kMxSeg); }
constexpr int kMxMaxK = 1 << 22;
constexpr long long kMxMaxSegs = (1LL << 27) - 8;   // of a matrix (34 G values): eight go to a workgroup of 256 lanes, and a launch has
                                                    // fewer than 2^32 lanes
inline bool bad_shape_mx(long long rows, int K) {
    return rows <= 0 || K <= 0 || K > kMxMaxK || rows * mx_segs(K) > kMxMaxSegs;
}

// Tiles of `tile` rows that R rows in E groups (and the rows behind them) take at most.
inline long long max_row_tiles(int R, int E, bool grouped, int tile) {
    const long long whole = ((long long)R + tile - 1) / tile;
    return grouped ? whole + std::min<long long>((long long)E + 1, R) : whole;
}

// The side of the product's tiles.  256 a side load least per product, and there is one to a compute unit; smaller ones fill the chip
// sooner.  Measured on plain products, with 256, 128 and 64 a side (us): 4096^3 42, 52, 84; 1500 x 8192 x 4096 (192 tiles of 256) 36,
// 41, 66; 2560 x 2560 x 4096 (100) 31, 27, 39; 1024 x 4096 x 4096 (64) 31, 15, 23; 512 x 4096 x 4096 (32) 27, 12, 12; 1024 x 1024 x
// 4096 (16) 28, 12, 9.  Rows in groups are counted as if they were one matrix: an expert of fewer rows than a tile has leaves the
// rest of it empty.
inline int mx4_product_side(int M, int N) {
    const long long big = ((long long)M + 255) / 256 * ((N + 255) / 256);
    return big >= 192 ? 256 : big * 4 >= 192 ? 128 : 64;
}

constexpr int kMx4Pass = 64;                  // rows of the 4-bit matrix that a pass of the gradients sums over
constexpr int kMx4MaxSlices = 32;

// How the work of a gradient is laid out: tiles of 64 * f a side, by how many groups of waves each, in how many slices.
struct Mx4Plan {
    int f, groups, slices;
};

template <bool WEIGHT>
inline Mx4Plan mx4_gradient_plan(int g_type, bool grouped, int E, int M, int N, int K, bool workspace = true) {
    auto tiles = [&](int side) { return ((long long)(WEIGHT ? N : M) + side - 1) / side * ((K + side - 1) / side) * (WEIGHT ? E : 1); };
    // passes of a tile, were the experts all alike
    const long long passes = ((WEIGHT ? (grouped ? M / E : M) : N) + kMx4Pass - 1) / kMx4Pass;
    // slices that make a workgroup for each compute unit, of at least `least` passes
    auto slices = [&](long long n, long long least) {
        return (int)std::max<long long>(1, std::min<long long>(std::min<long long>(256 / n, passes / least), workspace ? kMx4MaxSlices : 1));
    };
    // Measured in bfloat16 on plain products (us).  256 a side wherever they fill more than half of the chip: 4096^3 121, 128 a side 183;
    // dX of 2560 x 4096 x 4096 100 and 127; in two slices where they fill half of it and the sums are long: 4096 x 8192 x 2048 131, 128
    // a side 174.  128 a side likewise, with a second group up to one tile per compute unit: 2048^3 28, with one group 35, 64 a side 54.
    // 64 a side if those fill the chip and the sums are short: 1024^3 11, 128 a side in slices 21.  Then slices: 512 x 4096 x 4096 37,
    // without 45; dW of 8192 x 1024 x 1024 39, without 50; of 16384 x 256 x 256 15, without 91; dX of 64 x 1000 x 64 in slices of 4 passes
    // 7.8, of 8 9.1.  dX counts the rows of all experts as one matrix: a tile may be taller than what an expert has.
    const bool two_groups = g_type == APB_BF16 && tiles(128) <= 256;
    if (g_type == APB_BF16 && tiles(256) >= 144) return Mx4Plan{4, 1, 1};
    if (g_type == APB_BF16 && tiles(256) >= 96 && tiles(256) <= 128 && passes >= 64 && workspace) return Mx4Plan{4, 1, 2};
    if (tiles(128) >= 192) return Mx4Plan{2, two_groups ? 2 : 1, 1};
    if (tiles(64) >= 192 && passes <= 24) return Mx4Plan{1, 2, 1};
    const int shared = slices(tiles(128), g_type == APB_BF16 ? 20 : 12);      // (more parts of G: passes take longer, joining does not)
    if (tiles(128) * shared >= 128) return Mx4Plan{2, two_groups && shared == 1 ? 2 : 1, shared};
    // (sharing costs 3 us, a pass 0.35: two that share 8 passes lose 3 us against one, four that share 16 gain 1)
    const int quarters = slices(tiles(64), 4);
    return Mx4Plan{1, 2, quarters > 2 ? quarters : slices(tiles(64), 8)};
}

}  // namespace apb
