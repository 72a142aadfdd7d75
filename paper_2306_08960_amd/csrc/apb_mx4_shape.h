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

// The same for both projections of a gated block (N columns of each).  Experts of fewer than 512 rows on average take no tiles of 256:
// 16 experts of 256 rows, 2 x 2048 x 2048, 37 us with 128 a side and 44 with 256; 64 of 64, 2 x 1024 x 2048, 32 and 47; 64 of 256, rows
// spread unevenly, 70 and 88; of 512 rows, 2 x 2048 x 2048 on 4 experts, 23 and 22, 2 x 4096 x 2048 on 16 unevenly, 128 and 120.
inline int mx4_gated_side(int M, int N, int E, bool grouped) {
    const int side = mx4_product_side(M, 2 * N);
    return grouped && M / E < 512 ? std::min(side, 128) : side;
}

// Both projections of a gated block by the kernel for few rows (apb_mx4_few.hip): twice the weights to the same rows, and one launch
// instead of two.  Few rows, measured as for the plain products, one kernel : two (us): 2 x 4096 x 4096, 1 row 5.9 : 12.9, 16 rows
// 11.3 : 12.8, 32 rows 13.6 : 13.0; 2 x 8192 x 8192, 16 rows 25.0 : 32.5; 64 experts of 2 x 1024 x 2048, a row each 26.7 : 27.4, 4 rows
// 29.2 : 28.0; 16 experts of 2 x 2048 x 4096, 4 rows each 36.4 : 27.0.  More rows of little work, tiles of 16 rows that read the weights
// again: 1024 x 512 x 512 6.1 : 6.6, 256 x 2048 x 512 6.1 : 6.5, 128 x 2048 x 2048 10.9 : 8.5, 16384 x 64 x 64 10.6 : 8.8; 256 rows on 16
// experts of 2 x 512 x 512 6.1 : 6.9, 1024 rows 8.5 : 7.1, 64 rows on 8 of 2 x 1024 x 4096 18.4 : 12.5.  Called from Python, a launch less
// is 4 us less, and two are 12.9 whatever they do.  Below a K of 256 the work no longer falls with K (rows are padded to segments), so the
// outputs are bounded: 512 x 4096 x 32 11.2 : 7.2, 512 x 8192 x 32 20 : 9.4, 4096 x 2048 x 32 26 : 15; on 16 experts 512 x 2048 x 32
// 9.5 : 8.1, 16384 x 32 x 32 10.3 : 8.6, 4096 x 1024 x 32 23 : 11, 131072 x 4 x 32 63 : 41.  One segment, many outputs and tiles that are
// mostly empty: 32 x 262144 x 32 34 : 229, 64 x 8192 x 256 4.8 : 7.4, 64 x 524288 x 256 93 : 457, 256 x 24576 x 256 (tiles of 256 a side)
// 22 : 28, 256 x 24000 (of 128) 22 : 17; on 16 experts 512 x 8192 x 32 22 : 24, on 64 2048 x 16384 x 256 98 : 166, 4096 x 2048 31 : 27.
// (Of the two kernels' times 2.5 us are the quantization, which a call with 4-bit rows does not have.)
inline bool mx4_gated_is_little(int M, int N, int K, int E, bool grouped) {
    const int mean = grouped ? (M + E - 1) / E : M;              // rows of an expert, were they all alike
    const long long outputs = (long long)M * N;
    if (mean <= 16 && (!grouped || (long long)mean * K <= 8192)) return true;
    if (K <= kMxSeg && (grouped ? mean <= 32 && outputs >= 1 << 22 : M <= 64 || (M <= 256 && mx4_product_side(M, 2 * N) == 256))) return true;
    return K <= 2048 && M <= (grouped ? 16384 : 4096) &&
           outputs <= std::min<long long>((1LL << (grouped ? 27 : 28)) / K, 1 << (grouped ? 20 : 21));
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
