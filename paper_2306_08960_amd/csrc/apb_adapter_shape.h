// Launch shapes of the adapters' kernels: arithmetic on sizes only, kept apart from the device code so that a host compiler can
// walk it.
#pragma once

#include <algorithm>

#include "apb.h"

#ifdef __HIPCC__
#define APB_BOTH __host__ __device__
#else
#define APB_BOTH
#endif

namespace apb {

constexpr int kMaxParts = APB_ADAPTER_MAX_PARTS;
constexpr int kCols = 128;                    // of a wave, in up and gradient: eight to a lane
constexpr int kAdapterWaves = 4;              // of a workgroup there
constexpr int kUpRows = 64;                   // of a workgroup that streams them past B, at most

inline int rank_groups(int r) { return r <= 16 ? 1 : r <= 32 ? 2 : 4; }

// Rows to a workgroup that streams them past its share of B.
inline int up_rows(int S, int M, int N) {
    const long long columns = (N + kCols * kAdapterWaves - 1) / (kCols * kAdapterWaves);
    int rows = 16;
    while (rows < kUpRows && rows < (M + S - 1) / S && M / (2 * rows) * columns >= 1024) rows *= 2;
    return rows;
}

// Rows of an adapter to a workgroup of its gradient: so many that a workgroup comes to each compute unit, were they spread evenly, but at
// least 128, and no more than 16384 workgroups that may find none.  4100 rows of 4096, rank 16, four adapters (us): 512 workgroups 21.5,
// 256 16.0, 128 18.9; 8196 rows, rank 64: 55, 43, 48.  Up to 256 rows are never shared: joining takes 4 us and another launch.
inline int gradient_rows(int L, int M, int K, int r) {
    const int ranks = 16 * rank_groups(r);
    const long long columns = (long long)((K + kCols * kAdapterWaves - 1) / (kCols * kAdapterWaves)) * ((r + ranks - 1) / ranks);
    const long long rows = std::max<long long>(M * columns / 256, M * columns * L / 16384);
    return M <= 256 ? 256 : (int)std::min<long long>(1 << 24, std::max<long long>(128, (rows + 63) / 64 * 64));
}

// Groups of rows and of ranks to a workgroup of down, and parts of K: what takes least by a count of the bytes that the busiest compute
// unit brings (40 GB/s each), a quarter of a microsecond for each part that the readers of T will add up, and parts only where T stays
// small.  Measured (us; groups of rows, of ranks, parts): one row of 4096, rank 16: 1 1 1 5.8, 1 1 4 4.3, 1 1 8 4.1; 512 rows, rank 16:
// 1 1 1 10.0, 1 1 4 4.7; 4100 rows, rank 16: 1 1 1 12.2, 2 1 1 11.6; 8196 rows, rank 64: 1 1 1 68, 2 2 1 34, 4 4 1 25.
struct DownPlan {
    int rt, jt, parts;
};
inline DownPlan down_plan(int S, int M, int K, int r) {
    DownPlan best{1, 1, 1};
    double least = 1e30;
    for (int rt = 1; rt <= 4; rt *= 2)
        for (int jt = 1; jt <= rank_groups(r); jt *= 2)
            for (int parts = 1; parts <= kMaxParts; parts *= 2) {
                if (parts > 1 && ((long long)parts * M > 8192 || K < 512 * parts)) continue;
                const long long tiles = std::max<long long>((M + 16 * rt - 1) / (16 * rt), std::min(S, M)) * ((r + 16 * jt - 1) / (16 * jt));
                const long long rounds = (tiles * parts + 255) / 256;
                const double cost = (double)rounds * (rt + jt) / parts * K * 32 / 40e3 + 0.25 * parts;
                if (cost < least) {
                    least = cost;
                    best = DownPlan{rt, jt, parts};
                }
            }
    return best;
}

// Waves of a workgroup of down.
constexpr int down_waves(int rt, int jt) { return rt + jt <= 4 ? 16 : 8; }

// Where the slices of an adapter of more than `each` rows leave their sums, with `before` rows of other adapters before it: n rows have
// ceil(n / each) <= floor(2 n / each) slices, so those of different adapters never meet, whatever their rows.
APB_BOTH inline int place_of_slices(int before, int each) { return (int)(2LL * before / each); }
// ... and how many places M rows take at most.
inline long long places_of_slices(int M, int each) { return 2LL * M / each + 1; }

}  // namespace apb
