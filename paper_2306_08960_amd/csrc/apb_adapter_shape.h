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
constexpr int kCols = 128;                    // of a wave of up: eight to a lane
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

// Columns of X that the gradients of `adapters` make, in groups of 64, times the groups of ranks: workgroups, were the rows not shared.
inline long long gradient_groups(int adapters, int K, int r) {
    const int ranks = 16 * rank_groups(r);
    return (long long)((K + 63) / 64) * adapters * ((r + ranks - 1) / ranks);
}
// No more adapters than these have rows.
inline int active_adapters(int S, int L) { return std::min(S, L); }
// The gradient's workgroups go by adapter, or, where many adapters cannot have rows, by segment (the first of its adapter), and some that
// only clear.  us by adapter and by segment (clearing alone): 4100 rows of 4096 in four segments, 64 adapters of rank 16 24 and 19 (5), of
// rank 64 60 and 34 (11), 1024 of rank 16 255 and 53 (34); 64 segments of a row, 512 adapters 31 and 25 (19).
inline bool gradient_by_segment(int S, int L, int K, int r) { return L > S && gradient_groups(L - S, K, r) >= 1024; }
// Rows of an adapter to a workgroup of its gradient.  Where one workgroup for each of those fills the compute units, more than 8192 and
// four times the average are shared out, and otherwise so many that there is a workgroup to each unit, but at least 256 (sharing costs a
// launch and 4 us).  bfloat16, us: 4100 rows of 4096, rank 16, four adapters (256 groups) not shared 11.7, in pieces of 2048 rows 14.2, of
// 1024 17.7; one adapter (64 groups) 27.0, 18.4, 16.5; 2000 rows of 1024, rank 64, one adapter (16 groups) not shared 39, in pieces of 1024
// 25, of 512 16.5, of 256 13.1.
inline int gradient_rows(int S, int L, int M, int K, int r) {
    const int active = active_adapters(S, L);
    const long long mean = (M + active - 1) / active, slices = 256 / gradient_groups(active, K, r);
    return (int)(slices <= 1 ? std::max(8192LL, 4 * mean) : std::max(256LL, (mean / slices + 31) / 32 * 32));
}
// Groups of 16 ranks, columns to a lane and waves of such a workgroup.  A wave takes 32 rows at a time: as many waves as an adapter has
// rows for on average, and one for each 256 rows in case one adapter has most of them.  128 columns instead of 64, which halves how often T
// is read and split, where that leaves a workgroup to each compute unit.  bfloat16, us, with 64 and with 128: 16384 rows of 8192, rank 32
// 91 and 62, 4100 rows of 8192, rank 16 21 and 18, 2000 rows of 4096, rank 32, eight adapters 16 and 11; with half the workgroups
// 4100 rows of 4096, rank 32, four adapters 14 and 17.
struct GradientForm {
    int jt, nc, waves;
};
inline GradientForm gradient_form_of(int x_type, int S, int L, int M, int K, int r) {
    const int active = active_adapters(S, L), jt = rank_groups(r), chunks = std::max((M / active + 31) / 32, (M + 255) / 256);
    const bool wide = x_type == APB_F32;                         // (its operands take twice the registers)
    const int waves = chunks > 4 && !(wide && jt == 4) ? 8 : chunks > 1 ? 4 : 1;
    return GradientForm{jt, waves == 8 && !wide && jt <= 2 && K >= 128 && gradient_groups(active, K, r) >= 512 ? 8 : 4, waves};
}

// Groups of rows, rows, and groups of ranks to a workgroup of down, and parts of K: what takes least by a count of the bytes that the busiest
// compute unit brings (40 GB/s each; two a value, whatever the type, so that the parts depend on the sizes alone), a quarter of a
// microsecond for each part that the readers of T will add up, and parts only where T stays small.  Rows may be fewer than their groups
// hold, where more workgroups then share the work with still one to a compute unit.
// Measured (us; rows, groups of ranks, parts; X from memory where there is more than one row): one row of 4096, rank 16: 16 1 1 5.8, 16 1 4
// 4.3, 16 1 8 4.1; 512 rows, rank 16: 16 1 1 10.0, 16 1 4 4.7; 4100 rows, rank 16: 16 1 1 14.8, 17 1 1 11.0, 24 1 1 12.0, 32 1 1 12.9;
// 8196 rows, rank 64: 16 4 1 36, 32 4 1 33, 33 4 1 24, 48 4 1 27, 64 4 1 29.
struct DownPlan {
    int rt, tile, jt, parts;
};
inline DownPlan down_plan(int S, int M, int K, int r) {
    DownPlan best{1, 16, 1, 1};
    double least = 1e30;
    for (int rt = 1; rt <= 4; rt *= 2)
        for (int jt = 1; jt <= rank_groups(r); jt *= 2)
            for (int parts = 1; parts <= kMaxParts; parts *= 2) {
                if (parts > 1 && ((long long)parts * M > 8192 || K < 512 * parts)) continue;
                const long long segments = std::min(S, M), each = (long long)((r + 16 * jt - 1) / (16 * jt)) * parts;
                const long long tiles = std::max<long long>((M + 16 * rt - 1) / (16 * rt), segments), rounds = (tiles * each + 255) / 256;
                // as few rows as still leave one workgroup to a compute unit, with a last tile in each segment
                int tile = 16 * rt;
                while (tile > 8 * rt + 1 && ((M + tile - 2) / (tile - 1) + segments - 1) * each <= 256) --tile;
                if (rt == 1) tile = 16;
                const double cost = (double)rounds * (tile + 16 * jt) / parts * K * 2 / 40e3 + 0.25 * parts;
                if (cost < least) {
                    least = cost;
                    best = DownPlan{rt, tile, jt, parts};
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

// The slices of adapters behind their first ones: at most M / each of them, which have a workgroup each beside one for each adapter
// (bfloat16: 65536 rows of 4096 on 64 adapters of rank 16 131 us, with M / each workgroups for each adapter 181; on 256 adapters 247 and
// 622; 262144 rows of 1024 on 4096 adapters of rank 8 4.5 ms and 80).  Were all rows ordered by their adapter, the place k * each, k = 1 ..
// more_slices(M, each), lies among the rows of one adapter, with `before` rows of others before it, and stands for that adapter's slice
// number slice_at_place(k, before, each): 0, or more than it has, where there is none to stand for.  Every slice but the first ones has
// one place.
inline int more_slices(int M, int each) { return (M - 1) / each; }
APB_BOTH inline int slice_at_place(int k, int before, int each) { return k - before / each; }
// To find out which adapter's a slice is takes a few microseconds.  So there are workgroups for each of `firsts` adapters or segments and each
// of M / each slices, `groups` of them, as long as those that only exit are few.  us, so and by slice: 2506 of them (17979 rows of 435, 179
// adapters of rank 5) 28 and 31; 3710 (27505 of 28, 35 of rank 24) 22 and 12; 6963 (8469 of 12, 211 of rank 2) 30 and 11.
inline bool gradient_by_slice(int firsts, int M, int each, long long groups) { return firsts * groups * ((M - 1) / each) > 3072; }
// The same for the workgroups that join them, `columns` for each adapter, which exit sooner.
inline bool join_by_slice(int L, int M, int each, long long columns) { return L > more_slices(M, each) && L * columns > 8192; }

}  // namespace apb
