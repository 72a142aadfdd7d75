// Products of two 4-bit matrices, Y = A^ B^T, plain or grouped by expert.  The matrix instruction takes the blocks' scales beside the
// 4-bit values: a block's 32 products are summed exactly, and rounded once to float32 with the sum so far.
// Bound by the matrix cores, and for long products by the power they may draw: 8192^3 with a bfloat16 result, one call behind another,
// takes 262 us (4200 TFLOP/s) on random values and 191 on zeros, with the same instructions.  4096^3: 42 us (3260), 1024 x 4096 x
// 4096: 15 us.
#include <type_traits>

#include "apb_mx8.h"

namespace apb {
namespace {

constexpr int kThreads = 256;                 // four waves, two by two

// All of this wave's loads but the last `Behind` are in LDS and its reads of LDS have been answered; then so are everybody's.
template <int Behind>
__device__ __forceinline__ void arrived() {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(Behind) : "memory");
}

// Which tile a workgroup takes: workgroups go to the eight XCDs in turn, and sixteen in a row on one XCD take a block of 4 x 4
// tiles, which shares its operands in that XCD's cache.
__device__ __forceinline__ void tile_of(int id, int tiles_n, int& t, int& n) {
    const int xcd = id & 7, j = id >> 3;
    const int linear = (j >> 4) * 128 + xcd * 16 + (j & 15);
    const int super = linear / (4 * tiles_n), rest = linear - super * 4 * tiles_n;
    t = super * 4 + (rest & 3);
    n = rest >> 2;
}

constexpr int kHalf = kMxSeg / 2;             // values that a pass sums over
constexpr int kHalfBytes = kHalf / 2;
constexpr int kRing = 4;                      // passes of operands in LDS

// The two halves of a gated wave's sums: four of G and the four of U beside them.
template <int F>
__device__ __forceinline__ f32x4 four_gate(const f32x16 (&acc)[F][F], int x, int y, int q) { return four_sums<F>(acc[x][y], 4 * q); }
template <int F>
__device__ __forceinline__ f32x4 four_up(const f32x16 (&acc)[F][F], int x, int y, int q) {
    if constexpr (F == 1) return four_sums<F>(acc[x][y], 8 + 4 * q);
    else return four_sums<F>(acc[x][y + F / 2], 4 * q);
}

// What two lanes, 32 apart, have of two words: the lower lane's a and the upper one's a, or their b's.
__device__ __forceinline__ u32x2 exchange(uint32_t a, uint32_t b) {
    const auto v = __builtin_amdgcn_permlane32_swap(a, b, false, false);
    return u32x2{v[0], v[1]};
}

// G or U of a wave's tile in 8 bits.  A block of 32 columns of a row lies in the lanes (r, 0) and (r, 1), which exchange fours until
// each has 16 neighbours; with F == 1 it lies in two waves, which exchange their maxima through LDS (`tops`, 64 rows x 2).  WHOLE:
// every column of the tile is there.
template <int F, bool WHOLE, class SUMS>
__device__ __forceinline__ void save_tile(const SUMS& sums, uint32_t* tops, const Mx8& to, long long first, int rows, int col, int cols) {
    constexpr int kBlocks = (F + 1) / 2, kFours = F == 1 ? 2 : 4;
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave, r = lane & 31, h = lane >> 5;
#pragma unroll
    for (int x = 0; x < F; ++x)
#pragma unroll
        for (int y = 0; y < kBlocks; ++y) {
            float v[kFours][4];
            uint32_t most = 0;
#pragma unroll
            for (int q = 0; q < kFours; ++q) {
                const f32x4 s = sums(x, y, q);
#pragma unroll
                for (int i = 0; i < 4; ++i) {                    // (columns that are not there have another row's sums)
                    v[q][i] = WHOLE || 32 * y + 8 * q + 4 * h + i < cols ? s[i] : 0.0f;
                    most = max(most, float_bits(v[q][i]) & 0x7fffffffu);
                }
            }
            const u32x2 both = exchange(most, most);
            most = max(both[0], both[1]);
            if constexpr (F == 1) {
                tops[wave * 32 + r] = most;
                __syncthreads();
                most = max(most, tops[(wave ^ 1) * 32 + r]);
                __syncthreads();
            }
            const uint32_t code = scale8_code(most);
            const float inverse = scale8_inverse(code);
            uint32_t w[kFours];
#pragma unroll
            for (int q = 0; q < kFours; ++q) w[q] = encode8_four(v[q], inverse, code == 255u);
            const int k = col + 32 * y;                          // (a multiple of 32, or of 16 with F == 1)
            const long long at = (first + 32 * x + r) * to.blocks + k / kMx8Block;
            uint8_t* p = to.codes + at * kMx8Block + k % kMx8Block;
            const bool there = 32 * x + r < rows && (WHOLE || k / kMx8Block < to.blocks);
            if constexpr (F == 1) {
                const u32x2 eight = exchange(w[0], w[1]);
                if (there) *reinterpret_cast<u32x2*>(p + 8 * h) = eight;
            } else {
                const u32x2 a = exchange(w[0], w[kFours / 2]), b = exchange(w[1], w[kFours - 1]);
                if (there) *reinterpret_cast<u32x4*>(p + 16 * h) = u32x4{a[0], a[1], b[0], b[1]};
            }
            if (there && h == 0 && k % kMx8Block == 0) to.scales[at] = (uint8_t)code;
        }
}

// A gated wave's tile of 32 * F x 16 * F outputs.  `all`: the workgroup's LDS, which nobody else needs any more.
template <int F, int ACT>
__device__ __forceinline__ void store_gated(const f32x16 (&acc)[F][F], uint32_t lds, uint8_t* all, void* out, int type, long long first,
                                            long long ld, int rows, int col, int cols, const Act& act, const Mx8& saved, int M) {
    settled<F>();
    auto gate = [&](int x, int y, int q) { return four_gate<F>(acc, x, y, q); };
    auto up = [&](int x, int y, int q) { return four_up<F>(acc, x, y, q); };
    if (saved.codes) {
        uint32_t* tops = reinterpret_cast<uint32_t*>(all);
        // (with F == 1 a wave's 16 columns may be all there and its neighbour's not: both take the same branch, for the barriers)
        const int left = F == 1 ? cols + (col & 16) - 16 : cols;
        if (left >= 16 * F) {
            save_tile<F, true>(gate, tops, saved, first, rows, col, cols);
            save_tile<F, true>(up, tops, saved, M + first, rows, col, cols);
        } else {
            save_tile<F, false>(gate, tops, saved, first, rows, col, cols);
            save_tile<F, false>(up, tops, saved, M + first, rows, col, cols);
        }
    }
    auto sums = [&](int x, int y, int q) {
        const f32x4 g = gate(x, y, q), u = up(x, y, q);
        f32x4 v;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = act_value<ACT>(act, g[i]) * u[i];
        return v;
    };
    if (type == APB_F32) store_tile_as<APB_F32, F, true>(sums, lds, out, first, ld, rows, col, cols);
    else if (type == APB_BF16) store_tile_as<APB_BF16, F, true>(sums, lds, out, first, ld, rows, col, cols);
    else store_tile_as<APB_F16, F, true>(sums, lds, out, first, ld, rows, col, cols);
}

// A workgroup computes a tile of 64 * F x 64 * F outputs, a wave 32 * F x 32 * F.  A pass sums over half a segment, 128 values, in
// two steps of 64.  The rows' half segments go from memory straight to LDS, three passes ahead of the one being multiplied, and
// from there to registers a step ahead.  What keeps the matrix cores fed is the order of the instructions: a wave issues them one
// by one, a load or an LDS read that finds its queue full holds up the matrix instructions behind it, so every two of those are
// followed by one read for the next step and every few by one load.  In LDS the four 16-byte chunks of a half segment are
// permuted by the row's number (by exchanging what the lanes of a load ask for), so that 16 lanes reading the same chunk of 16
// rows meet every bank once.  Lane (r, h) holds 32 values of row r: step s multiplies blocks s (h = 0) and 2 + s (h = 1) of the
// half segment.  Rows of B go in the first operand: a lane then holds four neighbours of a row of Y.
//
// ACT, if not -1, is an apb_activation: both projections of a gated block.  Of the 32 * F rows of B that a wave multiplies, the first
// half are the gate's, the second the up projection's for the same 16 * F columns of Y, so a lane holds both factors of each of its
// outputs; N counts the columns of Y, the tile has 32 * F of them.  `saved`: where G and U go in 8 bits, if anywhere.
template <int F, int ACT>
__global__ __launch_bounds__(kThreads, F == 4 ? 1 : 2) void k_mx4_gemm(Mx A, Mx B, const int32_t* __restrict__ offsets, int E, int N,
                                                                       int tiles_n, int type, void* __restrict__ Y, long long ldy,
                                                                       Act act, Mx8 saved) {
    constexpr bool GATED = ACT >= 0;
    constexpr int kRows = 64 * F;                                // of either operand
    constexpr int kCols = GATED ? kRows / 2 : kRows;             // of the tile
    constexpr int kLoads = 2 * kRows / 16 / 4;                   // instructions of a wave that fetch a pass's codes
    constexpr int kScaleLoads = F == 4 ? 2 : 1;                  // ... its scales
    constexpr int kPass = kLoads + kScaleLoads;
    constexpr int kStage = 2 * kRows * (kHalfBytes + 4);
    __shared__ __align__(512) uint8_t lds[kRing * kStage];
    int tile, nt;
    tile_of(blockIdx.x, tiles_n, tile, nt);
    const RowTile t = find_row_tile(offsets, E, A.rows, kRows, tile);
    if (t.rows <= 0) return;
    const int n0 = nt * kCols;
    const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int r = lane & 31, h = lane >> 5;
    const int wm = (wave >> 1) * 32 * F, wn = (wave & 1) * 32 * F;
    if (t.e >= E) {
        const float zero[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        for (int i = threadIdx.x; i < t.rows * (kCols / 4); i += kThreads) {
            const int row = t.row0 + i / (kCols / 4), n = n0 + i % (kCols / 4) * 4;
            store4(Y, type, (long long)row * ldy + n, zero, N - n);
            if (GATED && saved.codes && n < saved.blocks * kMx8Block)
                for (int u = 0; u < 2; ++u) {
                    const long long at = ((long long)(u ? A.rows : 0) + row) * saved.blocks + n / kMx8Block;
                    *reinterpret_cast<uint32_t*>(saved.codes + at * kMx8Block + n % kMx8Block) = 0u;
                    if (n % kMx8Block == 0) saved.scales[at] = 0;
                }
        }
        return;
    }
    f32x16 acc[F][F];
#pragma unroll
    for (int x = 0; x < F; ++x)
#pragma unroll
        for (int y = 0; y < F; ++y)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[x][y][i] = 0.0f;

    // waves 0 and 1 fetch A's rows, 2 and 3 B's; rows beyond the tile's repeat its last one
    const bool fetch_b = wave >= 2;
    const int q0 = fetch_b ? (GATED ? 2 : 1) * t.e * N + n0 : t.row0, last = fetch_b ? N - 1 - n0 : t.rows - 1;
    // the row that takes place `row` of an operand in LDS, relative to q0, and whether it is one of the up projection's, N rows further
    auto row_at = [&](int row) { return min(GATED && fetch_b ? row / (32 * F) * 16 * F + (row & (16 * F - 1)) : row, last); };
    auto is_up = [&](int row) { return GATED && fetch_b && (row & (32 * F - 1)) >= 16 * F; };
    const uint32_t pitch = (uint32_t)A.segs * kMxSegBytes;
    const size_t up = GATED && fetch_b ? (size_t)N * pitch : 0;
    const uint8_t* codes = (fetch_b ? B.codes : A.codes) + (size_t)q0 * pitch;
    const uint8_t* scales = (fetch_b ? B.scales : A.scales) + (size_t)q0 * 8;
    const size_t scale_pitch = (size_t)(fetch_b ? B.rows : A.rows) * 8;
    uint32_t at[kLoads], scale_at[kScaleLoads];
    const int first = F == 1 ? 0 : (wave & 1) * (kRows / 2);     // (64 scales are one load: both waves fetch them)
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
        const int row = (wave & 1) * (kRows / 2) + 16 * i + (lane >> 2);
        at[i] = row_at(row) * pitch + 16 * ((lane & 3) ^ ((row >> 2) & 3));
    }
#pragma unroll
    for (int i = 0; i < kScaleLoads; ++i) {
        const int row = first + 64 * i + lane;
        scale_at[i] = 8 * (row_at(row) + (is_up(row) ? N : 0));
    }
    const uint32_t lds0 = __builtin_amdgcn_readfirstlane(lds_address(lds));
    const uint32_t to = lds0 + wave * kLoads * 1024;
    const uint32_t scales_to = lds0 + 2 * kRows * kHalfBytes + (fetch_b ? 4 * kRows : 0) + 4 * first;

    // the loads of a pass into a stage, one by one
    const uint8_t *codes_from, *scales_from;
    uint32_t codes_to, marks_to;
    auto aim = [&](int stage, int pass) {
        codes_from = codes + (size_t)pass * kHalfBytes;
        scales_from = scales + (size_t)(pass >> 1) * scale_pitch + 4 * (pass & 1);
        codes_to = to + stage;
        marks_to = scales_to + stage;
    };
    auto fetch = [&](int i) {
        // (of B's rows the second half of the loads are the up projection's)
        if (i < kLoads) load16_to_lds(codes_to + 1024 * i, GATED && i >= kLoads / 2 ? codes_from + up : codes_from, at[i]);
        else load4_to_lds(marks_to + 256 * (i - kLoads), scales_from, scale_at[i - kLoads]);
    };
    u32x4 fm[2][F], fn[2][F];
    int vm[2][F], vn[2][F];
    const uint8_t* row_m = lds + (wm + r) * kHalfBytes;
    const uint8_t* row_n = lds + (kRows + wn + r) * kHalfBytes;
    const uint8_t* marks = lds + 2 * kRows * kHalfBytes + 4 * r + 2 * h;
    // the reads of a step's operands, one by one, and of a pass's scales
    auto read = [&](int i, int stage, int s) {
        const int at = stage + 16 * ((2 * h + s) ^ ((r >> 2) & 3));
        if (i < F) fn[s][i] = *reinterpret_cast<const u32x4*>(row_n + 32 * i * kHalfBytes + at);
        else fm[s][i - F] = *reinterpret_cast<const u32x4*>(row_m + 32 * (i - F) * kHalfBytes + at);
    };
    auto read_scales = [&](int stage, int (&m)[F], int (&n)[F]) {
#pragma unroll
        for (int f = 0; f < F; ++f) {
            n[f] = *reinterpret_cast<const uint16_t*>(marks + stage + 4 * (kRows + wn + 32 * f));
            m[f] = *reinterpret_cast<const uint16_t*>(marks + stage + 4 * (wm + 32 * f));
        }
    };
    const int passes = 2 * A.segs;
#pragma unroll
    for (int p = 0; p < kRing - 1; ++p) {
        aim(p * kStage, min(p, passes - 1));
#pragma unroll
        for (int i = 0; i < kPass; ++i) fetch(i);
    }
    arrived<(kRing - 2) * kPass>();
#pragma unroll
    for (int i = 0; i < 2 * F; ++i) read(i, 0, 0);
    read_scales(0, vm[0], vn[0]);
    aim((kRing - 1) * kStage, min(kRing - 1, passes - 1));
#pragma unroll
    for (int i = 0; i < kPass / 2; ++i) fetch(i);                // (the other half under the first step's products)
    int now = 0;
    // Passes go in pairs, which is how a segment has them.  (Beyond the last pass it is fetched again: no branch in the loop.)
    for (int pass = 0; pass < passes; pass += 2) {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int next = now == (kRing - 1) * kStage ? 0 : now + kStage;
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                if (s == 1) {
                    // this pass's place is free and the next pass is there
                    arrived<(kRing - 2) * kPass>();
                    aim(now, min(pass + half + kRing, passes - 1));
                    read_scales(next, vm[1 - half], vn[1 - half]);
                }
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int i = 0; i < F * F; ++i) {
                    const int x = i / F, y = i % F;
                    acc[x][y] = s == 0 ? mfma32<0>(fn[0][y], fm[0][x], acc[x][y], vn[half][y], vm[half][x])
                                       : mfma32<1>(fn[1][y], fm[1][x], acc[x][y], vn[half][y], vm[half][x]);
                    // F * F products of a step, 2 * F reads; from one arrived() to the next kPass loads under 2 * F * F products
                    constexpr int kEach = F * F / (2 * F) > 0 ? F * F / (2 * F) : 1;
                    if (i % kEach == kEach - 1) {
#pragma unroll
                        for (int u = 0; u < (F == 1 ? 2 : 1); ++u)
                            if (s == 0) read(i / kEach * (F == 1 ? 2 : 1) + u, now, 1);
                            else read(i / kEach * (F == 1 ? 2 : 1) + u, next, 0);
                    }
                    const int slot = (s == 1 ? 0 : F * F) + i;   // products since arrived()
                    const int begin = slot * kPass / (2 * F * F), end = (slot + 1) * kPass / (2 * F * F);
#pragma unroll
                    for (int j = begin; j < end; ++j) fetch(j);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            now = next;
        }
    }
    arrived<0>();                                                // (nothing is under way to LDS any more)
    static_assert(4 * kTileLds<F> <= kRing * kStage, "a wave's tile passes through its share of the ring");
    if constexpr (GATED) {
        store_gated<F, ACT>(acc, lds0 + wave * kTileLds<F>, lds, Y, type, t.row0 + wm, ldy, min(32 * F, t.rows - wm), n0 + wn / 2, N - n0 - wn / 2,
                       act, saved, A.rows);
    } else {
        store_tile<F>(acc, lds0 + wave * kTileLds<F>, Y, type, t.row0 + wm, ldy, min(32 * F, t.rows - wm), n0 + wn, N - n0 - wn);
    }
}

template <int F, int ACT>
void launch_tiles(const Mx& A, const Mx& B, const int32_t* offsets, int E, int M, int N, int type, void* Y, long long ldy, const Act& act,
                  const Mx8& saved, hipStream_t s) {
    constexpr int kCols = ACT >= 0 ? 32 * F : 64 * F;
    const long long tiles_m = (max_row_tiles(M, E, offsets != nullptr, 64 * F) + 3) / 4 * 4;
    const int tiles_n = (N + kCols - 1) / kCols;
    const unsigned blocks = (unsigned)((tiles_m * tiles_n + 127) / 128 * 128);
    hipLaunchKernelGGL((k_mx4_gemm<F, ACT>), dim3(blocks), dim3(kThreads), 0, s, A, B, offsets, E, N, tiles_n, type, Y, ldy, act, saved);
}

int launch_mx4_gated(const Mx& A, const Mx& B, const int32_t* offsets, int E, int M, int N, int activation, int type, void* Y,
                     long long ldy, void* saved, hipStream_t s) {
    const int side = mx4_gated_side(M, N, E, offsets != nullptr);
    const Act act = act_of(activation);
    const Mx8 keep = mx8_view(saved, 2LL * M, N);
    auto with = [&](auto kind) {
        constexpr int kAct = decltype(kind)::value;
        if (side == 256) launch_tiles<4, kAct>(A, B, offsets, E, M, N, type, Y, ldy, act, keep, s);
        else if (side == 128) launch_tiles<2, kAct>(A, B, offsets, E, M, N, type, Y, ldy, act, keep, s);
        else launch_tiles<1, kAct>(A, B, offsets, E, M, N, type, Y, ldy, act, keep, s);
    };
    if (activation == APB_SILU) with(std::integral_constant<int, APB_SILU>{});
    else if (activation == APB_GELU) with(std::integral_constant<int, APB_GELU>{});
    else with(std::integral_constant<int, APB_RELU>{});
    APB_HIP(hipGetLastError());
    return APB_OK;
}

// The sizes of a gated product; N counts the columns of Y.  saved: both projections go to an 8-bit matrix, which has limits of its own.
bool bad_gated(int E, int M, int N, int K, const int32_t* offsets, bool saved) {
    return N <= 0 || N > kMxMaxK || bad_product(E, M, 2 * N, K, offsets) || (saved && bad_shape_mx8(2LL * M, N));
}

}  // namespace

int launch_mx4_gemm(const Mx& A, const Mx& B, const int32_t* offsets, int E, int M, int N, int type, void* Y, long long ldy,
                    hipStream_t s) {
    const int side = mx4_product_side(M, N);
    const Act none = {};
    const Mx8 nowhere = {};
    if (side == 256) launch_tiles<4, -1>(A, B, offsets, E, M, N, type, Y, ldy, none, nowhere, s);
    else if (side == 128) launch_tiles<2, -1>(A, B, offsets, E, M, N, type, Y, ldy, none, nowhere, s);
    else launch_tiles<1, -1>(A, B, offsets, E, M, N, type, Y, ldy, none, nowhere, s);
    APB_HIP(hipGetLastError());
    return APB_OK;
}

}  // namespace apb

using namespace apb;

extern "C" {

int apb_mx4_gemm(const void* A, const void* B, const int32_t* offsets, int E, int M, int N, int K, int type, void* Y,
                 long long ldy, void* stream) {
    if (!A || !B || !Y) return APB_ERR_NULL;
    if (bad_type(type)) return APB_ERR_TYPE;
    if (bad_product(E, M, N, K, offsets) || ldy < N) return APB_ERR_SHAPE;
    if (!aligned(A, 16) || !aligned(B, 16) || !aligned(Y, type_size(type)) || !aligned(offsets, 4)) return APB_ERR_ALIGN;
    const Mx a = mx_view(A, M, K), b = mx_view(B, E * N, K);
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    if (mx4_few_applies(offsets, E, M, K)) return launch_mx4_few(a, b, offsets, E, M, N, K, type, Y, ldy, s);
    return launch_mx4_gemm(a, b, offsets, E, M, N, type, Y, ldy, s);
}

size_t apb_mx4_linear_scratch_bytes(int grouped, int E, int M, int N, int K) {
    const int32_t some = 0, *offsets = grouped ? &some : nullptr;
    if (bad_product(E, M, N, K, offsets) || mx4_few_applies(offsets, E, M, K)) return 0;
    return apb_mx4_bytes(M, K);
}

int apb_mx4_linear(const void* X, int x_type, long long ldx, int rows_in, const int32_t* rows_from, const void* W,
                   const int32_t* offsets, int E, int M, int N, int K, void* scratch, int y_type, void* Y, long long ldy,
                   void* stream) {
    if (!X || !W || !scratch || !Y) return APB_ERR_NULL;
    if (bad_type(x_type) || bad_type(y_type)) return APB_ERR_TYPE;
    if (bad_product(E, M, N, K, offsets) || ldy < N || ldx < K || rows_in <= 0 || (!rows_from && rows_in != M)) return APB_ERR_SHAPE;
    if (!aligned(X, type_size(x_type)) || !aligned(W, 16) || !aligned(scratch, 16) || !aligned(Y, type_size(y_type)) ||
        !aligned(offsets, 4) || !aligned(rows_from, 4))
        return APB_ERR_ALIGN;
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    if (mx4_few_applies(offsets, E, M, K))
        return launch_mx4_few(X, x_type, ldx, rows_in, rows_from, mx_view(W, E * N, K), offsets, E, M, N, K, y_type, Y, ldy, s);
    const int rc = launch_mx4_quantize(X, x_type, ldx, 1, rows_in, rows_from, M, K, scratch, s);
    if (rc != APB_OK) return rc;
    return launch_mx4_gemm(mx_view(scratch, M, K), mx_view(W, E * N, K), offsets, E, M, N, y_type, Y, ldy, s);
}

int apb_mx4_gated_gemm(const void* A, const void* W, const int32_t* offsets, int E, int M, int N, int K, int activation, int type,
                       void* Y, long long ldy, void* saved, void* stream) {
    if (!A || !W || !Y) return APB_ERR_NULL;
    if (bad_type(type)) return APB_ERR_TYPE;
    if (bad_activation(activation)) return APB_ERR_VALUE;
    if (bad_gated(E, M, N, K, offsets, saved != nullptr) || ldy < N) return APB_ERR_SHAPE;
    if (!aligned(A, 16) || !aligned(W, 16) || !aligned(Y, type_size(type)) || !aligned(offsets, 4) || !aligned(saved, 16)) return APB_ERR_ALIGN;
    const Mx a = mx_view(A, M, K), w = mx_view(W, E * 2 * N, K);
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    if (!saved && mx4_few_gated_applies(offsets, E, M, N, K)) return launch_mx4_few_gated(a, w, offsets, E, M, N, K, activation, type, Y, ldy, s);
    return launch_mx4_gated(a, w, offsets, E, M, N, activation, type, Y, ldy, saved, s);
}

size_t apb_mx4_gated_linear_scratch_bytes(int grouped, int E, int M, int N, int K, int with_saved) {
    const int32_t some = 0, *offsets = grouped ? &some : nullptr;
    if (bad_gated(E, M, N, K, offsets, with_saved != 0) || (!with_saved && mx4_few_gated_applies(offsets, E, M, N, K))) return 0;
    return apb_mx4_bytes(M, K);
}

int apb_mx4_gated_linear(const void* X, int x_type, long long ldx, int rows_in, const int32_t* rows_from, const void* W,
                         const int32_t* offsets, int E, int M, int N, int K, int activation, void* scratch, int y_type, void* Y,
                         long long ldy, void* saved, void* stream) {
    if (!X || !W || !scratch || !Y) return APB_ERR_NULL;
    if (bad_type(x_type) || bad_type(y_type)) return APB_ERR_TYPE;
    if (bad_activation(activation)) return APB_ERR_VALUE;
    if (bad_gated(E, M, N, K, offsets, saved != nullptr) || ldy < N || ldx < K || rows_in <= 0 || (!rows_from && rows_in != M))
        return APB_ERR_SHAPE;
    if (!aligned(X, type_size(x_type)) || !aligned(W, 16) || !aligned(scratch, 16) || !aligned(Y, type_size(y_type)) ||
        !aligned(offsets, 4) || !aligned(rows_from, 4) || !aligned(saved, 16))
        return APB_ERR_ALIGN;
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    const Mx w = mx_view(W, E * 2 * N, K);
    if (!saved && mx4_few_gated_applies(offsets, E, M, N, K))
        return launch_mx4_few_gated(X, x_type, ldx, rows_in, rows_from, w, offsets, E, M, N, K, activation, y_type, Y, ldy, s);
    const int rc = launch_mx4_quantize(X, x_type, ldx, 1, rows_in, rows_from, M, K, scratch, s);
    if (rc != APB_OK) return rc;
    return launch_mx4_gated(mx_view(scratch, M, K), w, offsets, E, M, N, activation, y_type, Y, ldy, saved, s);
}

}  // extern "C"
