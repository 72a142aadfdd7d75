// Products of two 4-bit matrices, Y = A^ B^T, plain or grouped by expert.
#include "apb_mx4.h"

namespace apb {
namespace {

constexpr int kThreads = 256;                 // four waves, two by two

// Every wave's loads are in LDS and every wave's reads of LDS before this point have been answered.
__device__ __forceinline__ void arrived() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); }
// Which tile a workgroup takes: workgroups go to the eight XCDs in turn, and sixteen in a row on one XCD take a block of 4 x 4
// tiles, which shares its operands in that XCD's cache.
__device__ __forceinline__ void tile_of(int id, int tiles_n, int& t, int& n) {
    const int xcd = id & 7, j = id >> 3;
    const int linear = (j >> 4) * 128 + xcd * 16 + (j & 15);
    const int super = linear / (4 * tiles_n), rest = linear - super * 4 * tiles_n;
    t = super * 4 + (rest & 3);
    n = rest >> 2;
}

// A workgroup computes a tile of 64 * F x 64 * F outputs, a wave 32 * F x 32 * F.  The rows' segments of 256 values (a line of
// 128 bytes each) go from memory straight to LDS, one segment ahead of the one being multiplied, and from there to registers
// one step (64 values) ahead.  In LDS the eight 16-byte chunks of a line are permuted by the row's number (by exchanging what the
// lanes of a load ask for), so that 32 lanes reading the same chunk of 32 rows meet every bank equally often.  Lane (r, h)
// holds 32 values of row r: step s multiplies block s (h = 0) and block 4 + s (h = 1) of the segment, so that a lane's four
// scales are one word.  Rows of B go in the first operand: a lane then holds four neighbours of a row of Y.
template <int F>
__global__ __launch_bounds__(kThreads, F == 4 ? 1 : 2) void k_mx4_gemm(Mx A, Mx B, const int32_t* __restrict__ offsets, int E, int N,
                                                                       int tiles_n, int type, void* __restrict__ Y, long long ldy) {
    constexpr int kRows = 64 * F;                                // of either operand
    constexpr int kLoads = 2 * kRows / 8 / 4;                    // instructions of a wave that fetch a segment's codes
    constexpr int kScaleLoads = 2 * kRows / 32 / 4;              // ... its scales
    constexpr int kStage = 2 * kRows * (kMxSegBytes + 8);
    __shared__ __align__(16) uint8_t lds[2 * kStage];
    int tile, nt;
    tile_of(blockIdx.x, tiles_n, tile, nt);
    const RowTile t = find_row_tile(offsets, E, A.rows, kRows, tile);
    if (t.rows <= 0) return;
    const int n0 = nt * kRows;
    const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int r = lane & 31, h = lane >> 5;
    const int wm = (wave >> 1) * 32 * F, wn = (wave & 1) * 32 * F;
    if (t.e >= E) {
        const float zero[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        for (int i = threadIdx.x; i < t.rows * (kRows / 4); i += kThreads) {
            const int n = n0 + i % (kRows / 4) * 4;
            store4(Y, type, (long long)(t.row0 + i / (kRows / 4)) * ldy + n, zero, N - n);
        }
        return;
    }
    const int segs = A.segs;
    f32x16 acc[F][F];
#pragma unroll
    for (int x = 0; x < F; ++x)
#pragma unroll
        for (int y = 0; y < F; ++y)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[x][y][i] = 0.0f;

    // waves 0 and 1 fetch A's rows, 2 and 3 B's; rows beyond the tile's repeat its last one
    const bool fetch_b = wave >= 2;
    const int q0 = fetch_b ? t.e * N + n0 : t.row0, last = fetch_b ? N - 1 - n0 : t.rows - 1;
    const uint32_t pitch = (uint32_t)A.segs * kMxSegBytes;
    const uint8_t* codes = (fetch_b ? B.codes : A.codes) + (size_t)q0 * pitch;
    const uint8_t* scales = (fetch_b ? B.scales : A.scales) + (size_t)q0 * 8;
    const size_t scale_pitch = (size_t)(fetch_b ? B.rows : A.rows) * 8;
    uint32_t at[kLoads], scale_at[kScaleLoads];
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
        const int row = (wave & 1) * (kRows / 2) + 8 * i + (lane >> 3);
        at[i] = min(row, last) * pitch + 16 * ((lane & 7) ^ (row & 7));
    }
#pragma unroll
    for (int i = 0; i < kScaleLoads; ++i)
        scale_at[i] = 8 * min((wave & 1) * (kRows / 2) + 32 * i + (lane >> 1), last) + 4 * (lane & 1);
    const uint32_t lds0 = __builtin_amdgcn_readfirstlane(lds_address(lds));
    const uint32_t to = lds0 + wave * kLoads * 1024, scales_to = lds0 + 2 * kRows * kMxSegBytes + wave * kScaleLoads * 256;

    auto fetch = [&](int stage, int seg) {
        const uint8_t* p = codes + (size_t)seg * kMxSegBytes;
        const uint8_t* q = scales + (size_t)seg * scale_pitch;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) load16_to_lds(to + stage + 1024 * i, p, at[i]);
#pragma unroll
        for (int i = 0; i < kScaleLoads; ++i) load4_to_lds(scales_to + stage + 256 * i, q, scale_at[i]);
    };
    u32x4 fm[2][F], fn[2][F];
    int vm[F], vn[F], next_m[F], next_n[F];
    const uint8_t* row_m = lds + (wm + r) * kMxSegBytes;
    const uint8_t* row_n = lds + (kRows + wn + r) * kMxSegBytes;
    const uint8_t* row_s = lds + 2 * kRows * kMxSegBytes + 8 * r + 4 * h;
    auto read = [&](int from, int s, u32x4 (&m)[F], u32x4 (&n)[F]) {
        const int at = from + 16 * ((4 * h + s) ^ (r & 7));
#pragma unroll
        for (int f = 0; f < F; ++f) {
            m[f] = *reinterpret_cast<const u32x4*>(row_m + 32 * f * kMxSegBytes + at);
            n[f] = *reinterpret_cast<const u32x4*>(row_n + 32 * f * kMxSegBytes + at);
        }
    };
    auto read_scales = [&](int from, int (&m)[F], int (&n)[F]) {
#pragma unroll
        for (int f = 0; f < F; ++f) {
            m[f] = *reinterpret_cast<const int*>(row_s + from + 8 * (wm + 32 * f));
            n[f] = *reinterpret_cast<const int*>(row_s + from + 8 * (kRows + wn + 32 * f));
        }
    };
    // (reads stay ahead of the products they are hidden under)
#define APB_MULTIPLY(S, SET)                                                                               \
    __builtin_amdgcn_sched_barrier(0);                                                                     \
    _Pragma("unroll") for (int x = 0; x < F; ++x) _Pragma("unroll") for (int y = 0; y < F; ++y)            \
        acc[x][y] = mfma32<S>(fn[SET][y], fm[SET][x], acc[x][y], vn[y], vm[x]);                              \
    __builtin_amdgcn_sched_barrier(0)
    // A segment per pass.  The last step's operands are in registers before the barrier, behind which the segment after next takes
    // this one's place in LDS and the next one's first operands are read, under the last step's products.  (The last segment is
    // fetched again where there is none after it: no branch in the loop.)
    fetch(0, 0);
    arrived();
    fetch(kStage, min(1, segs - 1));
    read(0, 0, fm[0], fn[0]);
    read_scales(0, vm, vn);
    int now = 0;
    for (int seg = 0; seg < segs; ++seg) {
        read(now, 1, fm[1], fn[1]);
        APB_MULTIPLY(0, 0);
        read(now, 2, fm[0], fn[0]);
        APB_MULTIPLY(1, 1);
        read(now, 3, fm[1], fn[1]);
        APB_MULTIPLY(2, 0);
        arrived();
        fetch(now, min(seg + 2, segs - 1));
        now = kStage - now;
        read(now, 0, fm[0], fn[0]);
        read_scales(now, next_m, next_n);
        APB_MULTIPLY(3, 1);
#pragma unroll
        for (int f = 0; f < F; ++f) {
            vm[f] = next_m[f];
            vn[f] = next_n[f];
        }
    }
    arrived();                                                   // (nothing is under way to LDS when the workgroup ends)
#pragma unroll
    for (int x = 0; x < F; ++x) {
        const int m = wm + 32 * x + r;
        if (m >= t.rows) continue;
        const long long row = (long long)(t.row0 + m) * ldy;
#pragma unroll
        for (int y = 0; y < F; ++y)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int n = n0 + wn + 32 * y + 8 * g + 4 * h;
                const float v[4] = {acc[x][y][4 * g], acc[x][y][4 * g + 1], acc[x][y][4 * g + 2], acc[x][y][4 * g + 3]};
                store4(Y, type, row + n, v, N - n);
            }
    }
}

template <int F>
void launch_tiles(const Mx& A, const Mx& B, const int32_t* offsets, int E, int M, int N, int type, void* Y, long long ldy, hipStream_t s) {
    const long long tiles_m = (max_row_tiles(M, E, offsets != nullptr, 64 * F) + 3) / 4 * 4;
    const int tiles_n = (N + 64 * F - 1) / (64 * F);
    const unsigned blocks = (unsigned)((tiles_m * tiles_n + 127) / 128 * 128);
    hipLaunchKernelGGL((k_mx4_gemm<F>), dim3(blocks), dim3(kThreads), 0, s, A, B, offsets, E, N, tiles_n, type, Y, ldy);
}

}  // namespace

int launch_mx4_gemm(const Mx& A, const Mx& B, const int32_t* offsets, int E, int M, int N, int type, void* Y, long long ldy,
                    hipStream_t s) {
    const long long big = ((long long)M + 255) / 256 * ((N + 255) / 256);
    if (big >= 192) launch_tiles<4>(A, B, offsets, E, M, N, type, Y, ldy, s);
    else if (big * 4 >= 192) launch_tiles<2>(A, B, offsets, E, M, N, type, Y, ldy, s);
    else launch_tiles<1>(A, B, offsets, E, M, N, type, Y, ldy, s);
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

}  // extern "C"
