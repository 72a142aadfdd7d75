// Low-rank adapters of many requests: T = scale X A^T (down), Y = Y0 + T B (up), dA = sum T^T X (gradient), every row with the factors of
// its segment's adapter.  A and B have their long side contiguous, so that each of them and each of the gradients' operands is read
// in whole lines and all directions are these three kernels.
#include <type_traits>

#include "apb_adapter_shape.h"
#include "apb_mx8.h"

namespace apb {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kAdapterWaves;
static_assert(kThreads == kWaves * kWave, "a workgroup of up and of the join");
constexpr int kList = 1024;                    // rows of an adapter whose numbers a workgroup of the gradient holds at a time
constexpr int kStage = 64;                    // ranks of T that are in LDS at a time

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

struct Segments {
    const int32_t *offsets, *adapter;
    int S, L, M;
};

// Segment s's adapter, -1 for none; first row and number of rows.  (Loads that do not wait for one another.)
__device__ __forceinline__ int rows_of(const Segments& seg, int s, int& first, int& count) {
    const int at = min(s, seg.S - 1);
    const int a = seg.adapter ? seg.adapter[at] : at;
    first = seg.offsets ? min(max(seg.offsets[at], 0), seg.M) : 0;
    count = (seg.offsets ? max(first, min(seg.offsets[at + 1], seg.M)) : seg.M) - first;
    if (s >= seg.S) count = 0;
    return s < seg.S && a >= 0 && a < seg.L ? a : -1;
}

// The t-th tile of `tile` rows: its rows, none of two segments, and their adapter.  Called by whole waves, like find_row_tile; the rows
// behind the last segment are tiles as well.
struct SegmentTile {
    int a, row0, rows;
};
__device__ __forceinline__ SegmentTile find_tile(const Segments& seg, int tile, int t) {
    const int lane = threadIdx.x & (kWave - 1);
    int before = 0, behind = 0;
    for (int base = 0; base <= seg.S; base += kWave) {
        const int s = base + lane;
        int first, count;
        const int a = rows_of(seg, s, first, count);
        const int last = __shfl(first + count, min(seg.S - 1 - base, kWave - 1), kWave);      // (of segments so far)
        if (s == seg.S) {
            first = base == seg.S ? behind : last;
            count = seg.M - first;
        }
        behind = last;
        const int tiles = (count + tile - 1) / tile;
        int upto = tiles;
#pragma unroll
        for (int d = 1; d < kWave; d <<= 1) {
            const int v = __shfl_up(upto, d, kWave);
            if (lane >= d) upto += v;
        }
        const unsigned long long hit = __ballot(t < before + upto);
        if (hit) {
            const int src = __builtin_amdgcn_readfirstlane(__ffsll((long long)hit) - 1);
            const int from = __builtin_amdgcn_readlane(before + upto - tiles, src);
            const int row0 = __builtin_amdgcn_readlane(first, src) + (t - from) * tile;
            const int end = __builtin_amdgcn_readlane(first + count, src);
            return SegmentTile{__builtin_amdgcn_readlane(a, src), row0, min(tile, end - row0)};
        }
        before += __builtin_amdgcn_readlane(upto, kWave - 1);
    }
    return SegmentTile{-1, 0, 0};
}

// d[i, n] += sum over eight values of each of the four lanes of a row: a's row i in lanes i, i + 16, ..., b's row n likewise.
template <int TYPE>
__device__ __forceinline__ f32x4 multiply8(const Eight<TYPE>& a, const Eight<TYPE>& b, f32x4 d) {
    if constexpr (TYPE == APB_BF16) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a.w[0]), __builtin_bit_cast(bf16x8, b.w[0]), d, 0, 0, 0);
    } else if constexpr (TYPE == APB_F16) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a.w[0]), __builtin_bit_cast(f16x8, b.w[0]), d, 0, 0, 0);
    } else {
        float x[8], y[8];
        floats(a, x);
        floats(b, y);
#pragma unroll
        for (int q = 0; q < 8; ++q) d = __builtin_amdgcn_mfma_f32_16x16x4f32(x[q], y[q], d, 0, 0, 0);
        return d;
    }
}

// A workgroup takes `tile` rows of a segment, up to 16 * RT, 16 * JT ranks and one part of K; its waves take lines of 128 bytes of all those rows in
// turn and join their sums in LDS.  A line is loaded by eight neighbouring lanes and goes through LDS of the wave's own: in the order
// of the operands, sixteen neighbouring lanes would ask for sixteen lines, and a compute unit would be brought 17 bytes a cycle.  The
// next lines are under way while these are multiplied.  In LDS the eight 16-byte pieces of a line are permuted by the row's number, so
// that eight lanes reading the same piece of eight rows meet every bank once.  8196 rows of 4096 in bfloat16: rank 16 16 us, rank 64
// 24 (67 MB are 13), in the order of the operands 24 and 50.
template <int TYPE, int RT, int JT, int WAVES>
__global__ __launch_bounds__(WAVES * kWave) void k_adapter_down(const void* __restrict__ X, long long ldx, const void* __restrict__ A,
                                                                Segments seg, const float* __restrict__ scale, int K, int r, int lines_each, int tile,
                                                                float* __restrict__ T) {
    constexpr int kW = WAVES, kPiece = TYPE == APB_F32 ? 4 : 8, kLine = 8 * kPiece;       // values of 16 and of 128 bytes
    constexpr int kLoads = 2 * (RT + JT);                        // of a wave for a line of all rows, eight rows each
    __shared__ union {
        uint8_t lines[kW][kLoads * 1024];
        f32x4 sums[kW][RT * JT][kWave];
    } lds;
    const SegmentTile t = find_tile(seg, tile, blockIdx.x);
    if (t.rows <= 0) return;
    const int j0 = blockIdx.y * 16 * JT, ranks = min(16 * JT, r - j0);
    float* out = T + ((size_t)blockIdx.z * seg.M + t.row0) * r + j0;
    const int a = t.a;
    if (a < 0) {
        for (int i = threadIdx.x; i < t.rows * ranks; i += kW * kWave) out[(size_t)(i / ranks) * r + i % ranks] = 0.0f;
        return;
    }
    const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), i = lane & 15, g = lane >> 4;
    const int sub = lane >> 3, piece = lane & 7;
    // (rows and ranks that are not there repeat the last ones)
    const uint8_t* at[kLoads];
#pragma unroll
    for (int n = 0; n < kLoads; ++n) {
        const int row = 8 * n + sub;
        const long long first = n < 2 * RT ? (t.row0 + min(row, t.rows - 1)) * ldx : ((long long)a * r + j0 + min(row - 16 * RT, ranks - 1)) * K;
        at[n] = static_cast<const uint8_t*>(n < 2 * RT ? X : A) + first * (TYPE == APB_F32 ? 4 : 2) + 16 * piece;
    }
    u32x4 v[kLoads];
    auto fetch = [&](int line) {
        const int have = K - line * kLine - kPiece * piece;
        if ((line + 1) * kLine <= K) {
#pragma unroll
            for (int n = 0; n < kLoads; ++n) v[n] = load16_any(at[n] + 128LL * line);
        } else {
#pragma unroll 1
            for (int n = 0; n < kLoads; ++n) {
                u32x4 w;
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    if constexpr (TYPE == APB_F32) {
                        w[q] = q < have ? reinterpret_cast<const uint32_t*>(at[n] + 128LL * line)[q] : 0u;
                    } else {
                        const uint16_t* p = reinterpret_cast<const uint16_t*>(at[n] + 128LL * line) + 2 * q;
                        w[q] = (2 * q < have ? (uint32_t)p[0] : 0u) | (2 * q + 1 < have ? (uint32_t)p[1] << 16 : 0u);
                    }
                }
#pragma unroll
                for (int u = 0; u < kLoads; ++u)
                    if (u == n) v[u] = w;
            }
        }
    };
    f32x4 acc[RT][JT];
#pragma unroll
    for (int x = 0; x < RT; ++x)
#pragma unroll
        for (int j = 0; j < JT; ++j) acc[x][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    uint8_t* mine = lds.lines[wave];
    auto operand = [&](int row, int h) { return *reinterpret_cast<const u32x4*>(mine + row * 128 + 16 * ((4 * h + g) ^ (row & 7))); };
    const int last = min((int)(blockIdx.z + 1) * lines_each, (K + kLine - 1) / kLine);
    int line = blockIdx.z * lines_each + wave;
    if (line < last) fetch(line);
    for (; line < last; line += kW) {
#pragma unroll
        for (int n = 0; n < kLoads; ++n) *reinterpret_cast<u32x4*>(mine + (8 * n + sub) * 128 + 16 * (piece ^ sub)) = v[n];
        if (line + kW < last) fetch(line + kW);
        // (the wave's own writes and reads of LDS stay in this order)
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        Eight<TYPE> xv[TYPE == APB_F32 ? 1 : 2][RT], av[TYPE == APB_F32 ? 1 : 2][JT];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int x = 0; x < RT; ++x) xv[TYPE == APB_F32 ? 0 : h][x].w[TYPE == APB_F32 ? h : 0] = operand(16 * x + i, h);
#pragma unroll
            for (int j = 0; j < JT; ++j) av[TYPE == APB_F32 ? 0 : h][j].w[TYPE == APB_F32 ? h : 0] = operand(16 * (RT + j) + i, h);
        }
#pragma unroll
        for (int h = 0; h < (TYPE == APB_F32 ? 1 : 2); ++h)
#pragma unroll
            for (int x = 0; x < RT; ++x)
#pragma unroll
                for (int j = 0; j < JT; ++j) acc[x][j] = multiply8<TYPE>(av[h][j], xv[h][x], acc[x][j]);
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    }
    __syncthreads();
#pragma unroll
    for (int x = 0; x < RT; ++x)
#pragma unroll
        for (int j = 0; j < JT; ++j) lds.sums[wave][x * JT + j][lane] = acc[x][j];
    __syncthreads();
    const float by = scale ? scale[a] : 1.0f;
    for (int n = wave; n < RT * JT; n += kW) {
        f32x4 v = lds.sums[0][n][lane];
#pragma unroll
        for (int w = 1; w < kW; ++w) v += lds.sums[w][n][lane];
        const int row = 16 * (n / JT) + i, j = 16 * (n % JT) + 4 * g;
        if (row < t.rows)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                if (j + q < ranks) out[(size_t)row * r + j + q] = v[q] * by;
    }
}

// N values of T from `from` on, `step` apart, its parts added up in order: loads that do not wait for one another.
template <int N, class INDEX>
__device__ __forceinline__ void sum_parts(const float* __restrict__ from, const INDEX (&at)[N], int parts, size_t pitch, float (&v)[N]) {
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = from[at[e]];
    for (int p = 1; p < parts; p += 2) {
        float w[2][N];
        const float* one = from + p * pitch;
        const float* two = from + min(p + 1, parts - 1) * pitch;
#pragma unroll
        for (int e = 0; e < N; ++e) {
            w[0][e] = one[at[e]];
            w[1][e] = two[at[e]];
        }
#pragma unroll
        for (int e = 0; e < N; ++e) {
            v[e] += w[0][e];
            if (p + 1 < parts) v[e] += w[1][e];
        }
    }
}

// Rows without an adapter: Y = Y0, or zeros.
template <int TYPE>
__device__ __forceinline__ void copy_rows(const void* Y0, long long ldy0, void* Y, long long ldy, const SegmentTile& t, int c, int have, int g) {
    for (int row = g; row < t.rows; row += 4) {
        float v[8] = {};
        if (Y0) floats(load_some<TYPE>(Y0, (t.row0 + row) * ldy0 + c, have), v);
        store8<TYPE>(Y, (t.row0 + row) * ldy + c, have, v);
    }
}

// A workgroup takes 16 * RT rows of a segment and kCols columns a wave.  Products in float32: the rows' T, its parts added up, lies in
// LDS; of B a lane has eight neighbours of a row, and product t of eight takes the t-th of each lane, so that it ends up with eight
// neighbours of Y.
template <int TYPE, int RT>
__global__ __launch_bounds__(kThreads) void k_adapter_up(const float* __restrict__ T, int parts, const void* __restrict__ B, Segments seg,
                                                         int N, int r, const void* Y0, long long ldy0, void* Y, long long ldy) {
    constexpr int kPitch = kStage + 1;
    __shared__ float lds[16 * RT * kPitch];
    const SegmentTile t = find_tile(seg, 16 * RT, blockIdx.x);
    if (t.rows <= 0) return;
    const int a = t.a;
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave, i = lane & 15, g = lane >> 4;
    const int c = (blockIdx.y * kWaves + wave) * kCols + 8 * i, have = N - c;
    if (a < 0) {
        if (Y0 != Y) copy_rows<TYPE>(Y0, ldy0, Y, ldy, t, c, have, g);
        return;
    }
    f32x4 acc[RT][8];
#pragma unroll
    for (int x = 0; x < RT; ++x)
#pragma unroll
        for (int q = 0; q < 8; ++q) acc[x][q] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    for (int j0 = 0; j0 < r; j0 += kStage) {
        const int ranks = min(kStage, r - j0);
        for (int n = threadIdx.x; n < 16 * RT * kStage; n += kThreads) {
            const int row = n / kStage, j = n % kStage;
            float v[1];
            sum_parts<1>(T + (size_t)t.row0 * r + j0, {min(row, t.rows - 1) * r + min(j, ranks - 1)}, parts, (size_t)seg.M * r, v);
            lds[row * kPitch + j] = row < t.rows && j < ranks ? v[0] : 0.0f;
        }
        __syncthreads();
        for (int j = g; j - g < ranks; j += 4) {
            float b[8];
            floats(load_some<TYPE>(B, ((long long)a * r + j0 + j) * N + c, j < ranks ? have : 0), b);
#pragma unroll
            for (int x = 0; x < RT; ++x) {
                const float v = lds[(16 * x + i) * kPitch + j];
#pragma unroll
                for (int q = 0; q < 8; ++q) acc[x][q] = __builtin_amdgcn_mfma_f32_16x16x4f32(v, b[q], acc[x][q], 0, 0, 0);
            }
        }
        __syncthreads();
    }
#pragma unroll
    for (int x = 0; x < RT; ++x)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int row = 16 * x + 4 * g + q;
            if (row >= t.rows) continue;
            float v[8] = {};
            if (Y0) floats(load_some<TYPE>(Y0, (t.row0 + row) * ldy0 + c, have), v);
#pragma unroll
            for (int n = 0; n < 8; ++n) v[n] += acc[x][n][q];
            store8<TYPE>(Y, (t.row0 + row) * ldy + c, have, v);
        }
}

// ---- 16-bit factors: T as a sum of 16-bit parts ---------------------------------------------------------------------------------

// Eight floats to `PARTS` bfloat16 operands whose sum they are, to 2^-8 of each part's last: two parts 2^-16, three 2^-24.  A part stays
// finite, so that an infinity is left to the last one.
template <int PARTS>
__device__ __forceinline__ void bf16_parts(float (&t)[8], Eight<APB_BF16> (&out)[PARTS]) {
    constexpr float kMost = 3.3895314e38f;                       // the largest bfloat16
#pragma unroll
    for (int p = 0; p < PARTS; ++p) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            float v[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float& x = t[2 * q + e];
                v[e] = x;
                if (p + 1 < PARTS) {
                    v[e] = fminf(fmaxf((float)(__bf16)x, -kMost), kMost);
                    x -= v[e];
                }
            }
            out[p].w[0][q] = pack2(APB_BF16, v[0], v[1]);
        }
    }
}

// Eight rows of eight 16-bit neighbours -> eight columns of eight.
__device__ __forceinline__ void transpose8(const u32x4 (&row)[8], u32x4 (&col)[8]) {
#pragma unroll
    for (int n = 0; n < 8; ++n)
#pragma unroll
        for (int d = 0; d < 4; ++d)
            col[n][d] = __builtin_amdgcn_perm(row[2 * d + 1][n / 2], row[2 * d][n / 2], n & 1 ? 0x07060302u : 0x05040100u);
}

// ---- eight neighbours of a row of n, from element c on, by loads without a branch ---------------------------------------------------
//
// A branch around a load makes the compiler wait for the loads before it.  So a wave asks once whether all of its lanes have eight
// elements (WHOLE) and runs one of two copies of its loop; in the other one a lane loads the row's last eight and, when it uses
// them, moves those that are its own to the front.  What stands behind them is unspecified, and so is everything from c >= n on.
template <int TYPE, bool WHOLE>
__device__ __forceinline__ Eight<TYPE> load_row(const void* X, long long row, int c, int n) {
    return load_eight<TYPE>(X, row + (WHOLE ? c : min(c, n - 8)));
}
template <int TYPE, bool WHOLE>
__device__ __forceinline__ Eight<TYPE> settle(const Eight<TYPE>& x, int c, int n) {
    if constexpr (WHOLE) return x;
    const int by = n < 8 ? 0 : max(c - (n - 8), 0) & 7;          // elements to move by
    Eight<TYPE> v = x;
#pragma unroll
    for (int d = 2; d >= 1; d >>= 1)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const uint32_t from = q + d < 4 ? v.w[0][(q + d) & 3] : 0u;
            v.w[0][q] = by & (2 * d) ? from : v.w[0][q];
        }
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const uint32_t next = q < 3 ? v.w[0][(q + 1) & 3] : 0u;
        v.w[0][q] = by & 1 ? v.w[0][q] >> 16 | next << 16 : v.w[0][q];
    }
    return v;
}

// Two operands to eight ranks of a row of T.  float16 has few exponents, so the row is scaled by the power of two that takes its largest
// value (`top`, as bits) to 2^13 .. 2^14, and `back` takes the sums back: off by 2^-22 of a value or 2^-39 of the row's largest,
// whichever is more.  bfloat16: 2^-16 of a value.
template <int TYPE>
__device__ __forceinline__ void split(float (&t)[8], uint32_t top, u32x4& hi, u32x4& lo, float& back) {
    back = 1.0f;
    if constexpr (TYPE == APB_BF16) {
        Eight<APB_BF16> part[2];
        bf16_parts<2>(t, part);
        hi = part[0].w[0];
        lo = part[1].w[0];
    } else {
        // (exponents 14 .. 254 have a scale and its inverse among the normal numbers; below, T * 2^126 is small enough as it is)
        const uint32_t ex = top >> 23, up = ex == 255u ? 127u : 267u - max(ex, 14u);
        const float scale = __builtin_bit_cast(float, up << 23);
        back = __builtin_bit_cast(float, (254u - up) << 23);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            f16x2 h, l;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const float x = t[2 * q + e] * scale;
                h[e] = (_Float16)fminf(fmaxf(x, -65504.0f), 65504.0f);
                l[e] = (_Float16)(x - (float)h[e]);
            }
            hi[q] = __builtin_bit_cast(uint32_t, h);
            lo[q] = __builtin_bit_cast(uint32_t, l);
        }
    }
}

// Y = Y0 + T B with factors of 16 bits, for N >= 8 and ranks up to 32 * CH, or up to 16 with CH == 0.  A workgroup puts the T of its
// rows into LDS as two operands of 16 bits; a wave keeps its 128 columns of B in registers, eight columns to a lane, as operands that
// sum over 32 ranks, and streams Y0 past them, 16 rows at a time, the next ones under way.  Up to 16 ranks, both operands of T fit
// into one product, over the same B twice.  WHOLE: N is a multiple of 128, so the second copy of the loop and its registers are not
// there (4100 x 4096, rank 16: 15.0 us, 16.7 with it; 67 MB are 13).
template <int TYPE, int CH, bool WHOLE>
__global__ __launch_bounds__(kThreads) void k_adapter_up16(const float* __restrict__ T, int parts, const void* __restrict__ B, Segments seg,
                                                           int tile, int N, int r, const void* Y0, long long ldy0, void* Y,
                                                           long long ldy) {
    constexpr int kSteps = CH == 0 ? 1 : CH, kOctets = CH == 0 ? 2 : 4 * CH;
    constexpr int kPitch = 32 * kOctets + 16;
    __shared__ __align__(16) uint8_t lds[kUpRows * kPitch];
    __shared__ float backs[kUpRows];
    const SegmentTile t = find_tile(seg, tile, blockIdx.z * gridDim.y + blockIdx.y);
    if (t.rows <= 0) return;
    const int a = t.a;
    const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), i = lane & 15, g = lane >> 4;
    const int c0 = (blockIdx.x * kWaves + wave) * kCols, c = c0 + 8 * i, have = N - c;
    if (a < 0) {
        if (Y0 != Y) copy_rows<TYPE>(Y0, ldy0, Y, ldy, t, c, have, g);
        return;
    }
    const bool whole = WHOLE ? c0 < N : c0 + kCols <= N;         // (the same answer for the whole wave)
    Eight<TYPE> row[kSteps][8], y0[4] = {};
    auto fetch_b = [&](auto whole) {
#pragma unroll
        for (int h = 0; h < kSteps; ++h)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int j = CH == 0 ? 8 * (g & 1) + e : 32 * h + 8 * g + e;
                row[h][e] = load_row<TYPE, decltype(whole)::value>(B, ((long long)a * r + min(j, r - 1)) * N, c, N);
            }
    };
    auto fetch = [&](int x, auto whole) {
        if (Y0)
#pragma unroll
            for (int q = 0; q < 4; ++q) y0[q] = load_row<TYPE, decltype(whole)::value>(Y0, (t.row0 + min(x + 4 * g + q, t.rows - 1)) * ldy0, c, N);
    };
    if (whole) {
        fetch_b(std::true_type{});
        fetch(0, std::true_type{});
    } else if (!WHOLE && c0 < N) {
        fetch_b(std::false_type{});
        fetch(0, std::false_type{});
    }
    for (int n = threadIdx.x; n < (t.rows + 15) / 16 * 16 * kOctets; n += kThreads) {
        const int row = n / kOctets, octet = n % kOctets;
        float v[8];
        int at[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) at[q] = min(row, t.rows - 1) * r + min(8 * octet + q, r - 1);
        sum_parts<8>(T + (size_t)t.row0 * r, at, parts, (size_t)seg.M * r, v);
#pragma unroll
        for (int q = 0; q < 8; ++q) v[q] = row < t.rows && 8 * octet + q < r ? v[q] : 0.0f;
        uint32_t top = 0;
        if constexpr (TYPE == APB_F16) {
#pragma unroll
            for (int q = 0; q < 8; ++q) top = max(top, float_bits(v[q]) & 0x7fffffffu);
#pragma unroll
            for (int d = 1; d < kOctets; d <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, d, kWave));
        }
        u32x4 hi, lo;
        float back;
        split<TYPE>(v, top, hi, lo, back);
        *reinterpret_cast<u32x4*>(lds + row * kPitch + 16 * octet) = hi;
        *reinterpret_cast<u32x4*>(lds + row * kPitch + 16 * (kOctets + octet)) = lo;
        if (TYPE == APB_F16 && octet == 0) backs[row] = back;
    }
    __syncthreads();
    if (c0 >= N) return;
    auto stream = [&](auto whole) {
        constexpr bool kWhole = decltype(whole)::value;
        u32x4 b[kSteps][8];
#pragma unroll
        for (int h = 0; h < kSteps; ++h) {
            u32x4 rows[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const bool there = (CH == 0 ? 8 * (g & 1) : 32 * h + 8 * g) + e < r;
                const u32x4 v = settle<TYPE, kWhole>(row[h][e], c, N).w[0];
                rows[e] = there ? v : u32x4{0u, 0u, 0u, 0u};
            }
            transpose8(rows, b[h]);
        }
        for (int x = 0; x < t.rows; x += 16) {
            Eight<TYPE> was[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) was[q] = settle<TYPE, kWhole>(y0[q], c, N);
            if (x + 16 < t.rows) fetch(x + 16, whole);
            f32x4 acc[8];
#pragma unroll
            for (int n = 0; n < 8; ++n) acc[n] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
            const uint8_t* from = lds + (x + i) * kPitch + 16 * g;   // (with CH == 0 the four octets of both operands)
#pragma unroll
            for (int h = 0; h < kSteps; ++h) {
                Eight<TYPE> hi, lo, bn;
                hi.w[0] = *reinterpret_cast<const u32x4*>(from + 64 * h);
                if (CH > 0) lo.w[0] = *reinterpret_cast<const u32x4*>(from + 64 * (kSteps + h));
#pragma unroll
                for (int n = 0; n < 8; ++n) {
                    bn.w[0] = b[h][n];
                    if (CH > 0) acc[n] = multiply8<TYPE>(lo, bn, acc[n]);
                    acc[n] = multiply8<TYPE>(hi, bn, acc[n]);
                }
            }
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int row = x + 4 * g + q;
                const float back = TYPE == APB_F16 ? backs[row] : 1.0f;
                float v[8];
                floats(was[q], v);
#pragma unroll
                for (int n = 0; n < 8; ++n) {
                    const float sum = TYPE == APB_F16 ? acc[n][q] * back : acc[n][q];
                    v[n] += sum;
                }
                if (row < t.rows) store8<TYPE>(Y, (t.row0 + row) * ldy + c, kWhole ? 8 : have, v);
            }
        }
    };
    if (WHOLE || whole) stream(std::true_type{});
    else stream(std::false_type{});
}

// ---- gradients --------------------------------------------------------------------------------------------------------------

// The sum over a wave's lanes.
__device__ __forceinline__ int total(int v) {
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, true);       // (lanes 1, 2, 4, 8 before, of a row of sixteen)
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, true);
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, true);
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, true);
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);      // (the last lane of the row before, to rows 1 and 3)
    v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);      // (of the first half, to the second)
    return __builtin_amdgcn_readlane(v, kWave - 1);
}

// What a wave knows of the segments, a lane each: the last ones that it has looked at, or all if there are no more of them than lanes.
struct Known {
    int its, first, count;
};
// The rows of adapter a, and of all adapters before it.  (A loop of few instructions rather than loads side by side: a workgroup
// comes here once, and fetching instructions takes as long as waiting for the loads.)
struct Span {
    int rows, before;
};
// fresh: `known` is nothing yet.
__device__ __forceinline__ Span span_of(const Segments& seg, int a, Known& known, bool fresh) {
    const int lane = threadIdx.x & (kWave - 1);
    int rows = 0, before = 0;
#pragma unroll 1
    for (int base = 0; base < seg.S; base += kWave) {
        if (fresh || seg.S > kWave) known.its = rows_of(seg, base + lane, known.first, known.count);
        rows += known.its == a ? known.count : 0;
        before += known.its >= 0 && known.its < a ? known.count : 0;
    }
    // (together they are no more than M; of offsets that do not ascend, that much is kept)
    rows = min(total(min(rows, seg.M)), seg.M);
    return Span{rows, min(total(min(before, seg.M)), seg.M - rows)};
}

// The adapter of segment s, if it is the first segment of it; -1 otherwise.
__device__ __forceinline__ int first_segment_of(const Segments& seg, int s) {
    const int lane = threadIdx.x & (kWave - 1);
    int first, count;
    const int a = rows_of(seg, s, first, count);
    for (int base = 0; base < s; base += kWave)
        if (__ballot(base + lane < s && rows_of(seg, base + lane, first, count) == a)) return -1;
    return __builtin_amdgcn_readfirstlane(a);
}

// Slice `number` of adapter a, which has these rows; a < 0: none.
struct Slice {
    int a, number;
    Span span;
};
// What the place k * each stands for (slice_at_place): a slice of the last adapter with no more rows before it, or none.
__device__ __forceinline__ Slice slice_at(const Segments& seg, int k, int each, Known& known) {
    Slice slice{0, 0, {}};
    bool fresh = true;
    int to = seg.L;
#pragma unroll 1
    for (;;) {
        const int middle = (slice.a + to) / 2;                   // (at last slice.a itself)
        const Span span = span_of(seg, middle, known, fresh);
        fresh = false;
        if (span.before > k * each) {
            to = middle;
        } else {
            slice.span = span;
            if (middle == slice.a) break;
            slice.a = middle;
        }
    }
    slice.number = slice_at_place(k, slice.span.before, each);
    if (slice.number <= 0 || slice.number >= (slice.span.rows + each - 1) / each) slice.a = -1;
    return slice;
}

// 32 rows of X as they are loaded: of eight of them NC neighbours to a lane.  Rows 8 g + e, for operands that sum over eight rows; an X of
// float32 goes into products over four rows, row 4 e + g of a lane.
template <int XT, int NC>
struct Rows32 {
    uint32_t w[8][NC * (XT == APB_F32 ? 4 : XT == APB_MX8 ? 1 : 2) / 4];
    uint8_t scale[8];
};
template <int XT>
__device__ __forceinline__ int row_of(int e, int g) { return XT == APB_F32 ? 4 * e + g : 8 * g + e; }

// `rows`: the numbers of the 32 rows.  WHOLE: all columns of the workgroup are there; otherwise the values come one by one, the row's
// last one in the place of those that are not (loads without a branch, which would make the loads before it be waited for).
template <int XT, int NC, bool WHOLE>
__device__ __forceinline__ void load_rows(Rows32<XT, NC>& x, const void* X, long long ldx, const Mx8& x8, const int* rows, int g, int c, int K) {
    constexpr int kWords = sizeof(x.w[0]) / 4;
    typedef uint32_t words __attribute__((ext_vector_type(kWords)));
    typedef words words_any __attribute__((aligned(1)));
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const long long row = rows[row_of<XT>(e, g)];
        if constexpr (XT == APB_MX8) {
            const int at = min(c, x8.blocks * kMx8Block - NC);   // (its rows are padded)
            if constexpr (kWords == 1) x.w[e][0] = *reinterpret_cast<const uint32_t*>(x8.codes + row * x8.blocks * kMx8Block + at);
            else __builtin_memcpy(x.w[e], x8.codes + row * x8.blocks * kMx8Block + at, sizeof(x.w[e]));
            x.scale[e] = x8.scales[row * x8.blocks + at / kMx8Block];
        } else if constexpr (WHOLE) {
            const words v = *reinterpret_cast<const words_any*>(static_cast<const uint8_t*>(X) + (row * ldx + c) * (XT == APB_F32 ? 4 : 2));
#pragma unroll
            for (int q = 0; q < kWords; ++q) x.w[e][q] = v[q];
        } else if constexpr (XT == APB_F32) {
#pragma unroll
            for (int q = 0; q < NC; ++q) x.w[e][q] = static_cast<const uint32_t*>(X)[row * ldx + min(c + q, K - 1)];
        } else {
            const uint16_t* p = static_cast<const uint16_t*>(X) + row * ldx;
#pragma unroll
            for (int q = 0; q < kWords; ++q) x.w[e][q] = p[min(c + 2 * q, K - 1)] | (uint32_t)p[min(c + 2 * q + 1, K - 1)] << 16;
        }
    }
}
// Rows that are not there as zeros (they repeat the last one, and zero times infinity is not zero).
template <int XT, int NC>
__device__ __forceinline__ void clear_rows(Rows32<XT, NC>& x, int rows, int g) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const bool there = row_of<XT>(e, g) < rows;
#pragma unroll
        for (int q = 0; q < (int)sizeof(x.w[0]) / 4; ++q) x.w[e][q] = there ? x.w[e][q] : 0u;
        if (XT == APB_MX8) x.scale[e] = there ? x.scale[e] : (uint8_t)0;
    }
}
// Column n of the lane's as bfloat16 operands of eight rows: 16-bit floats in one or two parts, 8-bit values in one.
template <int XT>
constexpr int kXParts = XT == APB_F16 ? 2 : 1;
template <int XT, int NC>
__device__ __forceinline__ void column(const Rows32<XT, NC>& x, int n, Eight<APB_BF16> (&out)[kXParts<XT>]) {
#pragma unroll
    for (int d = 0; d < 4; ++d) {
        if constexpr (XT == APB_MX8) {
            out[0].w[0][d] = pack2(APB_BF16, decode8(x.w[2 * d][n / 4], n & 3, scale_value(x.scale[2 * d])),
                                   decode8(x.w[2 * d + 1][n / 4], n & 3, scale_value(x.scale[2 * d + 1])));
        } else {
            const uint32_t w = __builtin_amdgcn_perm(x.w[2 * d + 1][n / 2], x.w[2 * d][n / 2], n & 1 ? 0x07060302u : 0x05040100u);
            if constexpr (XT == APB_BF16) {
                out[0].w[0][d] = w;
            } else {
                const f16x2 h = __builtin_bit_cast(f16x2, w);
                const uint32_t hi = pack2(APB_BF16, (float)h[0], (float)h[1]);
                out[0].w[0][d] = hi;
                out[1].w[0][d] = pack2(APB_BF16, (float)h[0] - __builtin_bit_cast(float, hi << 16),
                                       (float)h[1] - __builtin_bit_cast(float, hi & 0xffff0000u));
            }
        }
    }
}

// The sums of adapters without rows, n each, in pieces of kPiece: part `part` of `parts`.
__device__ __forceinline__ void clear_adapters(const Segments& seg, long long n, int part, int parts, float* dA) {
    constexpr int kPiece = 4096;
    const int pieces = (int)((n + kPiece - 1) / kPiece);
    const float zero[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    Known known;
    int last = -1;
    bool empty = false;
    const long long all = (long long)pieces * seg.L, each = (all + parts - 1) / parts;
    for (long long u = part * each; u < std::min(all, (part + 1) * each); ++u) {
        const int a = (int)(u / pieces);
        if (a != last) {
            empty = span_of(seg, a, known, true).rows == 0;
            last = a;
        }
        if (!empty) continue;
        const long long from = (u - (long long)a * pieces) * kPiece, end = std::min<long long>(from + kPiece, n);
        for (long long k = from + 4 * threadIdx.x; k < end; k += 4 * blockDim.x) store4(dA, APB_F32, a * n + k, zero, (int)(end - k));
    }
}

// WHOLE: K is 16 * NC or more; the last workgroup's columns then end with the row's, and those that two workgroups have get the same
// values twice.  (Rows of 8 bits are padded, and their columns stay in blocks.)
//
// A workgroup takes one adapter (by_segment: that of a segment), 16 * JT ranks, 16 * NC columns, and the first `each` of the adapter's rows,
// or those of another of its slices (`more` workgroups, for every adapter as many or by_slice), counted through all of its segments, whose
// numbers it lists in LDS; its waves take 32 of them at a time in turn, by themselves, the next ones under
// way, and join their sums in LDS.  T, its parts added up, comes to registers in the order of the operand and is split there into three
// bfloat16 parts (an X of float32 goes with T as it is through float32 products); X is transposed in registers.  With waves that share a
// tile of rows in LDS and each take columns of their own, every wave waits at barriers for the slowest load, and an adapter's rows have
// to be shared out much sooner: 16384 rows of 8192, rank 32, bfloat16 65 us and now 62 (268 MB are 52); 8196 of 4096, rank 64 43 and 35 (67 MB are 13; T is
// split anew for each of 64 groups of columns); 4100 of 4096, rank 16 16 and 11.7 (34 MB are 7); 512 of 4096, rank 32 13.4 and 7.0.
template <int XT, int JT, int NC, int WAVES, bool WHOLE>
__global__ __launch_bounds__(WAVES * kWave) void k_adapter_gradient(const float* __restrict__ T, int parts, const void* __restrict__ X,
                                                                    long long ldx, Mx8 x8, Segments seg, int K, int r, int rank_tiles,
                                                                    int by_segment, int by_slice, int each, int more, float* __restrict__ dA,
                                                                    float* __restrict__ shared) {
    constexpr int kChunk = 32, kRanks = 16 * JT;
    __shared__ f32x4 sums[WAVES][JT * NC][kWave];
    __shared__ int list[kList + kChunk];
    const int unit = blockIdx.y / rank_tiles, firsts = by_segment ? seg.S : seg.L;
    const int j0 = blockIdx.y % rank_tiles * kRanks;
    if (unit >= firsts + more) {
        const int behind = (firsts + more) * rank_tiles;
        clear_adapters(seg, (long long)r * K, (blockIdx.y - behind) * gridDim.x + blockIdx.x, (gridDim.y - behind) * gridDim.x, dA);
        return;
    }
    Known known;
    Slice slice{unit % firsts, unit / firsts, {}};
    if (unit >= firsts && by_slice) {
        slice = slice_at(seg, unit - firsts + 1, each, known);
        if (slice.a < 0) return;
    } else {
        if (by_segment) slice.a = first_segment_of(seg, slice.a);
        if (slice.a < 0) return;
        slice.span = span_of(seg, slice.a, known, true);
        if (slice.number > 0 && slice.number * each >= slice.span.rows) return;
    }
    const int a = slice.a;
    const Span span = slice.span;
    const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), i = lane & 15, g = lane >> 4;
    const int c0 = XT == APB_MX8 ? blockIdx.x * 16 * NC : WHOLE ? min((int)blockIdx.x * 16 * NC, K - 16 * NC) : 0, c = c0 + NC * i;
    const int lo = slice.number * each, hi = min(lo + each, span.rows);
    f32x4 acc[JT][NC];
#pragma unroll
    for (int j = 0; j < JT; ++j)
#pragma unroll
        for (int n = 0; n < NC; ++n) acc[j][n] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

    // the numbers of the adapter's rows start .. start + rows - 1; behind them the last one again, up to a whole chunk
    auto list_rows = [&](int start, int rows) {
        if (wave == 0) {
            int before = 0;
            for (int base = 0; base < seg.S && before < start + rows; base += kWave) {
                if (seg.S > kWave) known.its = rows_of(seg, base + lane, known.first, known.count);
                for (unsigned long long left = __ballot(known.its == a && known.count > 0); left; left &= left - 1) {
                    const int src = __builtin_amdgcn_readfirstlane(__ffsll((long long)left) - 1);
                    const int from = __builtin_amdgcn_readlane(known.first, src), n = __builtin_amdgcn_readlane(known.count, src);
                    const int skip = max(start - before, 0), end = min(n, start + rows - before);
                    for (int k = skip + lane; k < end; k += kWave) list[before + k - start] = from + k;
                    if (before + n >= start + rows && lane < kChunk && end > skip) list[rows + lane] = from + end - 1;
                    before += n;
                    if (before >= start + rows) break;
                }
            }
        }
        __syncthreads();
    };
    struct Chunk {
        Rows32<XT, NC> x;
        float t[JT][8];
    };
    auto fetch = [&](Chunk& v, int m) {
        load_rows<XT, NC, WHOLE>(v.x, X, ldx, x8, list + m, g, c, K);
        size_t at[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) at[e] = (size_t)list[m + row_of<XT>(e, g)] * r;
#pragma unroll
        for (int j = 0; j < JT; ++j) sum_parts<8>(T + min(j0 + 16 * j + i, r - 1), at, parts, (size_t)seg.M * r, v.t[j]);
    };
    auto multiply = [&](Chunk& v, int rows) {
        if (rows < kChunk) {
            clear_rows<XT, NC>(v.x, rows, g);
#pragma unroll
            for (int j = 0; j < JT; ++j)
#pragma unroll
                for (int e = 0; e < 8; ++e) v.t[j][e] = row_of<XT>(e, g) < rows ? v.t[j][e] : 0.0f;
        }
        if constexpr (XT == APB_F32) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
#pragma unroll
                for (int j = 0; j < JT; ++j)
#pragma unroll
                    for (int n = 0; n < NC; ++n) {
                        const uint32_t bits = v.x.w[e][n];
                        acc[j][n] = __builtin_amdgcn_mfma_f32_16x16x4f32(v.t[j][e], __builtin_bit_cast(float, bits), acc[j][n], 0, 0, 0);
                    }
        } else {
            Eight<APB_BF16> t[JT][3];
#pragma unroll
            for (int j = 0; j < JT; ++j) bf16_parts<3>(v.t[j], t[j]);
#pragma unroll
            for (int n = 0; n < NC; ++n) {
                Eight<APB_BF16> xv[kXParts<XT>];
                column<XT, NC>(v.x, n, xv);
#pragma unroll
                for (int j = 0; j < JT; ++j) {
                    // (the smallest first; the third part of T times the second of X is below 2^-24)
                    if constexpr (kXParts<XT> == 2) {
                        acc[j][n] = multiply8<APB_BF16>(t[j][1], xv[1], acc[j][n]);
                        acc[j][n] = multiply8<APB_BF16>(t[j][0], xv[1], acc[j][n]);
                    }
#pragma unroll
                    for (int p = 2; p >= 0; --p) acc[j][n] = multiply8<APB_BF16>(t[j][p], xv[0], acc[j][n]);
                }
            }
        }
    };
    for (int start = lo; start < hi; start += kList) {
        const int rows = min(hi - start, kList);
        list_rows(start, rows);
        Chunk v;
        int m = wave * kChunk;
        if (m < rows) fetch(v, m);
        for (; m < rows; m += WAVES * kChunk) {
            Chunk now = v;
            if (m + WAVES * kChunk < rows) fetch(v, m + WAVES * kChunk);
            multiply(now, rows - m);
        }
        if (start + kList < hi) __syncthreads();                 // (the list has been read)
    }
#pragma unroll
    for (int j = 0; j < JT; ++j)
#pragma unroll
        for (int n = 0; n < NC; ++n) sums[wave][j * NC + n][lane] = acc[j][n];
    __syncthreads();
    // rank 16 j + 4 g + q of columns NC i ..
    float* out = span.rows > each ? shared + (size_t)(place_of_slices(span.before, each) + slice.number) * r * K : dA + (size_t)a * r * K;
    for (int n = threadIdx.x; n < JT * 256; n += WAVES * kWave) {
        const int q = n & 3, from = n >> 2 & 63, j = n >> 8;
        const int rank = j0 + 16 * j + 4 * (from >> 4) + q, col = c0 + NC * (from & 15);
        if (rank >= r || col >= K) continue;
        float v[NC];
#pragma unroll
        for (int e = 0; e < NC; ++e) {
            v[e] = sums[0][j * NC + e][from][q];
#pragma unroll
            for (int w = 1; w < WAVES; ++w) v[e] += sums[w][j * NC + e][from][q];
        }
#pragma unroll
        for (int e = 0; e < NC; e += 4) {
            const float four[4] = {v[e], v[e + 1], v[e + 2], v[e + 3]};
            store4(out, APB_F32, (long long)rank * K + col + e, four, K - col - e);
        }
    }
}

// The slices of the adapters that have several, added up in order.  by_slice: a workgroup takes a slice behind an adapter's first one, and
// that of its second has the adapter.
__global__ __launch_bounds__(kThreads) void k_adapter_join(const float* __restrict__ shared, Segments seg, int by_slice, int each,
                                                           long long n, float* __restrict__ dA) {
    Known known;
    Slice slice{(int)blockIdx.y, 1, {}};
    if (by_slice) slice = slice_at(seg, blockIdx.y + 1, each, known);
    else slice.span = span_of(seg, slice.a, known, true);
    if (slice.a < 0 || slice.number != 1 || slice.span.rows <= each) return;
    const int a = slice.a;
    const Span span = slice.span;
    const int slices = (span.rows + each - 1) / each;
    const float* from = shared + (size_t)place_of_slices(span.before, each) * n;
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    __shared__ f32x4 sums[kWaves][kWave];
    // four neighbours to a lane; a wave takes every fourth slice, eight at a time
    for (long long k0 = (long long)blockIdx.x * 4 * kWave; k0 < n; k0 += (long long)gridDim.x * 4 * kWave) {
        const long long k = k0 + 4 * lane;
        const int have = (int)std::min<long long>(n - k, 4);
        f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
        for (int z = wave; z < slices; z += 8 * kWaves) {
            u32x4 w[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const float* at = from + min(z + u * kWaves, slices - 1) * n + k;
                if (have >= 4) w[u] = load16_any(at);
                else
#pragma unroll
                    for (int q = 0; q < 4; ++q) w[u][q] = q < have ? float_bits(at[q]) : 0u;
            }
#pragma unroll
            for (int u = 0; u < 8; ++u)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const uint32_t bits = w[u][q];
                    if (z + u * kWaves < slices) v[q] += __builtin_bit_cast(float, bits);
                }
        }
        sums[wave][lane] = v;
        __syncthreads();
        if (wave == 0) {
#pragma unroll
            for (int w = 1; w < kWaves; ++w) v += sums[w][lane];
            const float all[4] = {v[0], v[1], v[2], v[3]};
            store4(dA, APB_F32, a * n + k, all, have);
        }
        __syncthreads();
    }
}

bool bad_adapter(int S, int L, int M, int K, int r, const int32_t* offsets, const int32_t* adapter) {
    return S <= 0 || S > APB_ADAPTER_MAX_S || L <= 0 || L > APB_ADAPTER_MAX_L || M <= 0 || M > (1 << 24) || K <= 0 || K > kMxMaxK || r <= 0 ||
           r > APB_ADAPTER_MAX_R || (!offsets && S != 1) || (!adapter && S != L);
}

template <int TYPE, int RT, int JT>
void down_tiles(const void* X, long long ldx, const void* A, const Segments& seg, const float* scale, int K, int r, int tile, int parts,
                float* T, hipStream_t s) {
    constexpr int kLine = TYPE == APB_F32 ? 32 : 64, kW = down_waves(RT, JT);
    const int lines = (K + kLine - 1) / kLine, each = (lines + parts - 1) / parts;
    const dim3 grid((unsigned)max_row_tiles(seg.M, seg.S, seg.offsets != nullptr, tile), (unsigned)((r + 16 * JT - 1) / (16 * JT)), (unsigned)parts);
    hipLaunchKernelGGL((k_adapter_down<TYPE, RT, JT, kW>), grid, dim3(kW * kWave), 0, s, X, ldx, A, seg, scale, K, r, each, tile, T);
}
template <int TYPE>
void down(const void* X, long long ldx, const void* A, const Segments& seg, const float* scale, int K, int r, float* T, hipStream_t s) {
    const DownPlan p = down_plan(seg.S, seg.M, K, r);
    auto with = [&](auto rt, auto jt) {
        down_tiles<TYPE, decltype(rt)::value, decltype(jt)::value>(X, ldx, A, seg, scale, K, r, p.tile, p.parts, T, s);
    };
    auto with_rows = [&](auto rt) {
        if (p.jt == 1) with(rt, std::integral_constant<int, 1>{});
        else if (p.jt == 2) with(rt, std::integral_constant<int, 2>{});
        else with(rt, std::integral_constant<int, 4>{});
    };
    if (p.rt == 1) with_rows(std::integral_constant<int, 1>{});
    else if (p.rt == 2) with_rows(std::integral_constant<int, 2>{});
    else with_rows(std::integral_constant<int, 4>{});
}

template <int TYPE, int RT>
void up_tiles(const float* T, int parts, const void* B, const Segments& seg, int N, int r, const void* Y0, long long ldy0, void* Y,
              long long ldy, hipStream_t s) {
    const dim3 grid((unsigned)max_row_tiles(seg.M, seg.S, seg.offsets != nullptr, 16 * RT), (unsigned)((N + kCols * kWaves - 1) / (kCols * kWaves)));
    hipLaunchKernelGGL((k_adapter_up<TYPE, RT>), grid, dim3(kThreads), 0, s, T, parts, B, seg, N, r, Y0, ldy0, Y, ldy);
}
template <int TYPE, int CH>
void up16_tiles(const float* T, int parts, const void* B, const Segments& seg, int N, int r, const void* Y0, long long ldy0, void* Y,
                long long ldy, hipStream_t s) {
    const int tile = up_rows(seg.S, seg.M, N);
    // neighbouring workgroups take neighbouring columns
    const unsigned tiles = (unsigned)max_row_tiles(seg.M, seg.S, seg.offsets != nullptr, tile), most = 32768;
    const dim3 grid((unsigned)((N + kCols * kWaves - 1) / (kCols * kWaves)), std::min(tiles, most), (tiles + most - 1) / most);
    auto launch = [&](auto whole) {
        hipLaunchKernelGGL((k_adapter_up16<TYPE, CH, decltype(whole)::value>), grid, dim3(kThreads), 0, s, T, parts, B, seg, tile, N, r, Y0, ldy0,
                           Y, ldy);
    };
    if (N % kCols == 0) launch(std::true_type{});
    else launch(std::false_type{});
}
template <int TYPE>
void up(const float* T, int parts, const void* B, const Segments& seg, int N, int r, const void* Y0, long long ldy0, void* Y, long long ldy,
        hipStream_t s) {
    if constexpr (TYPE != APB_F32) if (N >= 8) {
        if (r <= 16) return up16_tiles<TYPE, 0>(T, parts, B, seg, N, r, Y0, ldy0, Y, ldy, s);
        if (r <= 32) return up16_tiles<TYPE, 1>(T, parts, B, seg, N, r, Y0, ldy0, Y, ldy, s);
        if (r <= 64) return up16_tiles<TYPE, 2>(T, parts, B, seg, N, r, Y0, ldy0, Y, ldy, s);
        if (r <= 128) return up16_tiles<TYPE, 4>(T, parts, B, seg, N, r, Y0, ldy0, Y, ldy, s);
    }
    if (up_rows(seg.S, seg.M, N) == kUpRows) up_tiles<TYPE, 4>(T, parts, B, seg, N, r, Y0, ldy0, Y, ldy, s);
    else up_tiles<TYPE, 1>(T, parts, B, seg, N, r, Y0, ldy0, Y, ldy, s);
}

template <int XT, int JT, int NC, int WAVES>
void gradient_form(const float* T, int parts, const void* X, long long ldx, const Mx8& x8, const Segments& seg, int K, int r, int each,
                   float* dA, float* shared, hipStream_t s) {
    const int rank_tiles = (r + 16 * JT - 1) / (16 * JT);
    const int by_segment = gradient_by_segment(seg.S, seg.L, K, r);
    const unsigned columns = (unsigned)((K + 16 * NC - 1) / (16 * NC));
    const int firsts = by_segment ? seg.S : seg.L;
    const bool by_slice = gradient_by_slice(firsts, seg.M, each, (long long)columns * rank_tiles);
    const int more = by_slice ? more_slices(seg.M, each) : firsts * ((seg.M - 1) / each);
    const dim3 grid(columns, (unsigned)((firsts + more) * rank_tiles + (by_segment ? (1024 + columns - 1) / columns : 0)));
    auto launch = [&](auto whole) {
        hipLaunchKernelGGL((k_adapter_gradient<XT, JT, NC, WAVES, decltype(whole)::value>), grid, dim3(WAVES * kWave), 0, s, T, parts, X, ldx, x8,
                           seg, K, r, rank_tiles, by_segment, by_slice, each, more, dA, shared);
    };
    if constexpr (XT == APB_MX8 || NC == 8) launch(std::true_type{});
    else if (K >= 16 * NC) launch(std::true_type{});
    else launch(std::false_type{});
}
template <int XT>
void gradient(const float* T, int parts, const void* X, long long ldx, const Mx8& x8, const Segments& seg, int K, int r, int each,
              float* dA, float* shared, hipStream_t s) {
    const GradientForm form = gradient_form_of(XT, seg.S, seg.L, seg.M, K, r);
    auto with = [&](auto ranks) {
        constexpr int kJt = decltype(ranks)::value;
        if (form.waves == 1) return gradient_form<XT, kJt, 4, 1>(T, parts, X, ldx, x8, seg, K, r, each, dA, shared, s);
        if (form.waves == 4) return gradient_form<XT, kJt, 4, 4>(T, parts, X, ldx, x8, seg, K, r, each, dA, shared, s);
        if constexpr (XT != APB_F32 && kJt <= 2)
            if (form.nc == 8) return gradient_form<XT, kJt, 8, 8>(T, parts, X, ldx, x8, seg, K, r, each, dA, shared, s);
        if constexpr (XT != APB_F32 || kJt <= 2) gradient_form<XT, kJt, 4, 8>(T, parts, X, ldx, x8, seg, K, r, each, dA, shared, s);
    };
    if (form.jt == 1) with(std::integral_constant<int, 1>{});
    else if (form.jt == 2) with(std::integral_constant<int, 2>{});
    else with(std::integral_constant<int, 4>{});
}

}  // namespace
}  // namespace apb

using namespace apb;

extern "C" {

int apb_adapter_parts(int S, int M, int K, int r) {
    static const int32_t some = 0;
    return bad_adapter(S, 1, M, K, r, &some, &some) ? 0 : down_plan(S, M, K, r).parts;
}

int apb_adapter_down(const void* X, int type, long long ldx, const void* A, const int32_t* offsets, const int32_t* adapter,
                     const float* scale, int S, int L, int M, int K, int r, float* T, void* stream) {
    if (!X || !A || !T) return APB_ERR_NULL;
    if (bad_type(type)) return APB_ERR_TYPE;
    if (bad_adapter(S, L, M, K, r, offsets, adapter) || ldx < K) return APB_ERR_SHAPE;
    if (!aligned(X, type_size(type)) || !aligned(A, type_size(type)) || !aligned(T, 4) || !aligned(offsets, 4) || !aligned(adapter, 4) ||
        !aligned(scale, 4))
        return APB_ERR_ALIGN;
    const Segments seg{offsets, adapter, S, L, M};
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    if (type == APB_F32) down<APB_F32>(X, ldx, A, seg, scale, K, r, T, s);
    else if (type == APB_BF16) down<APB_BF16>(X, ldx, A, seg, scale, K, r, T, s);
    else down<APB_F16>(X, ldx, A, seg, scale, K, r, T, s);
    APB_HIP(hipGetLastError());
    return APB_OK;
}

int apb_adapter_up(const float* T, int parts, const void* B, int type, const int32_t* offsets, const int32_t* adapter, int S, int L,
                   int M, int N, int r, const void* Y0, long long ldy0, void* Y, long long ldy, void* stream) {
    if (!T || !B || !Y) return APB_ERR_NULL;
    if (bad_type(type)) return APB_ERR_TYPE;
    if (bad_adapter(S, L, M, N, r, offsets, adapter) || parts <= 0 || parts > kMaxParts || ldy < N || (Y0 && ldy0 < N) || (Y0 == Y && ldy0 != ldy))
        return APB_ERR_SHAPE;
    if (!aligned(T, 4) || !aligned(B, type_size(type)) || !aligned(Y, type_size(type)) || !aligned(Y0, type_size(type)) ||
        !aligned(offsets, 4) || !aligned(adapter, 4))
        return APB_ERR_ALIGN;
    const Segments seg{offsets, adapter, S, L, M};
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    if (type == APB_F32) up<APB_F32>(T, parts, B, seg, N, r, Y0, ldy0, Y, ldy, s);
    else if (type == APB_BF16) up<APB_BF16>(T, parts, B, seg, N, r, Y0, ldy0, Y, ldy, s);
    else up<APB_F16>(T, parts, B, seg, N, r, Y0, ldy0, Y, ldy, s);
    APB_HIP(hipGetLastError());
    return APB_OK;
}

size_t apb_adapter_gradient_workspace_bytes(int S, int L, int M, int K, int r) {
    static const int32_t some = 0;
    if (bad_adapter(S, L, M, K, r, &some, &some)) return 0;
    const int each = gradient_rows(S, L, M, K, r);
    return M > each ? (size_t)places_of_slices(M, each) * r * K * sizeof(float) : 0;
}

int apb_adapter_gradient(const float* T, int parts, const void* X, int x_type, long long ldx, const int32_t* offsets,
                         const int32_t* adapter, int S, int L, int M, int K, int r, float* dA, void* workspace, size_t workspace_bytes,
                         void* stream) {
    if (!T || !X || !dA) return APB_ERR_NULL;
    if (bad_type(x_type) && x_type != APB_MX8) return APB_ERR_TYPE;
    if (bad_adapter(S, L, M, K, r, offsets, adapter) || parts <= 0 || parts > kMaxParts ||
        (x_type == APB_MX8 ? bad_shape_mx8(M, K) : ldx < K))
        return APB_ERR_SHAPE;
    if (!aligned(T, 4) || !aligned(X, x_type == APB_MX8 ? 16 : type_size(x_type)) || !aligned(dA, 4) || !aligned(workspace, 4) ||
        !aligned(offsets, 4) || !aligned(adapter, 4))
        return APB_ERR_ALIGN;
    const Segments seg{offsets, adapter, S, L, M};
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    const size_t need = apb_adapter_gradient_workspace_bytes(S, L, M, K, r);
    const bool join = need != 0 && workspace != nullptr && workspace_bytes >= need;
    const int each = join ? gradient_rows(S, L, M, K, r) : M;
    float* shared = static_cast<float*>(workspace);
    const Mx8 x8 = mx8_view(X, M, K);
    if (x_type == APB_F32) gradient<APB_F32>(T, parts, X, ldx, x8, seg, K, r, each, dA, shared, s);
    else if (x_type == APB_BF16) gradient<APB_BF16>(T, parts, X, ldx, x8, seg, K, r, each, dA, shared, s);
    else if (x_type == APB_F16) gradient<APB_F16>(T, parts, X, ldx, x8, seg, K, r, each, dA, shared, s);
    else gradient<APB_MX8>(T, parts, X, ldx, x8, seg, K, r, each, dA, shared, s);
    APB_HIP(hipGetLastError());
    if (join) {
        const long long n = (long long)r * K;
        const int columns = (int)std::min<long long>((n + 4 * kWave - 1) / (4 * kWave), 4096);
        const bool by_slice = join_by_slice(L, M, each, columns);
        const dim3 grid((unsigned)columns, (unsigned)(by_slice ? more_slices(M, each) : L));
        hipLaunchKernelGGL(k_adapter_join, grid, dim3(kThreads), 0, s, shared, seg, by_slice, each, n, dA);
        APB_HIP(hipGetLastError());
    }
    return APB_OK;
}

}  // extern "C"
