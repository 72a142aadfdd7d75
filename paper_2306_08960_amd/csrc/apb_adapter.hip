// Low-rank adapters of many requests: T = scale X A^T (down), Y = Y0 + T B (up), dA = sum T^T X (gradient), every row with the factors of
// its segment's adapter.  A and B have their long side contiguous, so that each of them and each of the gradients' operands is read
// in whole lines and all directions are these three kernels.
#include "apb_mx8.h"

namespace apb {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;
constexpr int kMaxParts = 32;
constexpr int kMaxSlices = 32;
constexpr int kCols = 128;                    // of a wave, in up and gradient: eight to a lane
constexpr int kStage = 64;                    // ranks of T that are in LDS at a time

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

struct Segments {
    const int32_t *offsets, *adapter;
    int S, L, M;
};

__device__ __forceinline__ int adapter_of(const Segments& g, int s) {
    if (s >= g.S) return -1;
    const int a = g.adapter ? g.adapter[s] : s;
    return a < g.L ? a : -1;
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

// A workgroup takes 16 * RT rows of a segment, 16 * JT ranks and one part of K; its waves take chunks of 128 bytes of the rows in turn,
// straight from memory in the order of the operands (a row's four lanes read a whole line), and join their sums in LDS.
template <int TYPE, int RT, int JT>
__global__ __launch_bounds__(kThreads) void k_adapter_down(const void* __restrict__ X, long long ldx, const void* __restrict__ A, Segments seg,
                                                           const float* __restrict__ scale, int K, int r, int chunks_each,
                                                           float* __restrict__ T) {
    constexpr int kChunk = TYPE == APB_F32 ? 32 : 64, kEach = kChunk / 4;        // values of a row: in a chunk, of a lane
    __shared__ f32x4 sums[kWaves][RT * JT][kWave];
    const RowTile t = find_row_tile(seg.offsets, seg.S, seg.M, 16 * RT, blockIdx.x);
    if (t.rows <= 0) return;
    const int j0 = blockIdx.z * 16 * JT, ranks = min(16 * JT, r - j0);
    float* out = T + ((size_t)blockIdx.y * seg.M + t.row0) * r + j0;
    const int a = adapter_of(seg, t.e);
    if (a < 0) {
        for (int i = threadIdx.x; i < t.rows * ranks; i += kThreads) out[(size_t)(i / ranks) * r + i % ranks] = 0.0f;
        return;
    }
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave, i = lane & 15, g = lane >> 4;
    long long x_at[RT], a_at[JT];
#pragma unroll
    for (int x = 0; x < RT; ++x) x_at[x] = (t.row0 + min(16 * x + i, t.rows - 1)) * ldx;
#pragma unroll
    for (int j = 0; j < JT; ++j) a_at[j] = ((long long)a * r + min(j0 + 16 * j + i, r - 1)) * K;
    f32x4 acc[RT][JT];
#pragma unroll
    for (int x = 0; x < RT; ++x)
#pragma unroll
        for (int j = 0; j < JT; ++j) acc[x][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    const int last = min((int)(blockIdx.y + 1) * chunks_each, (K + kChunk - 1) / kChunk);
    for (int c = blockIdx.y * chunks_each + wave; c < last; c += kWaves) {
#pragma unroll
        for (int h = 0; h < kEach / 8; ++h) {
            const int k = c * kChunk + kEach * g + 8 * h;
            Eight<TYPE> xv[RT], av[JT];
#pragma unroll
            for (int x = 0; x < RT; ++x) xv[x] = load_some<TYPE>(X, x_at[x] + k, K - k);
#pragma unroll
            for (int j = 0; j < JT; ++j) av[j] = load_some<TYPE>(A, a_at[j] + k, K - k);
#pragma unroll
            for (int x = 0; x < RT; ++x)
#pragma unroll
                for (int j = 0; j < JT; ++j) acc[x][j] = multiply8<TYPE>(av[j], xv[x], acc[x][j]);
        }
    }
#pragma unroll
    for (int x = 0; x < RT; ++x)
#pragma unroll
        for (int j = 0; j < JT; ++j) sums[wave][x * JT + j][lane] = acc[x][j];
    __syncthreads();
    const float by = scale ? scale[a] : 1.0f;
    for (int n = wave; n < RT * JT; n += kWaves) {
        f32x4 v = sums[0][n][lane];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) v += sums[w][n][lane];
        const int row = 16 * (n / JT) + i, j = 16 * (n % JT) + 4 * g;
        if (row < t.rows)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                if (j + q < ranks) out[(size_t)row * r + j + q] = v[q] * by;
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
    const RowTile t = find_row_tile(seg.offsets, seg.S, seg.M, 16 * RT, blockIdx.x);
    if (t.rows <= 0) return;
    const int a = adapter_of(seg, t.e);
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave, i = lane & 15, g = lane >> 4;
    const int c = (blockIdx.y * kWaves + wave) * kCols + 8 * i, have = N - c;
    if (a < 0) {
        if (Y0 == Y) return;
        for (int row = g; row < t.rows; row += 4) {
            float v[8] = {};
            if (Y0) floats(load_some<TYPE>(Y0, (t.row0 + row) * ldy0 + c, have), v);
            store8<TYPE>(Y, (t.row0 + row) * ldy + c, have, v);
        }
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
            float v = 0.0f;
            if (row < t.rows && j < ranks)
                for (int p = 0; p < parts; ++p) v += T[((size_t)p * seg.M + t.row0 + row) * r + j0 + j];
            lds[row * kPitch + j] = v;
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

// Eight neighbours of a row of X as float32; XT: an apb_type or APB_MX8.
template <int XT>
__device__ __forceinline__ void row_values(const void* X, long long ldx, const Mx8& x8, long long row, int c, int have, float (&v)[8]) {
    if constexpr (XT == APB_MX8) {
        if (have <= 0) {
#pragma unroll
            for (int q = 0; q < 8; ++q) v[q] = 0.0f;
            return;
        }
        const u32x2 w = *reinterpret_cast<const u32x2*>(x8.codes + row * x8.blocks * kMx8Block + c);
        const float scale = scale_value(x8.scales[row * x8.blocks + c / kMx8Block]);
#pragma unroll
        for (int q = 0; q < 8; ++q) v[q] = decode8(w[q / 4], q & 3, scale);
    } else {
        floats(load_some<XT>(X, row * ldx + c, have), v);
    }
}

// Segment s's rows if its adapter is a: first row and number.
__device__ __forceinline__ void rows_of(const Segments& seg, int s, int a, int& first, int& count) {
    first = count = 0;
    if (s >= seg.S || adapter_of(seg, s) != a) return;
    first = seg.offsets ? min(max(seg.offsets[s], 0), seg.M) : 0;
    count = (seg.offsets ? max(first, min(seg.offsets[s + 1], seg.M)) : seg.M) - first;
}

// A workgroup takes one adapter, 16 * JT ranks, kCols columns a wave, and a slice of the adapter's rows, counted through all of its
// segments.
template <int XT, int JT>
__global__ __launch_bounds__(kThreads) void k_adapter_gradient(const float* __restrict__ T, int parts, const void* __restrict__ X,
                                                               long long ldx, Mx8 x8, Segments seg, int K, int r, int rank_tiles,
                                                               float* __restrict__ out) {
    const int a = blockIdx.y / rank_tiles, j0 = blockIdx.y % rank_tiles * 16 * JT;
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave, i = lane & 15, g = lane >> 4;
    const int c = (blockIdx.x * kWaves + wave) * kCols + 8 * i;
    int total = 0;
    for (int base = 0; base < seg.S; base += kWave) {
        int first, count;
        rows_of(seg, base + lane, a, first, count);
#pragma unroll
        for (int d = 1; d < kWave; d <<= 1) count += __shfl_xor(count, d, kWave);
        total += count;
    }
    const int each = ((total + (int)gridDim.z - 1) / (int)gridDim.z + 3) / 4 * 4;
    const int lo = blockIdx.z * each, hi = min(lo + each, total);
    f32x4 acc[JT][8];
#pragma unroll
    for (int j = 0; j < JT; ++j)
#pragma unroll
        for (int q = 0; q < 8; ++q) acc[j][q] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    int before = 0;
    for (int base = 0; base < seg.S && before < hi; base += kWave) {
        int first, count;
        rows_of(seg, base + lane, a, first, count);
        for (unsigned long long left = __ballot(count > 0); left; left &= left - 1) {
            const int src = __builtin_amdgcn_readfirstlane(__ffsll((long long)left) - 1);
            const int from = __builtin_amdgcn_readlane(first, src), rows = __builtin_amdgcn_readlane(count, src);
            const int end = from + min(rows, hi - before);
            for (int m = from + max(lo - before, 0); m < end; m += 4) {
                const int row = m + g;
                float v[8], tv[JT];
                row_values<XT>(X, ldx, x8, row, c, row < end ? K - c : 0, v);
#pragma unroll
                for (int j = 0; j < JT; ++j) {
                    tv[j] = 0.0f;
                    if (row < end && j0 + 16 * j + i < r)
                        for (int p = 0; p < parts; ++p) tv[j] += T[((size_t)p * seg.M + row) * r + j0 + 16 * j + i];
                }
#pragma unroll
                for (int j = 0; j < JT; ++j)
#pragma unroll
                    for (int q = 0; q < 8; ++q) acc[j][q] = __builtin_amdgcn_mfma_f32_16x16x4f32(tv[j], v[q], acc[j][q], 0, 0, 0);
            }
            before += rows;
        }
    }
    out += ((size_t)blockIdx.z * seg.L + a) * r * K;
#pragma unroll
    for (int j = 0; j < JT; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int rank = j0 + 16 * j + 4 * g + q;
            if (rank >= r) continue;
            float v[8];
#pragma unroll
            for (int n = 0; n < 8; ++n) v[n] = acc[j][n][q];
            store8<APB_F32>(out, (long long)rank * K + c, K - c, v);
        }
}

// The slices' sums added up in order.
__global__ __launch_bounds__(kThreads) void k_adapter_join(const float* __restrict__ parts, int slices, long long n, float* __restrict__ out) {
    for (long long i = (long long)blockIdx.x * kThreads + threadIdx.x; i < n; i += (long long)gridDim.x * kThreads) {
        float v = parts[i];
        for (int s = 1; s < slices; ++s) v += parts[s * n + i];
        out[i] = v;
    }
}

bool bad_adapter(int S, int L, int M, int K, int r, const int32_t* offsets, const int32_t* adapter) {
    return S <= 0 || S > APB_ADAPTER_MAX_S || L <= 0 || L > APB_ADAPTER_MAX_L || M <= 0 || M > (1 << 24) || K <= 0 || K > kMxMaxK || r <= 0 ||
           r > APB_ADAPTER_MAX_R || (!offsets && S != 1) || (!adapter && S != L);
}

// Groups of 16 rows that a workgroup takes: four where segments have them on average.
int row_groups(int S, int M) { return (M + S - 1) / S > 32 ? 4 : 1; }
int rank_groups(int r) { return r <= 16 ? 1 : r <= 32 ? 2 : 4; }

int down_parts(int S, int M, int K, int r) {
    const int rows = 16 * row_groups(S, M), ranks = 16 * rank_groups(r);
    const long long tiles = std::max<long long>((M + rows - 1) / rows, std::min(S, M)) * ((r + ranks - 1) / ranks);
    // two chunks to a wave at least
    return (int)std::max<long long>(1, std::min<long long>(std::min<long long>(512 / tiles, K / 512), kMaxParts));
}

int gradient_slices(int L, int M, int K, int r) {
    const int ranks = 16 * rank_groups(r);
    const long long tiles = (long long)((K + kCols * kWaves - 1) / (kCols * kWaves)) * L * ((r + ranks - 1) / ranks);
    return (int)std::max<long long>(1, std::min<long long>(std::min<long long>(512 / tiles, M / L / 32), kMaxSlices));
}

template <int TYPE, int RT, int JT>
void down_tiles(const void* X, long long ldx, const void* A, const Segments& seg, const float* scale, int K, int r, int parts, float* T,
                hipStream_t s) {
    constexpr int kChunk = TYPE == APB_F32 ? 32 : 64;
    const int chunks = (K + kChunk - 1) / kChunk, each = (chunks + parts - 1) / parts;
    const dim3 grid((unsigned)max_row_tiles(seg.M, seg.S, seg.offsets != nullptr, 16 * RT), (unsigned)parts, (unsigned)((r + 16 * JT - 1) / (16 * JT)));
    hipLaunchKernelGGL((k_adapter_down<TYPE, RT, JT>), grid, dim3(kThreads), 0, s, X, ldx, A, seg, scale, K, r, each, T);
}
template <int TYPE, int RT>
void down_ranks(const void* X, long long ldx, const void* A, const Segments& seg, const float* scale, int K, int r, int parts, float* T,
                hipStream_t s) {
    const int j = rank_groups(r);
    if (j == 1) down_tiles<TYPE, RT, 1>(X, ldx, A, seg, scale, K, r, parts, T, s);
    else if (j == 2) down_tiles<TYPE, RT, 2>(X, ldx, A, seg, scale, K, r, parts, T, s);
    else down_tiles<TYPE, RT, 4>(X, ldx, A, seg, scale, K, r, parts, T, s);
}
template <int TYPE>
void down(const void* X, long long ldx, const void* A, const Segments& seg, const float* scale, int K, int r, float* T, hipStream_t s) {
    const int parts = down_parts(seg.S, seg.M, K, r);
    if (row_groups(seg.S, seg.M) == 4) down_ranks<TYPE, 4>(X, ldx, A, seg, scale, K, r, parts, T, s);
    else down_ranks<TYPE, 1>(X, ldx, A, seg, scale, K, r, parts, T, s);
}

template <int TYPE, int RT>
void up_tiles(const float* T, int parts, const void* B, const Segments& seg, int N, int r, const void* Y0, long long ldy0, void* Y,
              long long ldy, hipStream_t s) {
    const dim3 grid((unsigned)max_row_tiles(seg.M, seg.S, seg.offsets != nullptr, 16 * RT), (unsigned)((N + kCols * kWaves - 1) / (kCols * kWaves)));
    hipLaunchKernelGGL((k_adapter_up<TYPE, RT>), grid, dim3(kThreads), 0, s, T, parts, B, seg, N, r, Y0, ldy0, Y, ldy);
}
template <int TYPE>
void up(const float* T, int parts, const void* B, const Segments& seg, int N, int r, const void* Y0, long long ldy0, void* Y, long long ldy,
        hipStream_t s) {
    if (row_groups(seg.S, seg.M) == 4) up_tiles<TYPE, 4>(T, parts, B, seg, N, r, Y0, ldy0, Y, ldy, s);
    else up_tiles<TYPE, 1>(T, parts, B, seg, N, r, Y0, ldy0, Y, ldy, s);
}

template <int XT, int JT>
void gradient_tiles(const float* T, int parts, const void* X, long long ldx, const Mx8& x8, const Segments& seg, int K, int r, int slices,
                    float* out, hipStream_t s) {
    const int rank_tiles = (r + 16 * JT - 1) / (16 * JT);
    const dim3 grid((unsigned)((K + kCols * kWaves - 1) / (kCols * kWaves)), (unsigned)(seg.L * rank_tiles), (unsigned)slices);
    hipLaunchKernelGGL((k_adapter_gradient<XT, JT>), grid, dim3(kThreads), 0, s, T, parts, X, ldx, x8, seg, K, r, rank_tiles, out);
}
template <int XT>
void gradient(const float* T, int parts, const void* X, long long ldx, const Mx8& x8, const Segments& seg, int K, int r, int slices,
              float* out, hipStream_t s) {
    const int j = rank_groups(r);
    if (j == 1) gradient_tiles<XT, 1>(T, parts, X, ldx, x8, seg, K, r, slices, out, s);
    else if (j == 2) gradient_tiles<XT, 2>(T, parts, X, ldx, x8, seg, K, r, slices, out, s);
    else gradient_tiles<XT, 4>(T, parts, X, ldx, x8, seg, K, r, slices, out, s);
}

}  // namespace
}  // namespace apb

using namespace apb;

extern "C" {

int apb_adapter_parts(int S, int M, int K, int r) {
    static const int32_t some = 0;
    return bad_adapter(S, 1, M, K, r, &some, &some) ? 0 : down_parts(S, M, K, r);
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

size_t apb_adapter_gradient_workspace_bytes(int L, int M, int K, int r) {
    static const int32_t some = 0;
    if (bad_adapter(1, L, M, K, r, &some, &some)) return 0;
    const int slices = gradient_slices(L, M, K, r);
    return slices > 1 ? (size_t)slices * L * r * K * sizeof(float) : 0;
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
    const size_t need = apb_adapter_gradient_workspace_bytes(L, M, K, r);
    const bool shared = need != 0 && workspace != nullptr && workspace_bytes >= need;
    const int slices = shared ? gradient_slices(L, M, K, r) : 1;
    float* out = shared ? static_cast<float*>(workspace) : dA;
    const Mx8 x8 = mx8_view(X, M, K);
    if (x_type == APB_F32) gradient<APB_F32>(T, parts, X, ldx, x8, seg, K, r, slices, out, s);
    else if (x_type == APB_BF16) gradient<APB_BF16>(T, parts, X, ldx, x8, seg, K, r, slices, out, s);
    else if (x_type == APB_F16) gradient<APB_F16>(T, parts, X, ldx, x8, seg, K, r, slices, out, s);
    else gradient<APB_MX8>(T, parts, X, ldx, x8, seg, K, r, slices, out, s);
    APB_HIP(hipGetLastError());
    if (shared) {
        const long long n = (long long)L * r * K;
        const unsigned blocks = (unsigned)std::min<long long>((n + kThreads - 1) / kThreads, 4096);
        hipLaunchKernelGGL(k_adapter_join, dim3(blocks), dim3(kThreads), 0, s, static_cast<const float*>(workspace), slices, n, dA);
        APB_HIP(hipGetLastError());
    }
    return APB_OK;
}

}  // extern "C"
