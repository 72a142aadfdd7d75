// Products of two 4-bit matrices, Y = A^ B^T, plain or grouped by expert.
#include "apb_mx4.h"

namespace apb {
namespace {

constexpr int kThreads = 256;

template <int S>
__device__ __forceinline__ f32x16 mfma(const i32x8& a, const i32x8& b, const f32x16& c, int sa, int sb) {
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, c, 4, 4, S, sa, S, sb);
}

__device__ __forceinline__ i32x8 operand(const uint8_t* p) {
    const u32x4 w = *reinterpret_cast<const u32x4*>(p);
    return i32x8{(int)w[0], (int)w[1], (int)w[2], (int)w[3], 0, 0, 0, 0};
}

// A wave computes 32 x 32 outputs.  Lane (r, h) holds 32 values of row r: of a segment of 256, step s multiplies block s
// (h = 0) and block 4 + s (h = 1), so that a lane's four scales are one word.  Rows of B go in the first operand: a lane then
// holds four neighbours of a row of Y.
__global__ __launch_bounds__(kThreads) void k_mx4_gemm(Mx A, Mx B, const int32_t* __restrict__ offsets, int E, int N, int type,
                                                       void* __restrict__ Y, long long ldy, bool vec) {
    const RowTile t = find_row_tile(offsets, E, A.rows, 32, blockIdx.x);
    const int n0 = (blockIdx.y * (kThreads / kWave) + threadIdx.x / kWave) * 32;
    if (t.rows <= 0 || n0 >= N) return;
    const int lane = threadIdx.x & (kWave - 1), r = lane & 31, h = lane >> 5;
    f32x16 c;
#pragma unroll
    for (int i = 0; i < 16; ++i) c[i] = 0.0f;
    if (t.e < E) {
        const int m = t.row0 + min(r, t.rows - 1), n = t.e * N + min(n0 + r, N - 1);
        const uint8_t* a = A.codes + (size_t)m * A.segs * kMxSegBytes + 64 * h;
        const uint8_t* b = B.codes + (size_t)n * B.segs * kMxSegBytes + 64 * h;
        const uint8_t* sa = A.scales + (size_t)m * 8 + 4 * h;
        const uint8_t* sb = B.scales + (size_t)n * 8 + 4 * h;
        for (int seg = 0; seg < A.segs; ++seg) {
            const int wa = *reinterpret_cast<const int*>(sa + (size_t)seg * A.rows * 8);
            const int wb = *reinterpret_cast<const int*>(sb + (size_t)seg * B.rows * 8);
            c = mfma<0>(operand(b), operand(a), c, wb, wa);
            c = mfma<1>(operand(b + 16), operand(a + 16), c, wb, wa);
            c = mfma<2>(operand(b + 32), operand(a + 32), c, wb, wa);
            c = mfma<3>(operand(b + 48), operand(a + 48), c, wb, wa);
            a += kMxSegBytes;
            b += kMxSegBytes;
        }
    }
    if (r >= t.rows) return;
    const long long row = (long long)(t.row0 + r) * ldy;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        const int n = n0 + 8 * g + 4 * h;
        const float v[4] = {c[4 * g], c[4 * g + 1], c[4 * g + 2], c[4 * g + 3]};
        store4(Y, type, row + n, v, N - n, vec);
    }
}

}  // namespace

int launch_mx4_gemm(const Mx& A, const Mx& B, const int32_t* offsets, int E, int M, int N, int type, void* Y, long long ldy,
                    hipStream_t s) {
    const dim3 grid((unsigned)max_row_tiles(M, E, offsets != nullptr, 32), (unsigned)((N + 127) / 128));
    hipLaunchKernelGGL(k_mx4_gemm, grid, dim3(kThreads), 0, s, A, B, offsets, E, N, type, Y, ldy, rows_aligned16(Y, ldy, type));
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
    return launch_mx4_gemm(mx_view(A, M, K), mx_view(B, E * N, K), offsets, E, M, N, type, Y, ldy,
                           reinterpret_cast<hipStream_t>(stream));
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
    const int rc = launch_mx4_quantize(X, x_type, ldx, 1, rows_in, rows_from, M, K, scratch, s);
    if (rc != APB_OK) return rc;
    return launch_mx4_gemm(mx_view(scratch, M, K), mx_view(W, E * N, K), offsets, E, M, N, y_type, Y, ldy, s);
}

}  // extern "C"
