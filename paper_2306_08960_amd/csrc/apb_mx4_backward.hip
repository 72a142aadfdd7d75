// Gradients of the 4-bit product at its quantized operands:
//      dX[m, k] = sum_n G[m, n] W^[n, k]          dW[n, k] = sum_m G[m, n] X^[m, k]
// Both sum over the ROWS of a 4-bit matrix, across its blocks, so its scales cannot ride along in the matrix instruction; its
// values, products of a level and a power of two, are exact in bfloat16, and the bfloat16 matrix instruction multiplies them
// with G.  A bfloat16 G is taken as it is; a float16 G is the sum of two bfloat16 values, a float32 G of three (each part takes
// the next 8 bits), and each part goes through the matrix cores, so no bit of G is dropped.
#include "apb_mx4.h"

namespace apb {
namespace {

constexpr int kThreads = 256;
constexpr int kTile = 128;                    // outputs of a workgroup: 128 x 128, of a wave 64 x 64
constexpr int kStep = 64;                     // summed over per pass: a line of 128 bytes of bfloat16 in LDS

template <int TYPE>
struct Parts {
    static constexpr int n = TYPE == APB_F32 ? 3 : TYPE == APB_F16 ? 2 : 1;
};

// Bit patterns of the bfloat16 parts of a value: each takes the leading 8 significant bits of what is left (truncated, so that
// no part is larger than the value and none overflows).  Bits below 2^-133, which bfloat16 has not, are lost.
template <int TYPE>
__device__ __forceinline__ void split(float v, uint16_t (&part)[Parts<TYPE>::n]) {
#pragma unroll
    for (int p = 0; p < Parts<TYPE>::n; ++p) {
        const uint32_t bits = __builtin_bit_cast(uint32_t, v);
        part[p] = (uint16_t)(bits >> 16);
        // an infinity is its own first part; a NaN leaves a NaN
        v = (bits & 0x7fffffffu) == 0x7f800000u ? 0.0f : v - __builtin_bit_cast(float, bits & 0xffff0000u);
    }
}

// LDS tiles: `row` (an output index) has kStep bfloat16 values, in chunks of eight.  The chunks of a row are permuted by the
// row's number so that neither a wave that writes one chunk of every eighth row nor one that reads the same chunk of 32
// successive rows meets a bank twice.
__device__ __forceinline__ int lds_at(int row, int chunk) { return row * kStep + 8 * (chunk ^ ((row + (row >> 3)) & 7)); }

// 8 x 8 transpose: in[c] holds the values of output indices 0..7 at summation index c as bit patterns, out[i] the eight
// summation indices of output index i
__device__ __forceinline__ u32x4 column(const uint16_t (&in)[8][8], int i) {
    u32x4 w;
#pragma unroll
    for (int q = 0; q < 4; ++q) w[q] = (uint32_t)in[2 * q][i] | (uint32_t)in[2 * q + 1][i] << 16;
    return w;
}

// OUT[i, j] = sum_c P[i, c] Q^[c, j] over the 4-bit matrix Q's rows c.
//   WEIGHT = false: P = G, i = row m of the group, c = n.     WEIGHT = true: P = G^T, i = n, c = row m of the group.
template <int TYPE, bool WEIGHT>
__global__ __launch_bounds__(kThreads) void k_mx4_backward(const void* __restrict__ G, long long ldg, Mx Q,
                                                           const int32_t* __restrict__ offsets, int E, int M, int N, int K,
                                                           int type, void* __restrict__ out, long long ldo, bool vec) {
    constexpr int NP = Parts<TYPE>::n;
    __shared__ uint16_t P[NP][kTile * kStep];
    __shared__ uint16_t Qs[kTile * kStep];
    const int j0 = blockIdx.y * kTile;
    int i0, rows_i, c0, rows_c, out_row;                         // outputs, summation range (rows of Q from c0 on)
    int g_row;                                                   // row of G that belongs to i0 (or to c0, WEIGHT)
    if (WEIGHT) {
        const int e = blockIdx.z;
        int a = 0, b = M;
        if (offsets) {
            a = min(max(offsets[e], 0), M);
            b = max(a, min(offsets[e + 1], M));
        }
        i0 = blockIdx.x * kTile;
        rows_i = min(kTile, N - i0);
        c0 = g_row = a;
        rows_c = b - a;
        out_row = e * N + i0;
    } else {
        const RowTile t = find_row_tile(offsets, E, M, kTile, blockIdx.x);
        if (t.rows <= 0) return;
        i0 = 0;
        rows_i = t.rows;
        c0 = t.e * N;
        rows_c = t.e < E ? N : 0;
        out_row = g_row = t.row0;
    }
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
    const int wi = (wave >> 1) * 64, wj = (wave & 1) * 64;
    f32x16 acc[2][2];
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int y = 0; y < 2; ++y)
#pragma unroll
            for (int q = 0; q < 16; ++q) acc[x][y][q] = 0.0f;

    for (int c = 0; c < rows_c; c += kStep) {
        __syncthreads();
        if (tid < kThreads / 2) {
            // G
            if (WEIGHT) {
                const int io = (tid & 15) * 8, co = tid >> 4;    // eight outputs, eight summation indices
                uint16_t v[NP][8][8];
#pragma unroll
                for (int q = 0; q < 8; ++q) {
                    const int cc = c + 8 * co + q;
                    const long long at = (long long)(g_row + cc) * ldg + i0 + io;
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        uint16_t part[NP];
                        split<TYPE>(cc < rows_c && io + i < rows_i ? load_f32(G, TYPE, at + i) : 0.0f, part);
#pragma unroll
                        for (int p = 0; p < NP; ++p) v[p][q][i] = part[p];
                    }
                }
#pragma unroll
                for (int p = 0; p < NP; ++p)
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        *reinterpret_cast<u32x4*>(&P[p][lds_at(io + i, co)]) = column(v[p], i);
            } else {
#pragma unroll
                for (int u = 0; u < 8; ++u) {
                    const int row = u * 16 + (tid >> 3), chunk = tid & 7;
                    uint16_t v[NP][8];
                    const long long at = (long long)(g_row + row) * ldg + c + 8 * chunk;
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        uint16_t part[NP];
                        split<TYPE>(row < rows_i && c + 8 * chunk + i < rows_c ? load_f32(G, TYPE, at + i) : 0.0f, part);
#pragma unroll
                        for (int p = 0; p < NP; ++p) v[p][i] = part[p];
                    }
#pragma unroll
                    for (int p = 0; p < NP; ++p) {
                        u32x4 w;
#pragma unroll
                        for (int q = 0; q < 4; ++q) w[q] = (uint32_t)v[p][2 * q] | (uint32_t)v[p][2 * q + 1] << 16;
                        *reinterpret_cast<u32x4*>(&P[p][lds_at(row, chunk)]) = w;
                    }
                }
            }
        } else {
            // eight rows of Q, eight neighbours each: one word of codes and one scale per row
            const int jo = (tid & 15) * 8, co = (tid >> 4) & 7, j = j0 + jo;
            uint16_t v[8][8];
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                const int cc = c + 8 * co + q;
                uint32_t w = 0;
                float scale = 0.0f;
                if (cc < rows_c) {
                    const size_t row = (size_t)c0 + cc;
                    w = *reinterpret_cast<const uint32_t*>(Q.codes + row * Q.segs * kMxSegBytes + j / 2);
                    scale = scale_value(Q.scales[((size_t)(j / kMxSeg) * Q.rows + row) * 8 + (j % kMxSeg) / kMxBlock]);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const auto p = i == 0   ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 0)
                                   : i == 1 ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 1)
                                   : i == 2 ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 2)
                                            : __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 3);
                    v[q][2 * i] = __builtin_bit_cast(uint16_t, (__bf16)(p[0] * scale));
                    v[q][2 * i + 1] = __builtin_bit_cast(uint16_t, (__bf16)(p[1] * scale));
                }
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) *reinterpret_cast<u32x4*>(&Qs[lds_at(jo + i, co)]) = column(v, i);
        }
        __syncthreads();
        const int r = lane & 31, h = lane >> 5;
#pragma unroll
        for (int ks = 0; ks < kStep / 16; ++ks) {
            bf16x8 b[2];
#pragma unroll
            for (int y = 0; y < 2; ++y) b[y] = *reinterpret_cast<const bf16x8*>(&Qs[lds_at(wj + 32 * y + r, 2 * ks + h)]);
#pragma unroll
            for (int p = 0; p < NP; ++p)
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    const bf16x8 a = *reinterpret_cast<const bf16x8*>(&P[p][lds_at(wi + 32 * x + r, 2 * ks + h)]);
#pragma unroll
                    for (int y = 0; y < 2; ++y) acc[x][y] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(b[y], a, acc[x][y], 0, 0, 0);
                }
        }
    }
    // the 4-bit matrix was the first operand: a lane holds four neighbours of an output row
    const int r = lane & 31, h = lane >> 5;
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        const int i = wi + 32 * x + r;
        if (i >= rows_i) continue;
        const long long row = (long long)(out_row + i) * ldo;
#pragma unroll
        for (int y = 0; y < 2; ++y)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int j = j0 + wj + 32 * y + 8 * g + 4 * h;
                const float v[4] = {acc[x][y][4 * g], acc[x][y][4 * g + 1], acc[x][y][4 * g + 2], acc[x][y][4 * g + 3]};
                store4(out, type, row + j, v, K - j, vec);
            }
    }
}

template <bool WEIGHT>
int launch(const void* G, int g_type, long long ldg, const Mx& Q, const int32_t* offsets, int E, int M, int N, int K, int type,
           void* out, long long ldo, hipStream_t s) {
    const unsigned tiles_i = (unsigned)(WEIGHT ? (N + kTile - 1) / kTile : max_row_tiles(M, E, offsets != nullptr, kTile));
    const dim3 grid(tiles_i, (unsigned)((K + kTile - 1) / kTile), (unsigned)(WEIGHT ? E : 1));
    const bool vec = rows_aligned16(out, ldo, type);
    if (g_type == APB_F32)
        hipLaunchKernelGGL((k_mx4_backward<APB_F32, WEIGHT>), grid, dim3(kThreads), 0, s, G, ldg, Q, offsets, E, M, N, K, type, out, ldo, vec);
    else if (g_type == APB_BF16)
        hipLaunchKernelGGL((k_mx4_backward<APB_BF16, WEIGHT>), grid, dim3(kThreads), 0, s, G, ldg, Q, offsets, E, M, N, K, type, out, ldo, vec);
    else
        hipLaunchKernelGGL((k_mx4_backward<APB_F16, WEIGHT>), grid, dim3(kThreads), 0, s, G, ldg, Q, offsets, E, M, N, K, type, out, ldo, vec);
    APB_HIP(hipGetLastError());
    return APB_OK;
}

int check(const void* G, int g_type, long long ldg, const void* Q, const int32_t* offsets, int E, int M, int N, int K, int type,
          const void* out, long long ldo) {
    if (!G || !Q || !out) return APB_ERR_NULL;
    if (bad_type(g_type) || bad_type(type)) return APB_ERR_TYPE;
    if (bad_product(E, M, N, K, offsets) || ldg < N || ldo < K) return APB_ERR_SHAPE;
    if (!aligned(G, type_size(g_type)) || !aligned(Q, 16) || !aligned(out, type_size(type)) || !aligned(offsets, 4)) return APB_ERR_ALIGN;
    return APB_OK;
}

}  // namespace
}  // namespace apb

using namespace apb;

extern "C" {

int apb_mx4_backward_input(const void* G, int g_type, long long ldg, const void* W, const int32_t* offsets, int E, int M,
                           int N, int K, int type, void* dX, long long ldx, void* stream) {
    const int rc = check(G, g_type, ldg, W, offsets, E, M, N, K, type, dX, ldx);
    if (rc != APB_OK) return rc;
    return launch<false>(G, g_type, ldg, mx_view(W, E * N, K), offsets, E, M, N, K, type, dX, ldx, reinterpret_cast<hipStream_t>(stream));
}

int apb_mx4_backward_weight(const void* G, int g_type, long long ldg, const void* X, const int32_t* offsets, int E, int M,
                            int N, int K, int type, void* dW, long long ldw, void* stream) {
    const int rc = check(G, g_type, ldg, X, offsets, E, M, N, K, type, dW, ldw);
    if (rc != APB_OK) return rc;
    return launch<true>(G, g_type, ldg, mx_view(X, M, K), offsets, E, M, N, K, type, dW, ldw, reinterpret_cast<hipStream_t>(stream));
}

}  // extern "C"
