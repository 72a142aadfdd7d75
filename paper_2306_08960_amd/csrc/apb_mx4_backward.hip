// Gradients of the 4-bit product at its quantized operands:
//      dX[m, k] = sum_n G[m, n] W^[n, k]          dW[n, k] = sum_m G[m, n] X^[m, k]
// Both sum over the ROWS of a 4-bit matrix, across its blocks, so its scales cannot ride along in the matrix instruction; its
// values, products of a level and a power of two, are exact in bfloat16, and the bfloat16 matrix instruction multiplies them
// with G.  A bfloat16 G is taken as it is; a float16 G is the sum of two bfloat16 values, a float32 G of three (each part takes
// the next 8 bits), and each part goes through the matrix cores, so no bit of G is dropped.
#include <type_traits>

#include "apb_mx4.h"

namespace apb {
namespace {

constexpr int kThreads = 256;
constexpr int kStep = 64;                     // summed over per pass: a line of 128 bytes of bfloat16 in LDS

template <int TYPE>
struct Parts {
    static constexpr int n = TYPE == APB_F32 ? 3 : TYPE == APB_F16 ? 2 : 1;
};

// LDS tiles: `row` (an output index) has kStep bfloat16 values, in chunks of eight.  The chunks of a row are permuted by the
// row's number so that neither a wave that writes one chunk of every eighth row nor one that reads the same chunk of 32
// successive rows meets a bank twice.
__device__ __forceinline__ int lds_at(int row, int chunk) { return row * kStep + 8 * (chunk ^ ((row + (row >> 3)) & 7)); }

// The bfloat16 parts of eight values, pairs of neighbours in a word: each takes the leading 8 significant bits of what is left
// (cut off, so that no part is larger than the value and none overflows).  Bits below 2^-133, which bfloat16 has not, are lost.
template <int TYPE>
__device__ __forceinline__ void split(const Eight<TYPE>& v, u32x4 (&part)[Parts<TYPE>::n]) {
    if (TYPE == APB_BF16) {
        part[0] = v.w[0];
        return;
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        float x[2];
        if (TYPE == APB_F32) {
            const uint32_t a = v.w[TYPE == APB_F32 ? q / 2 : 0][2 * q & 3], c = v.w[TYPE == APB_F32 ? q / 2 : 0][(2 * q & 3) + 1];
            x[0] = __builtin_bit_cast(float, a);
            x[1] = __builtin_bit_cast(float, c);
        } else {
            const uint32_t pair = v.w[0][q];
            const f16x2 p = __builtin_bit_cast(f16x2, pair);
            x[0] = (float)p[0];
            x[1] = (float)p[1];
        }
#pragma unroll
        for (int p = 0; p < Parts<TYPE>::n; ++p) {
            uint32_t bits[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                bits[i] = __builtin_bit_cast(uint32_t, x[i]);
                // an infinity is its own first part; a NaN leaves a NaN
                x[i] = (bits[i] & 0x7fffffffu) == 0x7f800000u ? 0.0f : x[i] - __builtin_bit_cast(float, bits[i] & 0xffff0000u);
            }
            part[p][q] = __builtin_amdgcn_perm(bits[1], bits[0], 0x07060302u);
        }
    }
}

// 8 x 8 transpose into LDS: in[c] holds the values of output indices row .. row+7 at summation index c, two to a word
__device__ __forceinline__ void store_transposed(uint16_t* tile, int row, int chunk, const u32x4 (&in)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        u32x4 w;
#pragma unroll
        for (int q = 0; q < 4; ++q)
            w[q] = __builtin_amdgcn_perm(in[2 * q + 1][i / 2], in[2 * q][i / 2], i & 1 ? 0x07060302u : 0x05040100u);
        *reinterpret_cast<u32x4*>(tile + lds_at(row + i, chunk)) = w;
    }
}

// OUT[i, j] = sum_c P[i, c] Q^[c, j] over the 4-bit matrix Q's rows c.
//   WEIGHT = false: P = G, i = row m of the group, c = n.     WEIGHT = true: P = G^T, i = n, c = row m of the group.
// A workgroup makes a tile of 64 * F x 64 * F outputs, a wave 32 * F x 32 * F.  A pass sums over 64 indices: while the matrix
// cores work on one buffer of LDS, the next pass's operands, loaded during the pass before, are brought into the other one as
// rows of output indices: 8 x 8 blocks transposed in registers, 4-bit values widened to bfloat16.
template <int TYPE, bool WEIGHT, int F>
__global__ __launch_bounds__(kThreads, F * Parts<TYPE>::n <= 2 ? 2 : 1) void k_mx4_backward(const void* __restrict__ G, long long ldg, Mx Q,
                                                                           const int32_t* __restrict__ offsets, int E, int M, int N,
                                                                           int K, int type, void* __restrict__ out, long long ldo) {
    constexpr int NP = Parts<TYPE>::n;
    constexpr int kTile = 64 * F;
    constexpr int kBuffer = (NP + 1) * kTile * kStep;
    __shared__ __align__(16) uint16_t lds[2 * kBuffer];
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
    const int wi = (wave >> 1) * 32 * F, wj = (wave & 1) * 32 * F;
    const int r = lane & 31, h = lane >> 5;
    // who brings in what: blocks of 8 x 8 of either operand
    const int unit = tid & (kTile - 1);
    const bool has_g = F == 4 || tid < kTile, has_q = F == 4 || (tid >= kTile && tid < 2 * kTile);
    const int block = 8 * (unit & (kTile / 8 - 1)), chunk = unit / (kTile / 8);       // output indices, summation indices / 8
    const int line = unit >> 3, part_of_line = unit & 7;                              // G of dX: rows as they lie in memory
    const uint8_t* q_codes = Q.codes + (j0 + block) / 2;
    const uint8_t* q_scales = Q.scales + (size_t)((j0 + block) / kMxSeg) * Q.rows * 8 + (j0 + block) % kMxSeg / kMxBlock;
    const uint32_t q_pitch = (uint32_t)Q.segs * kMxSegBytes;

    f32x16 acc[F][F];
#pragma unroll
    for (int x = 0; x < F; ++x)
#pragma unroll
        for (int y = 0; y < F; ++y)
#pragma unroll
            for (int q = 0; q < 16; ++q) acc[x][y][q] = 0.0f;

    Eight<TYPE> g[8];
    uint32_t code[8], scale[8];
    // WHOLE: the pass lies inside G and Q; otherwise what lies outside is zero
    auto load = [&](int c, auto whole) {
        constexpr bool WHOLE = decltype(whole)::value;
        if (has_g) {
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                if (WEIGHT) {
                    const int cc = c + 8 * chunk + u;
                    const int col = WHOLE ? min(i0 + block, N - 8) : i0 + block;
                    const long long at = (long long)(g_row + cc) * ldg + col;
                    g[u] = WHOLE ? load_eight<TYPE>(G, at) : load_some<TYPE>(G, at, cc < rows_c ? rows_i - block : 0);
                } else {
                    const int row = min(u * (kTile / 8) + line, rows_i - 1);
                    const long long at = (long long)(g_row + row) * ldg + c + 8 * part_of_line;
                    g[u] = WHOLE ? load_eight<TYPE>(G, at) : load_some<TYPE>(G, at, rows_c - c - 8 * part_of_line);
                }
            }
        }
        if (has_q) {
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const int cc = c + 8 * chunk + u;
                const bool there = WHOLE || cc < rows_c;
                const size_t row = (size_t)c0 + (WHOLE ? cc : min(cc, rows_c - 1));
                code[u] = *reinterpret_cast<const uint32_t*>(q_codes + row * q_pitch);
                scale[u] = q_scales[row * 8];
                if (!WHOLE) {
                    code[u] = there ? code[u] : 0u;
                    scale[u] = there ? scale[u] : 0u;
                }
            }
        }
    };
    auto bring = [&](uint16_t* buffer) {
        if (has_g) {
            if (WEIGHT) {
                u32x4 part[NP][8];
#pragma unroll
                for (int u = 0; u < 8; ++u) {
                    u32x4 v[NP];
                    split<TYPE>(g[u], v);
#pragma unroll
                    for (int p = 0; p < NP; ++p) part[p][u] = v[p];
                }
#pragma unroll
                for (int p = 0; p < NP; ++p) store_transposed(buffer + p * kTile * kStep, block, chunk, part[p]);
            } else {
#pragma unroll
                for (int u = 0; u < 8; ++u) {
                    u32x4 v[NP];
                    split<TYPE>(g[u], v);
#pragma unroll
                    for (int p = 0; p < NP; ++p)
                        *reinterpret_cast<u32x4*>(buffer + p * kTile * kStep + lds_at(u * (kTile / 8) + line, part_of_line)) = v[p];
                }
            }
        }
        if (has_q) {
            // (the conversion takes the scale as a float's exponent: every code is right as it is, 0 and NaN's 255 too)
            u32x4 v[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const float s = __builtin_bit_cast(float, scale[u] << 23);
                v[u][0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code[u], s, 0));
                v[u][1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code[u], s, 1));
                v[u][2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code[u], s, 2));
                v[u][3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code[u], s, 3));
            }
            store_transposed(buffer + NP * kTile * kStep, block, chunk, v);
        }
    };
    auto multiply = [&](const uint16_t* buffer, int ks) {
        bf16x8 b[F];
#pragma unroll
        for (int y = 0; y < F; ++y)
            b[y] = *reinterpret_cast<const bf16x8*>(buffer + NP * kTile * kStep + lds_at(wj + 32 * y + r, 2 * ks + h));
#pragma unroll
        for (int p = 0; p < NP; ++p)
#pragma unroll
            for (int x = 0; x < F; ++x) {
                const bf16x8 a = *reinterpret_cast<const bf16x8*>(buffer + p * kTile * kStep + lds_at(wi + 32 * x + r, 2 * ks + h));
#pragma unroll
                for (int y = 0; y < F; ++y) acc[x][y] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(b[y], a, acc[x][y], 0, 0, 0);
            }
    };
    constexpr std::true_type kWhole{};
    constexpr std::false_type kEdge{};
    // passes that lie inside both operands
    const int whole = !WEIGHT || rows_i == kTile || (N % 8 == 0) ? rows_c / kStep : 0;
    if (whole > 0) {
        load(0, kWhole);
        bring(lds);
        load(min(1, whole - 1) * kStep, kWhole);
        __syncthreads();
        for (int pass = 0; pass < whole; ++pass) {
            const uint16_t* now = lds + (pass & 1) * kBuffer;
            multiply(now, 0);
            multiply(now, 1);
            bring(lds + (1 - (pass & 1)) * kBuffer);             // (after the last pass: once more, unread)
            load(min(pass + 2, whole - 1) * kStep, kWhole);
            multiply(now, 2);
            multiply(now, 3);
            __syncthreads();
        }
    }
    for (int c = whole * kStep; c < rows_c; c += kStep) {
        load(c, kEdge);
        bring(lds);
        __syncthreads();
#pragma unroll
        for (int ks = 0; ks < kStep / 16; ++ks) multiply(lds, ks);
        __syncthreads();
    }
    // the 4-bit matrix was the first operand: a lane holds four neighbours of an output row
#pragma unroll
    for (int x = 0; x < F; ++x) {
        const int i = wi + 32 * x + r;
        if (i >= rows_i) continue;
        const long long row = (long long)(out_row + i) * ldo;
#pragma unroll
        for (int y = 0; y < F; ++y)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int j = j0 + wj + 32 * y + 8 * q + 4 * h;
                const float v[4] = {acc[x][y][4 * q], acc[x][y][4 * q + 1], acc[x][y][4 * q + 2], acc[x][y][4 * q + 3]};
                store4(out, type, row + j, v, K - j);
            }
    }
}

template <int TYPE, bool WEIGHT, int F>
void launch_tiles(const void* G, long long ldg, const Mx& Q, const int32_t* offsets, int E, int M, int N, int K, int type, void* out,
                  long long ldo, hipStream_t s) {
    constexpr int kTile = 64 * F;
    const unsigned tiles_i = (unsigned)(WEIGHT ? (N + kTile - 1) / kTile : max_row_tiles(M, E, offsets != nullptr, kTile));
    const dim3 grid(tiles_i, (unsigned)((K + kTile - 1) / kTile), (unsigned)(WEIGHT ? E : 1));
    hipLaunchKernelGGL((k_mx4_backward<TYPE, WEIGHT, F>), grid, dim3(kThreads), 0, s, G, ldg, Q, offsets, E, M, N, K, type, out, ldo);
}

template <int TYPE, bool WEIGHT>
void launch_type(const void* G, long long ldg, const Mx& Q, const int32_t* offsets, int E, int M, int N, int K, int type, void* out,
                 long long ldo, hipStream_t s) {
    const long long big = ((long long)(WEIGHT ? N : M) + 255) / 256 * ((K + 255) / 256) * (WEIGHT ? E : 1);
    if constexpr (TYPE == APB_BF16) {
        if (big >= 192) return launch_tiles<TYPE, WEIGHT, 4>(G, ldg, Q, offsets, E, M, N, K, type, out, ldo, s);
    }
    if (big * 4 >= 192) return launch_tiles<TYPE, WEIGHT, 2>(G, ldg, Q, offsets, E, M, N, K, type, out, ldo, s);
    launch_tiles<TYPE, WEIGHT, 1>(G, ldg, Q, offsets, E, M, N, K, type, out, ldo, s);
}

template <bool WEIGHT>
int launch(const void* G, int g_type, long long ldg, const Mx& Q, const int32_t* offsets, int E, int M, int N, int K, int type,
           void* out, long long ldo, hipStream_t s) {
    if (g_type == APB_F32) launch_type<APB_F32, WEIGHT>(G, ldg, Q, offsets, E, M, N, K, type, out, ldo, s);
    else if (g_type == APB_BF16) launch_type<APB_BF16, WEIGHT>(G, ldg, Q, offsets, E, M, N, K, type, out, ldo, s);
    else launch_type<APB_F16, WEIGHT>(G, ldg, Q, offsets, E, M, N, K, type, out, ldo, s);
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
