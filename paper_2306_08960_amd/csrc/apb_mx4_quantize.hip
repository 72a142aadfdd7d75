// Quantization to microscaled 4-bit blocks and back.  A block is 32 neighbours along K with one scale 2^e,
// e = floor(log2(max |x|)) - 2, so that the largest magnitude lies in [4, 8) * 2^e, and each value becomes the nearest of
// +-{0, .5, 1, 1.5, 2, 3, 4, 6} * 2^e (ties to the even index, beyond 6: 6).  The conversion instruction scales and rounds
// once, so the codes are defined to the bit.  Both directions are one pass over memory and bound by it: 16384 x 4096 bfloat16
// values, 134 MB and 36 MB of codes and scales, take 39 us there (4.4 TB/s; a large copy runs at 5.1) and 27 us back.
#include "apb_mx4.h"

namespace apb {
namespace {

constexpr int kThreads = 256;

// Rows whose values lie side by side.  32 lanes take a segment of 256 values of a row, eight each; the four lanes of a block
// exchange their maxima.  `item` counts segments row by row.
template <int TYPE>
__global__ __launch_bounds__(kThreads) void k_mx4_quantize(const void* __restrict__ X, long long row_stride, int rows_in,
                                                           const int32_t* __restrict__ rows_from, int rows, int K, int segs,
                                                           FastDiv by_segs, uint8_t* __restrict__ codes,
                                                           uint8_t* __restrict__ scales) {
    const uint32_t item = blockIdx.x * (kThreads / 32) + threadIdx.x / 32;
    const int l = threadIdx.x & 31;
    const int r = (int)by_segs.div(item), seg = (int)(item - (uint32_t)r * segs);
    if (r >= rows) return;
    const int src = rows_from ? rows_from[r] : r;
    const int k = seg * kMxSeg + 8 * l;
    const Eight<TYPE> v = load_some<TYPE>(X, (long long)src * row_stride + k, src >= 0 && src < rows_in ? K - k : 0);
    const uint32_t code = scale_code(top_of_four(top_bits(v)));
    *reinterpret_cast<uint32_t*>(codes + ((size_t)r * segs + seg) * kMxSegBytes + 4 * l) = encode8(v, code);
    if ((l & 3) == 0) scales[((size_t)seg * rows + r) * 8 + l / 4] = (uint8_t)code;
}

// Any strides: a lane takes a block of 32 values, neighbouring lanes neighbouring rows (the order of a K x M matrix), and the eight
// waves the blocks of a segment, so that codes and scales leave as whole lines, through LDS.  16384 x 4096 bfloat16 values of a
// K x M matrix: 59 us, 66 with each lane writing its own 16 bytes; two bytes to a lane, a load fetches one line for 64 rows.
constexpr int kStridedThreads = 8 * kWave;
template <int TYPE>
__global__ __launch_bounds__(kStridedThreads) void k_mx4_quantize_strided(const void* __restrict__ X, long long row_stride,
                                                                          long long col_stride, int rows_in,
                                                                          const int32_t* __restrict__ rows_from, int rows, int K,
                                                                          int segs, uint8_t* __restrict__ codes,
                                                                          uint8_t* __restrict__ scales) {
    constexpr int kPitch = kMxSegBytes + 16;                     // (rows start 4 banks apart)
    __shared__ __align__(16) uint8_t lines[kWave * kPitch];
    __shared__ __align__(16) uint8_t marks[kWave * 8];
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const int row0 = blockIdx.x * kWave, seg = blockIdx.y;
    const int r = min(row0 + lane, rows - 1), block = seg * 8 + wave;
    const int src = rows_from ? rows_from[r] : r;
    const int have = src >= 0 && src < rows_in ? K - block * kMxBlock : 0;
    const long long at = (long long)src * row_stride + (long long)block * kMxBlock * col_stride;
    Eight<TYPE> v[4];
    uint32_t top = 0;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            const long long i = at + (8 * g + q) * col_stride;
            if constexpr (TYPE == APB_F32) {
                v[g].w[q / 4][q & 3] = 8 * g + q < have ? static_cast<const uint32_t*>(X)[i] : 0u;
            } else {
                const uint32_t x = 8 * g + q < have ? static_cast<const uint16_t*>(X)[i] : 0u;
                v[g].w[0][q / 2] = q & 1 ? v[g].w[0][q / 2] | x << 16 : x;
            }
        }
        top = max(top, top_bits(v[g]));
    }
    const uint32_t code = scale_code(top);
    u32x4 w;
#pragma unroll
    for (int g = 0; g < 4; ++g) w[g] = encode8(v[g], code);
    *reinterpret_cast<u32x4*>(lines + lane * kPitch + 16 * wave) = w;
    marks[lane * 8 + wave] = (uint8_t)code;
    __syncthreads();
    const int there = min(kWave, rows - row0);
    const int line = threadIdx.x >> 3, chunk = threadIdx.x & 7;
    if (line < there)
        *reinterpret_cast<u32x4*>(codes + ((size_t)(row0 + line) * segs + seg) * kMxSegBytes + 16 * chunk) =
            *reinterpret_cast<const u32x4*>(lines + line * kPitch + 16 * chunk);
    if ((int)threadIdx.x < 2 * there)
        *reinterpret_cast<uint32_t*>(scales + ((size_t)seg * rows + row0) * 8 + 4 * threadIdx.x) =
            *reinterpret_cast<const uint32_t*>(marks + 4 * threadIdx.x);
}

__global__ __launch_bounds__(kThreads) void k_mx4_dequantize(Mx mx, int K, FastDiv by_segs, int type, void* __restrict__ X,
                                                             long long ldx) {
    const uint32_t item = blockIdx.x * (kThreads / 32) + threadIdx.x / 32;
    const int l = threadIdx.x & 31;
    const int r = (int)by_segs.div(item), seg = (int)(item - (uint32_t)r * mx.segs);
    const int k = seg * kMxSeg + 8 * l;
    if (r >= mx.rows || k >= K) return;
    const uint32_t w = *reinterpret_cast<const uint32_t*>(mx.codes + ((size_t)r * mx.segs + seg) * kMxSegBytes + 4 * l);
    const float scale = scale_value(mx.scales[((size_t)seg * mx.rows + r) * 8 + l / 4]);
    float v[2][4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const auto p = q == 0   ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 0)
                       : q == 1 ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 1)
                       : q == 2 ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 2)
                                : __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 3);
        v[q / 2][2 * (q & 1)] = p[0] * scale;
        v[q / 2][2 * (q & 1) + 1] = p[1] * scale;
    }
    const long long at = (long long)r * ldx + k;
    store4(X, type, at, v[0], K - k);
    store4(X, type, at + 4, v[1], K - k - 4);
}

template <int TYPE>
void quantize_type(const void* X, long long row_stride, long long col_stride, int rows_in, const int32_t* rows_from, int rows,
                   int K, uint8_t* codes, uint8_t* scales, hipStream_t s) {
    const int segs = mx_segs(K);
    if (col_stride == 1) {
        const unsigned blocks = (unsigned)(((long long)rows * segs + kThreads / 32 - 1) / (kThreads / 32));
        const FastDiv by_segs((uint32_t)segs);
        hipLaunchKernelGGL((k_mx4_quantize<TYPE>), dim3(blocks), dim3(kThreads), 0, s, X, row_stride, rows_in, rows_from, rows, K, segs,
                           by_segs, codes, scales);
        return;
    }
    const dim3 grid((unsigned)((rows + kWave - 1) / kWave), (unsigned)segs);
    hipLaunchKernelGGL((k_mx4_quantize_strided<TYPE>), grid, dim3(kStridedThreads), 0, s, X, row_stride, col_stride, rows_in, rows_from,
                       rows, K, segs, codes, scales);
}

}  // namespace

int launch_mx4_quantize(const void* X, int type, long long row_stride, long long col_stride, int rows_in,
                        const int32_t* rows_from, int rows, int K, void* mx, hipStream_t s) {
    uint8_t* codes = static_cast<uint8_t*>(mx);
    uint8_t* scales = codes + (size_t)rows * mx_segs(K) * kMxSegBytes;
    if (type == APB_F32) quantize_type<APB_F32>(X, row_stride, col_stride, rows_in, rows_from, rows, K, codes, scales, s);
    else if (type == APB_BF16) quantize_type<APB_BF16>(X, row_stride, col_stride, rows_in, rows_from, rows, K, codes, scales, s);
    else quantize_type<APB_F16>(X, row_stride, col_stride, rows_in, rows_from, rows, K, codes, scales, s);
    APB_HIP(hipGetLastError());
    return APB_OK;
}

}  // namespace apb

using namespace apb;

extern "C" {

size_t apb_mx4_bytes(int rows, int K) {
    if (bad_shape_mx(rows, K)) return 0;
    return (size_t)rows * mx_segs(K) * (kMxSegBytes + 8);
}

int apb_mx4_quantize(const void* X, int type, long long row_stride, long long col_stride, int rows_in,
                     const int32_t* rows_from, int rows, int K, void* mx, void* stream) {
    if (!X || !mx) return APB_ERR_NULL;
    if (bad_type(type)) return APB_ERR_TYPE;
    if (bad_shape_mx(rows, K) || rows_in <= 0 || (!rows_from && rows_in != rows)) return APB_ERR_SHAPE;
    if (!aligned(mx, 16) || !aligned(X, type_size(type)) || !aligned(rows_from, 4)) return APB_ERR_ALIGN;
    return launch_mx4_quantize(X, type, row_stride, col_stride, rows_in, rows_from, rows, K, mx, reinterpret_cast<hipStream_t>(stream));
}

int apb_mx4_dequantize(const void* mx, int rows, int K, int type, void* X, long long ldx, void* stream) {
    if (!X || !mx) return APB_ERR_NULL;
    if (bad_type(type)) return APB_ERR_TYPE;
    if (bad_shape_mx(rows, K) || ldx < K) return APB_ERR_SHAPE;
    if (!aligned(mx, 16) || !aligned(X, type_size(type))) return APB_ERR_ALIGN;
    const Mx m = mx_view(mx, rows, K);
    const unsigned blocks = (unsigned)(((long long)rows * m.segs + kThreads / 32 - 1) / (kThreads / 32));
    hipLaunchKernelGGL(k_mx4_dequantize, dim3(blocks), dim3(kThreads), 0, reinterpret_cast<hipStream_t>(stream), m, K,
                       FastDiv((uint32_t)m.segs), type, X, ldx);
    APB_HIP(hipGetLastError());
    return APB_OK;
}

}  // extern "C"
