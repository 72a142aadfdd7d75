// 8-bit activation checkpoints to and from float matrices, and the gated activation Y = act(G) * U with its gradients, element by
// element: streams, bound by memory.
#include "apb_mx8.h"

namespace apb {
namespace {

constexpr int kThreads = 256;
constexpr int kItems = kThreads / 4;          // blocks of 32 columns that a workgroup takes, four lanes each

// Which block of a rows x K matrix a lane has eight values of: row r, block c, columns k .. k + 7.
struct Place {
    int r, c, k;
};
__device__ __forceinline__ Place place_of(const FastDiv& by_blocks) {
    const uint32_t item = blockIdx.x * kItems + threadIdx.x / 4;
    const uint32_t r = by_blocks.div(item), c = item - r * by_blocks.d;
    return Place{(int)r, (int)c, (int)(c * kMx8Block + 8 * (threadIdx.x & 3))};
}

template <int TYPE>
__device__ __forceinline__ void put8(const Mx8& m, long long row, const Place& p, const Eight<TYPE>& x, const float (&v)[8]) {
    const uint32_t code = scale8_code(top_of_four(top_bits(x)));
    const float inverse = scale8_inverse(code);
    const u32x2 w = {encode8_four(v, inverse, code == 255u), encode8_four(v + 4, inverse, code == 255u)};
    *reinterpret_cast<u32x2*>(m.codes + (row * m.blocks + p.c) * kMx8Block + 8 * (threadIdx.x & 3)) = w;
    if ((threadIdx.x & 3) == 0) m.scales[row * m.blocks + p.c] = (uint8_t)code;
}
__device__ __forceinline__ void get8(const Mx8& m, long long row, const Place& p, float (&v)[8]) {
    const u32x2 w = *reinterpret_cast<const u32x2*>(m.codes + (row * m.blocks + p.c) * kMx8Block + 8 * (threadIdx.x & 3));
    const float scale = scale_value(m.scales[row * m.blocks + p.c]);
#pragma unroll
    for (int q = 0; q < 8; ++q) v[q] = decode8(w[q / 4], q & 3, scale);
}

template <int TYPE>
__global__ __launch_bounds__(kThreads) void k_mx8_quantize(const void* __restrict__ X, long long ldx, int rows, int K,
                                                           FastDiv by_blocks, Mx8 out) {
    const Place p = place_of(by_blocks);
    if (p.r >= rows) return;
    const Eight<TYPE> x = load_some<TYPE>(X, p.r * ldx + p.k, K - p.k);
    float v[8];
    floats(x, v);
    put8<TYPE>(out, p.r, p, x, v);
}

template <int TYPE>
__global__ __launch_bounds__(kThreads) void k_mx8_dequantize(Mx8 mx8, int rows, int K, FastDiv by_blocks, void* __restrict__ X,
                                                             long long ldx) {
    const Place p = place_of(by_blocks);
    if (p.r >= rows || p.k >= K) return;
    float v[8];
    get8(mx8, p.r, p, v);
    store8<TYPE>(X, p.r * ldx + p.k, K - p.k, v);
}

template <int TYPE>
__global__ __launch_bounds__(kThreads) void k_gated_forward(const void* __restrict__ GU, long long ldgu, int M, int N, FastDiv by_blocks,
                                                            Act act, void* __restrict__ Y, long long ldy, Mx8 saved) {
    const Place p = place_of(by_blocks);
    if (p.r >= M) return;
    const Eight<TYPE> xg = load_some<TYPE>(GU, p.r * ldgu + p.k, N - p.k);
    const Eight<TYPE> xu = load_some<TYPE>(GU, p.r * ldgu + N + p.k, N - p.k);
    float g[8], u[8], y[8];
    floats(xg, g);
    floats(xu, u);
    if (saved.codes) {
        put8<TYPE>(saved, p.r, p, xg, g);
        put8<TYPE>(saved, (long long)M + p.r, p, xu, u);
    }
#pragma unroll
    for (int q = 0; q < 8; ++q) y[q] = act_value(act, g[q]) * u[q];
    store8<TYPE>(Y, p.r * ldy + p.k, N - p.k, y);
}

// FROM: an apb_type or APB_MX8.  (dGU may be GU: a lane writes where it alone has read.)
template <int FROM, int TYPE>
__global__ __launch_bounds__(kThreads) void k_gated_backward(const void* GU, long long ldgu, Mx8 saved, const void* __restrict__ dY,
                                                             long long lddy, int M, int N, FastDiv by_blocks, Act act, void* dGU,
                                                             long long lddgu, void* __restrict__ Y, long long ldy) {
    const Place p = place_of(by_blocks);
    if (p.r >= M || p.k >= N) return;
    const int have = N - p.k;
    float g[8], u[8], d[8], dg[8], y[8];
    if constexpr (FROM == APB_MX8) {
        get8(saved, p.r, p, g);
        get8(saved, (long long)M + p.r, p, u);
    } else {
        floats(load_some<FROM>(GU, p.r * ldgu + p.k, have), g);
        floats(load_some<FROM>(GU, p.r * ldgu + N + p.k, have), u);
    }
    floats(load_some<TYPE>(dY, p.r * lddy + p.k, have), d);
#pragma unroll
    for (int q = 0; q < 8; ++q) {
        float value, slope;
        act_both(act, g[q], value, slope);
        y[q] = value * u[q];
        dg[q] = d[q] * u[q] * slope;
        d[q] *= value;
    }
    store8<TYPE>(dGU, p.r * lddgu + p.k, have, dg);
    store8<TYPE>(dGU, p.r * lddgu + N + p.k, have, d);
    if (Y) store8<TYPE>(Y, p.r * ldy + p.k, have, y);
}

unsigned workgroups(long long rows, int K) { return (unsigned)((rows * mx8_blocks(K) + kItems - 1) / kItems); }

template <int FROM>
void backward_from(const void* GU, long long ldgu, const Mx8& saved, const void* dY, int type, long long lddy, int M, int N, const Act& act,
                   void* dGU, long long lddgu, void* Y, long long ldy, hipStream_t s) {
    const dim3 grid(workgroups(M, N));
    const FastDiv by((uint32_t)mx8_blocks(N));
    if (type == APB_F32)
        hipLaunchKernelGGL((k_gated_backward<FROM, APB_F32>), grid, dim3(kThreads), 0, s, GU, ldgu, saved, dY, lddy, M, N, by, act, dGU, lddgu, Y, ldy);
    else if (type == APB_BF16)
        hipLaunchKernelGGL((k_gated_backward<FROM, APB_BF16>), grid, dim3(kThreads), 0, s, GU, ldgu, saved, dY, lddy, M, N, by, act, dGU, lddgu, Y, ldy);
    else
        hipLaunchKernelGGL((k_gated_backward<FROM, APB_F16>), grid, dim3(kThreads), 0, s, GU, ldgu, saved, dY, lddy, M, N, by, act, dGU, lddgu, Y, ldy);
}

}  // namespace
}  // namespace apb

using namespace apb;

extern "C" {

size_t apb_mx8_bytes(int rows, int K) {
    if (bad_shape_mx8(rows, K)) return 0;
    return (size_t)rows * mx8_blocks(K) * (kMx8Block + 1);
}

int apb_mx8_quantize(const void* X, int type, long long ldx, int rows, int K, void* mx8, void* stream) {
    if (!X || !mx8) return APB_ERR_NULL;
    if (bad_type(type)) return APB_ERR_TYPE;
    if (bad_shape_mx8(rows, K) || ldx < K) return APB_ERR_SHAPE;
    if (!aligned(mx8, 16) || !aligned(X, type_size(type))) return APB_ERR_ALIGN;
    const dim3 grid(workgroups(rows, K));
    const FastDiv by((uint32_t)mx8_blocks(K));
    const Mx8 out = mx8_view(mx8, rows, K);
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    if (type == APB_F32) hipLaunchKernelGGL((k_mx8_quantize<APB_F32>), grid, dim3(kThreads), 0, s, X, ldx, rows, K, by, out);
    else if (type == APB_BF16) hipLaunchKernelGGL((k_mx8_quantize<APB_BF16>), grid, dim3(kThreads), 0, s, X, ldx, rows, K, by, out);
    else hipLaunchKernelGGL((k_mx8_quantize<APB_F16>), grid, dim3(kThreads), 0, s, X, ldx, rows, K, by, out);
    APB_HIP(hipGetLastError());
    return APB_OK;
}

int apb_mx8_dequantize(const void* mx8, int rows, int K, int type, void* X, long long ldx, void* stream) {
    if (!X || !mx8) return APB_ERR_NULL;
    if (bad_type(type)) return APB_ERR_TYPE;
    if (bad_shape_mx8(rows, K) || ldx < K) return APB_ERR_SHAPE;
    if (!aligned(mx8, 16) || !aligned(X, type_size(type))) return APB_ERR_ALIGN;
    const dim3 grid(workgroups(rows, K));
    const FastDiv by((uint32_t)mx8_blocks(K));
    const Mx8 in = mx8_view(mx8, rows, K);
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    if (type == APB_F32) hipLaunchKernelGGL((k_mx8_dequantize<APB_F32>), grid, dim3(kThreads), 0, s, in, rows, K, by, X, ldx);
    else if (type == APB_BF16) hipLaunchKernelGGL((k_mx8_dequantize<APB_BF16>), grid, dim3(kThreads), 0, s, in, rows, K, by, X, ldx);
    else hipLaunchKernelGGL((k_mx8_dequantize<APB_F16>), grid, dim3(kThreads), 0, s, in, rows, K, by, X, ldx);
    APB_HIP(hipGetLastError());
    return APB_OK;
}

int apb_gated_forward(const void* GU, int type, long long ldgu, int M, int N, int activation, void* Y, long long ldy, void* saved,
                      void* stream) {
    if (!GU || !Y) return APB_ERR_NULL;
    if (bad_type(type)) return APB_ERR_TYPE;
    if (bad_activation(activation)) return APB_ERR_VALUE;
    if (bad_shape_mx8(saved ? 2LL * M : M, N) || ldgu < 2LL * N || ldy < N) return APB_ERR_SHAPE;
    if (!aligned(GU, type_size(type)) || !aligned(Y, type_size(type)) || !aligned(saved, 16)) return APB_ERR_ALIGN;
    const dim3 grid(workgroups(M, N));
    const FastDiv by((uint32_t)mx8_blocks(N));
    const Mx8 keep = mx8_view(saved, 2LL * M, N);
    const Act act = act_of(activation);
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    if (type == APB_F32) hipLaunchKernelGGL((k_gated_forward<APB_F32>), grid, dim3(kThreads), 0, s, GU, ldgu, M, N, by, act, Y, ldy, keep);
    else if (type == APB_BF16) hipLaunchKernelGGL((k_gated_forward<APB_BF16>), grid, dim3(kThreads), 0, s, GU, ldgu, M, N, by, act, Y, ldy, keep);
    else hipLaunchKernelGGL((k_gated_forward<APB_F16>), grid, dim3(kThreads), 0, s, GU, ldgu, M, N, by, act, Y, ldy, keep);
    APB_HIP(hipGetLastError());
    return APB_OK;
}

int apb_gated_backward(const void* GU, int gu_type, long long ldgu, const void* dY, int type, long long lddy, int M, int N,
                       int activation, void* dGU, long long lddgu, void* Y, long long ldy, void* stream) {
    if (!GU || !dY || !dGU) return APB_ERR_NULL;
    if ((bad_type(gu_type) && gu_type != APB_MX8) || bad_type(type)) return APB_ERR_TYPE;
    if (bad_activation(activation)) return APB_ERR_VALUE;
    if (bad_shape_mx8(gu_type == APB_MX8 ? 2LL * M : M, N) || (gu_type != APB_MX8 && ldgu < 2LL * N) || lddy < N || lddgu < 2LL * N || (Y && ldy < N) ||
        (GU == dGU && (gu_type != type || ldgu != lddgu)))
        return APB_ERR_SHAPE;
    if (!aligned(GU, gu_type == APB_MX8 ? 16 : type_size(gu_type)) || !aligned(dY, type_size(type)) || !aligned(dGU, type_size(type)) ||
        !aligned(Y, type_size(type)))
        return APB_ERR_ALIGN;
    const Act act = act_of(activation);
    const Mx8 saved = mx8_view(GU, 2LL * M, N);
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    if (gu_type == APB_MX8) backward_from<APB_MX8>(GU, ldgu, saved, dY, type, lddy, M, N, act, dGU, lddgu, Y, ldy, s);
    else if (gu_type == APB_F32) backward_from<APB_F32>(GU, ldgu, saved, dY, type, lddy, M, N, act, dGU, lddgu, Y, ldy, s);
    else if (gu_type == APB_BF16) backward_from<APB_BF16>(GU, ldgu, saved, dY, type, lddy, M, N, act, dGU, lddgu, Y, ldy, s);
    else backward_from<APB_F16>(GU, ldgu, saved, dY, type, lddy, M, N, act, dGU, lddgu, Y, ldy, s);
    APB_HIP(hipGetLastError());
    return APB_OK;
}

}  // extern "C"
