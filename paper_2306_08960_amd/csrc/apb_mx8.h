// 8-bit activation checkpoints and gated activations: what the kernels that write and read them share.
#pragma once

#include "apb_mx4.h"

namespace apb {

constexpr int kMx8Block = 32;
constexpr long long kMx8MaxBlocks = (1LL << 30) - 64;            // 64 go to a workgroup of 256 lanes, a launch has fewer than 2^32

inline int mx8_blocks(int K) { return (K + kMx8Block - 1) / kMx8Block; }
inline bool bad_shape_mx8(long long rows, int K) {
    return rows <= 0 || K <= 0 || K > kMxMaxK || rows * mx8_blocks(K) > kMx8MaxBlocks;
}

// An 8-bit matrix in memory (the layout of apb.h).
struct Mx8 {
    uint8_t* codes;                           // [rows][blocks * 32]
    uint8_t* scales;                          // [rows][blocks]
    int blocks;
};

inline Mx8 mx8_view(const void* p, long long rows, int K) {
    uint8_t* b = static_cast<uint8_t*>(const_cast<void*>(p));
    const int blocks = mx8_blocks(K);
    return Mx8{b, b ? b + rows * blocks * kMx8Block : b, blocks};
}

// From the largest magnitude's float bits: e + 127 of the block, 255 if it is not finite.
__device__ __forceinline__ uint32_t scale8_code(uint32_t top) {
    const uint32_t ex = top >> 23;
    return ex >= 255u ? 255u : ex > 6u ? ex - 6u : 0u;
}
// 2^-e (a normal number for every code that is not NaN's: 0 .. 248)
__device__ __forceinline__ float scale8_inverse(uint32_t code) { return __builtin_bit_cast(float, (254u - code) << 23); }

// Four values to four whole numbers in a word.  x * 2^-e, exact unless it is far below 1/2, is rounded once, to nearest even, where
// it is added to 3 * 2^22; the whole number then is in the low bits.
__device__ __forceinline__ uint32_t encode8_four(const float* v, float inverse, bool nan) {
    constexpr float kWhole = 12582912.0f;
    uint32_t i[4];
#pragma unroll
    for (int q = 0; q < 4; ++q)
        i[q] = float_bits(__builtin_amdgcn_fmed3f(__builtin_fmaf(v[q], inverse, kWhole), kWhole - 127.0f, kWhole + 127.0f));
    const uint32_t lo = __builtin_amdgcn_perm(i[1], i[0], 0x0c0c0400u), hi = __builtin_amdgcn_perm(i[3], i[2], 0x04000c0cu);
    return nan ? 0u : lo | hi;
}
__device__ __forceinline__ float decode8(uint32_t w, int q, float scale) { return (float)(int8_t)(w >> (8 * q)) * scale; }

// ---- activations ----------------------------------------------------------------------------------

// act(x) = x * s(z), z = x * (c0 + c1 * x^2), for SiLU (1, 0) and GELU; the constants times log2(e), as the exponential is one to
// base 2.  One form for all of them: what differs is uniform.
struct Act {
    float c0, c1;
    int relu;
};
inline bool bad_activation(int a) { return a != APB_SILU && a != APB_GELU && a != APB_RELU; }
inline Act act_of(int a) {
    const double log2e = 1.4426950408889634, c = 1.5957691216057308;           // 2 sqrt(2 / pi)
    if (a == APB_GELU) return Act{(float)(c * log2e), (float)(c * 0.044715 * log2e), 0};
    return Act{(float)log2e, 0.0f, a == APB_RELU};
}

// KIND: an apb_activation, or -1 for whichever `k` says.
// (x^2 is kept finite, for 0 * x^2; a NaN comes back in through x)
__device__ __forceinline__ float act_square(float x) { return fminf(x * x, 1e37f); }
template <int KIND = -1>
__device__ __forceinline__ float act_sigmoid(const Act& k, float x, float square) {
    const float z = KIND == APB_SILU ? k.c0 : __builtin_fmaf(k.c1, square, k.c0);
    return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-x * z));
}
// (the limit at -infinity: a finite value times s = 0)
__device__ __forceinline__ float act_times(float x, float s) { return fmaxf(x, -3.4028235e38f) * s; }
template <int KIND = -1>
__device__ __forceinline__ float act_value(const Act& k, float x) {
    const float relu = x < 0.0f ? 0.0f : x;
    if (KIND == APB_RELU || (KIND < 0 && k.relu)) return relu;
    return act_times(x, act_sigmoid<KIND>(k, x, KIND == APB_SILU ? 0.0f : act_square(x)));
}
__device__ __forceinline__ void act_both(const Act& k, float x, float& value, float& slope) {
    if (k.relu) {                                                // (a NaN is neither below nor above: both stay NaN)
        value = x < 0.0f ? 0.0f : x;
        slope = x > 0.0f ? 1.0f : x <= 0.0f ? 0.0f : x;
        return;
    }
    const float sq = act_square(x), s = act_sigmoid(k, x, sq);
    // s' = s (1 - s) z'; where s (1 - s) is 0, x may be infinite.  ln(2): the constants are to base 2
    const float p = s * (1.0f - s);
    value = act_times(x, s);
    slope = p == 0.0f ? s : __builtin_fmaf(x * p, 0.69314718f * __builtin_fmaf(3.0f * k.c1, sq, k.c0), s);
}

}  // namespace apb
