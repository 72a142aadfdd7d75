// What the kernels of the microscaled 4-bit matrices share: the layout, element types, groups of rows.
#pragma once

#include <algorithm>

#include "apb_internal.h"
#include "apb_mx4_shape.h"

namespace apb {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

// A 4-bit matrix in memory (the layout of apb.h).
struct Mx {
    const uint8_t* codes;                     // [rows][segs * 128]
    const uint8_t* scales;                    // [segs][rows][8]
    int rows, segs;
};

inline Mx mx_view(const void* p, int rows, int K) {
    const int segs = mx_segs(K);
    const uint8_t* b = static_cast<const uint8_t*>(p);
    return Mx{b, b + (size_t)rows * segs * kMxSegBytes, rows, segs};
}

// The sizes of a product and of its gradients: M rows in E groups (offsets) against E matrices of N rows.
inline bool bad_product(int E, int M, int N, int K, const int32_t* offsets) {
    return E <= 0 || E > APB_MOE_MAX_E || N <= 0 || (!offsets && E != 1) || bad_shape_mx(M, K) ||
           bad_shape_mx((long long)E * N, K) || (N + 127) / 128 > 65535;
}

inline bool bad_type(int t) { return t != APB_F32 && t != APB_BF16 && t != APB_F16; }
inline int type_size(int t) { return t == APB_F32 ? 4 : 2; }
inline bool aligned(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

// n / d for any 32-bit n without a division (Granlund and Montgomery, "Division by invariant integers using multiplication", 1994):
// m = ceil(2^(32+s) / d) with 2^s >= d is less than 1 above 2^(32+s) / d, so n * m is less than 2^(32+s) / d above n * 2^(32+s) / d:
// too little to reach the next whole quotient.
struct FastDiv {
    uint32_t mul, shift, d;
    __host__ explicit FastDiv(uint32_t div) : d(div) {
        uint32_t s = 0;
        while ((1ull << s) < div) ++s;
        shift = s;
        mul = (uint32_t)(((1ull << 32) * ((1ull << s) - div)) / div + 1);       // the multiplier without its bit 32
    }
    __device__ __forceinline__ uint32_t div(uint32_t n) const { return (uint32_t)(((uint64_t)__umulhi(n, mul) + n) >> shift); }
};

// ---- element types ------------------------------------------------------------------------------

__device__ __forceinline__ float load_f32(const void* p, int type, long long i) {
    if (type == APB_F32) return static_cast<const float*>(p)[i];
    if (type == APB_BF16) return (float)static_cast<const __bf16*>(p)[i];
    return (float)static_cast<const _Float16*>(p)[i];
}
// one rounding, to nearest even
__device__ __forceinline__ void store_f32(void* p, int type, long long i, float v) {
    if (type == APB_F32) static_cast<float*>(p)[i] = v;
    else if (type == APB_BF16) static_cast<__bf16*>(p)[i] = (__bf16)v;
    else static_cast<_Float16*>(p)[i] = (_Float16)v;
}
__device__ __forceinline__ uint32_t pack2(int type, float a, float b) {
    if (type == APB_BF16) {
        const bf16x2 v = {(__bf16)a, (__bf16)b};
        return __builtin_bit_cast(uint32_t, v);
    }
    const f16x2 v = {(_Float16)a, (_Float16)b};
    return __builtin_bit_cast(uint32_t, v);
}
// Vectors at any address: global memory takes them unaligned, so rows of any stride are read and written alike.
typedef u32x4 u32x4_any __attribute__((aligned(1)));
typedef u32x2 u32x2_any __attribute__((aligned(1)));
__device__ __forceinline__ u32x4 load16_any(const void* p) { return *static_cast<const u32x4_any*>(p); }
__device__ __forceinline__ u32x4 load16_once(const void* p) { return __builtin_nontemporal_load(static_cast<const u32x4_any*>(p)); }
__device__ __forceinline__ void store16_any(void* p, const u32x4& v) { *static_cast<u32x4_any*>(p) = v; }
__device__ __forceinline__ void store8_any(void* p, const u32x2& v) { *static_cast<u32x2_any*>(p) = v; }

__device__ __forceinline__ uint32_t float_bits(float v) { return __builtin_bit_cast(uint32_t, v); }

// four neighbours at element i, of which `count` exist
__device__ __forceinline__ void store4(void* p, int type, long long i, const float (&v)[4], int count) {
    if (count >= 4) {
        if (type == APB_F32)
            store16_any(static_cast<float*>(p) + i, u32x4{float_bits(v[0]), float_bits(v[1]), float_bits(v[2]), float_bits(v[3])});
        else
            store8_any(static_cast<uint16_t*>(p) + i, u32x2{pack2(type, v[0], v[1]), pack2(type, v[2], v[3])});
        return;
    }
#pragma unroll
    for (int q = 0; q < 4; ++q)
        if (q < count) store_f32(p, type, i + q, v[q]);
}

// Eight neighbours of a row as they lie in memory.
template <int TYPE>
struct Eight {
    u32x4 w[TYPE == APB_F32 ? 2 : 1];
};

template <int TYPE, bool ONCE = false>
__device__ __forceinline__ Eight<TYPE> load_eight(const void* X, long long at) {
    Eight<TYPE> v;
    const uint8_t* p = static_cast<const uint8_t*>(X) + at * (TYPE == APB_F32 ? 4 : 2);
    v.w[0] = ONCE ? load16_once(p) : load16_any(p);
    if constexpr (TYPE == APB_F32) v.w[1] = ONCE ? load16_once(p + 16) : load16_any(p + 16);
    return v;
}
// ... of which `have` exist; the others are zero.  ONCE: memory that is read once passes by the caches' other lines.
template <int TYPE, bool ONCE = false>
__device__ __forceinline__ Eight<TYPE> load_some(const void* X, long long at, int have) {
    if (have >= 8) return load_eight<TYPE, ONCE>(X, at);
    Eight<TYPE> v;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        if constexpr (TYPE == APB_F32) {
            v.w[0][q] = q < have ? static_cast<const uint32_t*>(X)[at + q] : 0u;
            v.w[1][q] = q + 4 < have ? static_cast<const uint32_t*>(X)[at + q + 4] : 0u;
        } else {
            const uint16_t* p = static_cast<const uint16_t*>(X) + at + 2 * q;
            v.w[0][q] = (2 * q < have ? (uint32_t)p[0] : 0u) | (2 * q + 1 < have ? (uint32_t)p[1] << 16 : 0u);
        }
    }
    return v;
}

template <int TYPE>
__device__ __forceinline__ void floats(const Eight<TYPE>& x, float (&v)[8]) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        if constexpr (TYPE == APB_F32) {
            const uint32_t a = x.w[0][q], b = x.w[1][q];         // (a bit cast of a vector's element itself takes the first's place)
            v[q] = __builtin_bit_cast(float, a);
            v[4 + q] = __builtin_bit_cast(float, b);
        } else {
            const uint32_t pair = x.w[0][q];
            if constexpr (TYPE == APB_BF16) {
                v[2 * q] = __builtin_bit_cast(float, pair << 16);
                v[2 * q + 1] = __builtin_bit_cast(float, pair & 0xffff0000u);
            } else {
                const f16x2 h = __builtin_bit_cast(f16x2, pair);
                v[2 * q] = (float)h[0];
                v[2 * q + 1] = (float)h[1];
            }
        }
    }
}
// eight neighbours of a row, of which `have` exist
template <int TYPE>
__device__ __forceinline__ void store8(void* X, long long at, int have, const float (&v)[8]) {
    if (have >= 8 && TYPE != APB_F32) {
        store16_any(static_cast<uint16_t*>(X) + at,
                    u32x4{pack2(TYPE, v[0], v[1]), pack2(TYPE, v[2], v[3]), pack2(TYPE, v[4], v[5]), pack2(TYPE, v[6], v[7])});
        return;
    }
    const float a[4] = {v[0], v[1], v[2], v[3]}, b[4] = {v[4], v[5], v[6], v[7]};
    store4(X, TYPE, at, a, have);
    store4(X, TYPE, at + 4, b, have - 4);
}

// ---- the scale of a block -------------------------------------------------------------------------

// from the largest magnitude's float bits (sign cleared): e + 127 of the block, 255 if it is not finite.  floor(log2) of a
// subnormal is below -126, so its e is -127 whatever it is.
__device__ __forceinline__ uint32_t scale_code(uint32_t top) {
    const uint32_t ex = top >> 23;
    return ex >= 255u ? 255u : ex > 2u ? ex - 2u : 0u;
}
// 2^e as a float (2^-127 is subnormal); NaN for 255
__device__ __forceinline__ float scale_value(uint32_t code) {
    return __builtin_bit_cast(float, code == 0u ? 0x00400000u : code == 255u ? 0x7fc00000u : code << 23);
}

typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

// The largest magnitude of eight values as the bits of a float (bits without their sign order like magnitudes; a NaN is above
// infinity).
template <int TYPE>
__device__ __forceinline__ uint32_t top_bits(const Eight<TYPE>& v) {
    if constexpr (TYPE == APB_F32) {
        uint32_t top = 0;
#pragma unroll
        for (int q = 0; q < 8; ++q) top = max(top, v.w[q / 4][q & 3] & 0x7fffffffu);
        return top;
    } else {
        u16x2 top = {0, 0};
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const uint32_t pair = v.w[0][q] & 0x7fff7fffu;
            top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, pair));
        }
        const uint16_t most = max(top[0], top[1]);
        if constexpr (TYPE == APB_BF16) return (uint32_t)most << 16;
        else return float_bits((float)__builtin_bit_cast(_Float16, most));
    }
}
// the larger of it among the four lanes of a block of 32
__device__ __forceinline__ uint32_t top_of_four(uint32_t v) {
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xb1, 0xf, 0xf, true));      // lanes 1 0 3 2
    return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4e, 0xf, 0xf, true));   // lanes 2 3 0 1
}

// Eight values -> eight nibbles.  The conversion divides by the power of two whose float has the scale code as its exponent and
// rounds once, to nearest even; that holds for codes 0 and 252 as well.
template <int TYPE, int B>
__device__ __forceinline__ uint32_t encode_pair(uint32_t w, const Eight<TYPE>& v, float scale) {
    if constexpr (TYPE == APB_F32) {
        const uint32_t a = v.w[B / 2][2 * B & 3], c = v.w[B / 2][(2 * B & 3) + 1];
        return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, __builtin_bit_cast(float, a), __builtin_bit_cast(float, c), scale, B);
    } else {
        const uint32_t pair = v.w[0][B];
        if constexpr (TYPE == APB_BF16) return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, pair), scale, B);
        else return __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(w, __builtin_bit_cast(f16x2, pair), scale, B);
    }
}
template <int TYPE>
__device__ __forceinline__ uint32_t encode8(const Eight<TYPE>& v, uint32_t code) {
    const float scale = __builtin_bit_cast(float, code << 23);
    uint32_t w = encode_pair<TYPE, 0>(0u, v, scale);
    w = encode_pair<TYPE, 1>(w, v, scale);
    w = encode_pair<TYPE, 2>(w, v, scale);
    w = encode_pair<TYPE, 3>(w, v, scale);
    return code == 255u ? 0u : w;
}

// ---- matrix instructions ----------------------------------------------------------------------------

// (the instruction reads the low four words of a 4-bit operand)
__device__ __forceinline__ i32x8 operand(const u32x4& w) { return i32x8{(int)w[0], (int)w[1], (int)w[2], (int)w[3], 0, 0, 0, 0}; }

// Products of 4-bit operands, 32 x 32 x 64 and 16 x 16 x 128; S: which byte of a scale word counts.  Sums within a block of 32 are
// exact, each block is added with one rounding.
template <int S>
__device__ __forceinline__ f32x16 mfma32(const u32x4& a, const u32x4& b, const f32x16& c, int sa, int sb) {
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(operand(a), operand(b), c, 4, 4, S, sa, S, sb);
}
template <int S>
__device__ __forceinline__ f32x4 mfma16(const u32x4& a, const u32x4& b, const f32x4& c, int sa, int sb) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(operand(a), operand(b), c, 4, 4, S, sa, S, sb);
}

// ---- loads to LDS --------------------------------------------------------------------------------------

// A load of 16 (4) bytes per lane that goes to LDS, to 16 (4) bytes per lane from `to` on, without passing through registers.  Written
// out because several segments can be under way: the compiler would wait for all of them before each read of LDS.  `to` is asked for in
// m0, where the instruction looks for it, so the compiler knows what m0 holds.  Whoever reads what arrived waits for it first
// (s_waitcnt vmcnt).
__device__ __forceinline__ void load16_to_lds(uint32_t to, const void* base, uint32_t offset) {
    asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"{m0}"(to), "v"(offset), "s"(base));
}
__device__ __forceinline__ void load4_to_lds(uint32_t to, const void* base, uint32_t offset) {
    asm volatile("s_nop 0\n\tglobal_load_lds_dword %1, %2" ::"{m0}"(to), "v"(offset), "s"(base));
}
__device__ __forceinline__ uint32_t lds_address(const void* p) {
    return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void*)p;
}
template <class T>
__device__ __forceinline__ T lds_load(uint32_t at) { return *(__attribute__((address_space(3))) const T*)(uintptr_t)at; }
template <class T>
__device__ __forceinline__ void lds_store(uint32_t at, const T& v) { *(__attribute__((address_space(3))) T*)(uintptr_t)at = v; }

// ---- from accumulators to rows -----------------------------------------------------------------------------

// Bytes of LDS that a wave needs to write its tile of 32 * F x 32 * F outputs (256 of float32 a row: in two halves).
template <int F>
constexpr int kTileLds = F == 4 ? 32768 : F * F * 4096;

// Four sums of an accumulator.  With F == 4 the accumulators fill the second half of the registers and are fetched from there where
// they are needed, and not all of them ahead of a branch.
template <int F>
__device__ __forceinline__ f32x4 four_sums(const f32x16& a, int i) {
    f32x4 v;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const float x = a[i + q];
        float y = x;
        if constexpr (F == 4) asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(y) : "a"(x));
        v[q] = y;
    }
    return v;
}

// Before the first of them: the compiler does not see that four_sums() reads what a matrix instruction wrote (32 cycles, for 8 passes
// of four).
template <int F>
__device__ __forceinline__ void settled() {
    if constexpr (F == 4) asm volatile("s_nop 15\n\ts_nop 15");
}

// SUMS(x, y, q): the lane's four outputs of row 32 x + r, columns 32 y + 8 q + 4 h + 0..3.  HALF: the tile has 16 * F columns.
template <int TYPE, int F, bool HALF, class SUMS>
__device__ __forceinline__ void store_tile_as(const SUMS& sums, uint32_t lds, void* out, long long first, long long ld, int rows,
                                              long long col, int cols) {
    constexpr int kSize = TYPE == APB_F32 ? 4 : 2, kEach = 16 / kSize;
    constexpr int kChunks = (HALF ? 1 : 2) * F * kSize, kPitch = 16 * kChunks;            // 16-byte chunks of a row
    constexpr int kX = F * 32 * kPitch <= kTileLds<F> ? F : F / 2;                // groups of 32 rows at a time
    constexpr int kStepRows = kWave / kChunks, kSteps = 32 * kX / kStepRows;
    constexpr int kAhead = kSteps < 8 ? kSteps : 8;
    // Where chunk c of a row is: the chunks are permuted by the row's number, so that lanes of many rows meet every bank once; 32
    // rows further the permutation is the same.  (The addresses of a row's chunks differ in bits that its first one has not.)
    auto first_of = [&](int row) {
        constexpr int kLine = kChunks < 16 ? 16 / kChunks : 1;              // rows that share the 64 banks
        return lds + row * kPitch + 16 * (row / kLine & (kChunks < 16 ? kChunks - 1 : 15));
    };
    const int lane = threadIdx.x & (kWave - 1), r = lane & 31, h = lane >> 5;
    const int chunk = lane & (kChunks - 1), sub = lane / kChunks;
    const int have = cols - chunk * kEach;
    const uint32_t mine = TYPE == APB_F32 ? first_of(r) ^ 16 * h : first_of(r) + 8 * h;
    const long long row_bytes = ld * kSize;
    uint8_t* to = static_cast<uint8_t*>(out) + (first + sub) * row_bytes + (col + chunk * kEach) * kSize;
#pragma unroll
    for (int x0 = 0; x0 < F; x0 += kX) {
#pragma unroll
        for (int x = x0; x < x0 + kX; ++x)
#pragma unroll
            for (int y = 0; y < (HALF ? (F + 1) / 2 : F); ++y)
#pragma unroll
                for (int q = 0; q < (HALF && F == 1 ? 2 : 4); ++q) {
                    const f32x4 a = sums(x, y, q);
                    const uint32_t rows_on = 32 * (x - x0) * kPitch;
                    if constexpr (TYPE == APB_F32)
                        lds_store((mine ^ 16 * (8 * y + 2 * q)) + rows_on, a);
                    else
                        lds_store((mine ^ 16 * (4 * y + q)) + rows_on,
                                  u32x2{pack2(TYPE, a[0], a[1]), pack2(TYPE, a[2], a[3])});
                }
        // (the wave's own writes and reads of LDS stay in this order)
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        const int there = min(rows - 32 * x0, 32 * kX);
        const long long step_bytes = kStepRows * row_bytes;
        uint8_t* p = to;
#pragma unroll 1
        for (int i = 0; i < there; i += kAhead * kStepRows) {
            u32x4 v[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) v[u] = lds_load<u32x4>(first_of(i + u * kStepRows + sub) ^ 16 * chunk);
#pragma unroll
            for (int u = 0; u < kAhead; ++u, p += step_bytes)
                if (i + u * kStepRows + sub < there && have >= kEach) store16_any(p, v[u]);
        }
        p = to;
        if (have > 0 && have < kEach)                                        // the last columns, one by one
#pragma unroll 1
            for (int row = sub; row < there; row += kStepRows, p += step_bytes)
#pragma unroll 1
                for (int q = 0; q < have; ++q) {
                    const uint32_t from = (first_of(row) ^ 16 * chunk) + kSize * q;
                    if constexpr (TYPE == APB_F32) reinterpret_cast<uint32_t*>(p)[q] = lds_load<uint32_t>(from);
                    else reinterpret_cast<uint16_t*>(p)[q] = lds_load<uint16_t>(from);
                }
        to += 32 * kX * row_bytes;
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    }
}

// A wave's tile of 32 * F x 32 * F outputs, which its lanes hold as the matrix instruction leaves them (acc[x][y], lane (r, h): of row
// 32 x + r the columns 32 y + 8 q + 4 h + 0..3), written to memory as rows: through LDS of the wave's own, so that a store covers
// whole lines of few rows instead of 16 or 32 bytes of each of 32.  Row i < rows goes to out + (first + i) * ld + col; columns from
// `cols` on are not there.  `lds`: an address, a multiple of 512.  Few
// instructions, each of which a tile fetches to run it once, and eight reads of LDS under way: 256 x 256 in bfloat16 take 2.3 us, in
// a form with a branch on the type at every conversion and a read at a time 7.5.
template <int F>
__device__ __forceinline__ void store_tile(const f32x16 (&acc)[F][F], uint32_t lds, void* out, int type, long long first, long long ld,
                                           int rows, long long col, int cols) {
    settled<F>();
    auto sums = [&](int x, int y, int q) { return four_sums<F>(acc[x][y], 4 * q); };
    if (type == APB_F32) store_tile_as<APB_F32, F, false>(sums, lds, out, first, ld, rows, col, cols);
    else if (type == APB_BF16) store_tile_as<APB_BF16, F, false>(sums, lds, out, first, ld, rows, col, cols);
    else store_tile_as<APB_F16, F, false>(sums, lds, out, first, ld, rows, col, cols);
}

// ---- groups of rows ---------------------------------------------------------------------------------

// Where a workgroup's tile of rows lies: rows row0 .. row0 + rows - 1 of group e; e == E: the rows that belong to no expert;
// rows == 0: no such tile.
struct RowTile {
    int e, row0, rows;
};

// The t-th tile of `tile` rows.  Called by whole waves, all lanes with the same t; each lane takes a group, a prefix sum over
// the lanes counts tiles, 64 groups at a time.
__device__ __forceinline__ RowTile find_row_tile(const int32_t* __restrict__ offsets, int E, int R, int tile, int t) {
    if (offsets == nullptr) {
        const int row0 = t * tile;
        return RowTile{0, row0, min(tile, R - row0)};
    }
    const int lane = threadIdx.x & (kWave - 1);
    int before = 0;
    for (int base = 0; base <= E; base += kWave) {
        const int e = base + lane;
        int a = 0, b = 0;
        if (e <= E) {
            a = min(max(offsets[e], 0), R);
            b = e < E ? max(a, min(offsets[e + 1], R)) : R;
        }
        const int tiles = (b - a + tile - 1) / tile;
        int upto = tiles;
#pragma unroll
        for (int d = 1; d < kWave; d <<= 1) {
            const int v = __shfl_up(upto, d, kWave);
            if (lane >= d) upto += v;
        }
        const unsigned long long hit = __ballot(t < before + upto);
        if (hit) {
            const int src = __builtin_amdgcn_readfirstlane(__ffsll((long long)hit) - 1);
            const int first = __builtin_amdgcn_readlane(before + upto - tiles, src);     // (scalars: what follows is uniform)
            const int ra = __builtin_amdgcn_readlane(a, src), rb = __builtin_amdgcn_readlane(b, src);
            const int row0 = ra + (t - first) * tile;
            return RowTile{base + src, row0, min(tile, rb - row0)};
        }
        before += __builtin_amdgcn_readlane(upto, kWave - 1);
    }
    return RowTile{E, R, 0};
}

// ---- launchers (one translation unit each) -----------------------------------------------------------

int launch_mx4_quantize(const void* X, int type, long long row_stride, long long col_stride, int rows_in,
                        const int32_t* rows_from, int rows, int K, void* mx, hipStream_t s);
// Few rows: may it run as the one kernel that streams the weights (apb_mx4_few.hip)?
bool mx4_few_applies(const int32_t* offsets, int E, int M, int K);
bool mx4_few_gated_applies(const int32_t* offsets, int E, int M, int N, int K);
int launch_mx4_few(const void* X, int x_type, long long ldx, int rows_in, const int32_t* rows_from, const Mx& W, const int32_t* offsets,
                   int E, int M, int N, int K, int type, void* Y, long long ldy, hipStream_t s);
int launch_mx4_few(const Mx& A, const Mx& W, const int32_t* offsets, int E, int M, int N, int K, int type, void* Y, long long ldy, hipStream_t s);
int launch_mx4_gemm(const Mx& A, const Mx& B, const int32_t* offsets, int E, int M, int N, int type, void* Y, long long ldy,
                    hipStream_t s);
// The same two with both projections of a gated block and its activation (N: of either projection).
int launch_mx4_few_gated(const void* X, int x_type, long long ldx, int rows_in, const int32_t* rows_from, const Mx& W,
                         const int32_t* offsets, int E, int M, int N, int K, int activation, int type, void* Y, long long ldy,
                         hipStream_t s);
int launch_mx4_few_gated(const Mx& A, const Mx& W, const int32_t* offsets, int E, int M, int N, int K, int activation, int type, void* Y,
                         long long ldy, hipStream_t s);

}  // namespace apb
