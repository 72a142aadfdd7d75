// Gradients of the 4-bit product at its quantized operands:
//      dX[m, k] = sum_n G[m, n] W^[n, k]          dW[n, k] = sum_m G[m, n] X^[m, k]
// Both sum over the ROWS of a 4-bit matrix, across its blocks, so its scales cannot ride along in the matrix instruction; its
// values, products of a level and a power of two, are exact in bfloat16, and the bfloat16 matrix instruction multiplies them
// with G.  A bfloat16 G is taken as it is; a float16 G is the sum of two bfloat16 values, a float32 G of three (each part takes
// the next 8 bits), and each part goes through the matrix cores, so no bit of G is dropped.
// Bound by the matrix cores and their power: dX and dW of 8192^3 in bfloat16, one call behind another, take 896 and 914 us (1230 and
// 1200 TFLOP/s; a large bfloat16 product of the library reaches 1400), of 4096^3 123 and 132.  With nothing but the first pass's
// operands, from the caches, the former is 3 % faster, so memory is not what it waits for.  Of 4096^3 with a float32 G 537 and 509 us,
// a float16 G 342 and 375: three and two times the products, a split that every tile repeats, tiles of 128 a side.
#include <utility>

#include "apb_mx4.h"

namespace apb {
namespace {

constexpr int kGroup = 256;                   // threads that make a tile: four waves
constexpr int kStep = kMx4Pass;               // summed over per pass: a line of 128 bytes of bfloat16 in LDS

template <int TYPE>
struct Parts {
    static constexpr int n = TYPE == APB_F32 ? 3 : TYPE == APB_F16 ? 2 : 1;
};

// LDS tiles: `row` (an output index) has kStep bfloat16 values, 128 bytes, in chunks of eight.  The chunks of a row are permuted by
// the row's number so that neither eight lanes that write two chunks of four rows some rows apart nor eight that read the same chunk
// of successive rows meet a bank twice; 32 rows further the permutation is the same.
constexpr int kRowBytes = 2 * kStep;
__device__ __forceinline__ uint32_t lds_at(int row, int chunk) { return row * kRowBytes + 16 * (chunk ^ ((row + 2 * (row >> 3)) & 7)); }

// N words at any address.
template <int N>
struct Words {
    uint32_t w[N];
};
template <int N, class Pointer>
__device__ __forceinline__ Words<N> load_words(Pointer p) {
    typedef uint32_t Vector __attribute__((ext_vector_type(N > 4 ? 4 : N)));
    typedef Vector Any __attribute__((aligned(1)));
    Words<N> v;
#pragma unroll
    for (int i = 0; i < N; i += 4) {
        const Vector x = *(__attribute__((address_space(1))) const Any*)(p + 4 * i);
#pragma unroll
        for (int q = 0; q < (N > 4 ? 4 : N); ++q) {
            if constexpr (N == 1) v.w[0] = __builtin_bit_cast(uint32_t, x);
            else v.w[i + q] = x[q];
        }
    }
    return v;
}
// `count` neighbours of a row of G from element `at` on, of which `have` exist; the others are zero
template <int TYPE, int COUNT>
__device__ __forceinline__ Words<COUNT * (TYPE == APB_F32 ? 4 : 2) / 4> load_some_words(const void* G, long long at, int have) {
    constexpr int kSize = TYPE == APB_F32 ? 4 : 2, N = COUNT * kSize / 4;
    if (have >= COUNT) return load_words<N>((__attribute__((address_space(1))) const uint8_t*)G + at * kSize);
    Words<N> v;
#pragma unroll
    for (int q = 0; q < N; ++q) {
        if constexpr (TYPE == APB_F32) {
            v.w[q] = q < have ? static_cast<const uint32_t*>(G)[at + q] : 0u;
        } else {
            const uint16_t* p = static_cast<const uint16_t*>(G) + at + 2 * q;
            v.w[q] = (2 * q < have ? (uint32_t)p[0] : 0u) | (2 * q + 1 < have ? (uint32_t)p[1] << 16 : 0u);
        }
    }
    return v;
}

// The bfloat16 parts of 2 * N neighbours, two to a word: each part takes the leading 8 significant bits of what is left (cut off,
// so that no part is larger than the value and none overflows).  Of a float32 value the second part is taken 2^7 and the third 2^15
// times as large, no larger than the value yet, and the parts' sums are kept apart until the end: bfloat16 ends at 2^-133, the value
// at 2^-149.  So nothing is lost of values from 2^-125 on, and less than 2^-148 of smaller ones.
constexpr float kSecond = 128.0f, kThird = 256.0f;               // ... than the part before
template <int TYPE, int N>
__device__ __forceinline__ void split(const Words<N * (TYPE == APB_F32 ? 2 : 1)>& v, Words<N> (&part)[Parts<TYPE>::n]) {
    if constexpr (TYPE == APB_BF16) {
        part[0] = v;
    } else {
#pragma unroll
        for (int q = 0; q < N; ++q) {
            float x[2];
            if constexpr (TYPE == APB_F32) {
                x[0] = __builtin_bit_cast(float, v.w[2 * q]);
                x[1] = __builtin_bit_cast(float, v.w[2 * q + 1]);
            } else {
                const f16x2 p = __builtin_bit_cast(f16x2, v.w[q]);
                x[0] = (float)p[0];
                x[1] = (float)p[1];
            }
#pragma unroll
            for (int p = 0; p < Parts<TYPE>::n; ++p) {
                uint32_t bits[2];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    bits[i] = float_bits(x[i]);
                    x[i] -= __builtin_bit_cast(float, bits[i] & 0xffff0000u);
                    if (TYPE == APB_F32) x[i] *= p == 0 ? kSecond : kThird;
                    // an infinity is its own first part; a NaN leaves a NaN
                    if (p == 0 && (bits[i] & 0x7fffffffu) == 0x7f800000u) x[i] = 0.0f;
                }
                part[p].w[q] = __builtin_amdgcn_perm(bits[1], bits[0], 0x07060302u);
            }
        }
    }
}

// f(0), f(1), ... f(N - 1), each with its number as a constant
template <class F, int... I>
__device__ __forceinline__ void each_of(F&& f, std::integer_sequence<int, I...>) { (f(std::integral_constant<int, I>{}), ...); }
template <int N, class F>
__device__ __forceinline__ void each(F&& f) { each_of(f, std::make_integer_sequence<int, N>{}); }

// One row of an 8 x 2N transpose: in[c] holds the values of 2N output indices at summation index c, two to a word; this is output
// index i's eight.
template <int N>
__device__ __forceinline__ u32x4 transposed(const Words<N> (&in)[8], int i) {
    u32x4 w;
#pragma unroll
    for (int q = 0; q < 4; ++q)
        w[q] = __builtin_amdgcn_perm(in[2 * q + 1].w[i / 2], in[2 * q].w[i / 2], i & 1 ? 0x07060302u : 0x05040100u);
    return w;
}

typedef __attribute__((address_space(1))) const uint8_t* Bytes;
// Where a lane loads from, as the load instruction has it: a base in scalar registers, which the compiler takes as it is instead of
// folding lane offsets into it, and a 32-bit offset, which it does not widen ahead of the loop.
__device__ __forceinline__ Bytes at_lane(Bytes& base, uint32_t& offset) {
    asm volatile("" : "+s"(base), "+v"(offset));
    return base + offset;
}

// All of this wave's reads and writes of LDS are done; then so are everybody's.  (Loads to registers stay under way.)
__device__ __forceinline__ void lds_ready() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// OUT[i, j] = sum_c P[i, c] Q^[c, j] over the 4-bit matrix Q's rows c.
//   WEIGHT = false: P = G, i = row m of the group, c = n.     WEIGHT = true: P = G^T, i = n, c = row m of the group.
// A workgroup makes a tile of 64 * F x 64 * F outputs, a wave 32 * F x 32 * F.  A pass sums over 64 indices in four steps of 16:
// while the matrix cores work on one buffer of LDS, the next pass's operands, loaded to registers a pass earlier, are brought into
// the other one as rows of output indices: 8 x 8 blocks transposed in registers, 4-bit values widened to bfloat16.  That work is
// cut into small tasks, and after every matrix instruction of the first three steps comes one of them and at most one read of the
// next step's operands, so that nothing waits behind them; the barrier stands before the fourth step, under which the next pass's
// first operands are read.
// Where there are few tiles and many passes, `slices` workgroups share a tile's passes: each writes its sums as a matrix of its own
// in the workspace, and k_mx4_join adds them up in order.
// Where there are few tiles, GROUPS = 2 groups of four waves work on one, each with buffers of its own and every second pass, and
// add up at the end, the first group's sums first.
template <int TYPE, bool WEIGHT, int F, int GROUPS>
__global__ __launch_bounds__(kGroup* GROUPS, F * Parts<TYPE>::n <= 2 || GROUPS == 2 ? 2 : 1) void
k_mx4_backward(const void* __restrict__ G, long long ldg, Mx Q, const int32_t* __restrict__ offsets, int E, int M, int N, int K,
               int slices, int type, void* __restrict__ out, long long ldo) {
    constexpr int NP = Parts<TYPE>::n;
    constexpr int kTile = 64 * F;
    constexpr int kPart = kTile * kRowBytes, kBuffer = (NP + 1) * kPart;      // parts of P, then Q
    __shared__ __align__(512) uint8_t shared[GROUPS * 2 * kBuffer];
    const int j0 = blockIdx.y * kTile;
    int i0, rows_i, c0, rows_c, out_row;                         // outputs, summation range (rows of Q from c0 on)
    int g_row;                                                   // row of G that belongs to i0 (or to c0, WEIGHT)
    if (WEIGHT) {
        const int e = blockIdx.z / slices;
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
    // this workgroup's share of the passes
    const int slice = blockIdx.z % slices;
    int g_col = WEIGHT ? i0 : 0;
    if (slices > 1) {
        const int passes = (rows_c + kStep - 1) / kStep;
        const int from = (int)((long long)passes * slice / slices) * kStep, upto = (int)((long long)passes * (slice + 1) / slices) * kStep;
        c0 += from;
        (WEIGHT ? g_row : g_col) += from;
        rows_c = min(rows_c, upto) - from;
        out = static_cast<float*>(out) + (size_t)slice * (WEIGHT ? (size_t)E * N : M) * K;
    }
    const int group = GROUPS == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / kGroup);
    const int tid = threadIdx.x & (kGroup - 1), lane = tid & (kWave - 1), wave = tid / kWave;
    uint8_t* lds = shared + group * 2 * kBuffer;
    const int wi = (wave >> 1) * 32 * F, wj = (wave & 1) * 32 * F;
    const int r = lane & 31, h = lane >> 5;
    // who brings in what: blocks of eight summation indices x W output indices of either operand, as many as there are threads;
    // of G as it lies in memory for dX, pieces of eight summation indices of kPieces rows
    constexpr int kSize = TYPE == APB_F32 ? 4 : 2, W = 2 * F, kPieces = 2 * F;
    const int block = W * ((tid & 3) | (tid >> 1 & 28)), chunk = (tid >> 2 & 1) | tid >> 6 << 1;
    const int line = tid >> 3, piece = tid & 7;
    const uint32_t q_pitch = (uint32_t)Q.segs * kMxSegBytes;

    // where a thread loads from: a scalar base and an offset of its own
    const Bytes g_base = (Bytes)G + ((long long)g_row * ldg + g_col) * kSize;
    const Bytes q_base = (Bytes)Q.codes + (size_t)c0 * q_pitch + j0 / 2;
    const Bytes s_base = (Bytes)Q.scales + ((size_t)(j0 / kMxSeg) * Q.rows + c0) * 8 + j0 % kMxSeg / kMxBlock;
    uint32_t q_at = 8 * chunk * q_pitch + block / 2, s_at = 64 * chunk + block / kMxBlock;
    const uint32_t g_pitch = (uint32_t)ldg * kSize;
    uint32_t g_at[WEIGHT ? 1 : kPieces];
    if constexpr (WEIGHT) {
        g_at[0] = 8 * chunk * g_pitch + min(block, N - W - i0) * kSize;               // (whole blocks: what is not there is not stored)
    } else {
#pragma unroll
        for (int u = 0; u < kPieces; ++u) g_at[u] = min(u * 32 + line, rows_i - 1) * g_pitch + 8 * piece * kSize;
    }
    // where it writes in LDS, and where it reads the operands of a step: in the first buffer, then by turns in either
    const uint32_t lds0 = lds_address(shared) + group * 2 * kBuffer;
    uint32_t to[W], g_to = lds0 + lds_at(line, piece), p_from[kStep / 16], q_from[kStep / 16];
#pragma unroll
    for (int i = 0; i < W; ++i) to[i] = lds0 + lds_at(block + i, chunk);
#pragma unroll
    for (int ks = 0; ks < kStep / 16; ++ks) {
        p_from[ks] = lds0 + lds_at(wi + r, 2 * ks + h);
        q_from[ks] = lds0 + NP * kPart + lds_at(wj + r, 2 * ks + h);
    }

    // The parts of a float32 G have sums of their own, for they are scaled.  And a matrix instruction waits for the one before it on
    // the same sums: a lone tile of 32 x 32 has several, one for each part of G or for every second step.
    constexpr int kSums = NP == 3 ? 3 : F > 1 ? 1 : 2;
    f32x16 sums[kSums][F][F];
#pragma unroll
    for (int n = 0; n < kSums; ++n)
#pragma unroll
        for (int x = 0; x < F; ++x)
#pragma unroll
            for (int y = 0; y < F; ++y)
#pragma unroll
                for (int q = 0; q < 16; ++q) sums[n][x][y][q] = 0.0f;
    f32x16(&acc)[F][F] = sums[0];

    constexpr int kGCount = WEIGHT ? 8 : kPieces, kGWords = (WEIGHT ? W : 8) * kSize / 4;
    Words<kGWords> g[kGCount];
    uint32_t code[8], scale[8];
    Words<W / 2> q_wide[8], g_part[NP][8];
    // the tasks: load, widen or split, store
    Bytes g_next, q_next, s_next;                                // of the pass to load
    auto aim = [&](int c) {
        g_next = g_base + (WEIGHT ? (size_t)c * g_pitch : (size_t)c * kSize);
        q_next = q_base + (size_t)c * q_pitch;
        s_next = s_base + (size_t)c * 8;
    };
    auto load_g = [&](int u) {
        g[u] = load_words<kGWords>(at_lane(g_next, g_at[WEIGHT ? 0 : u]));
        if constexpr (WEIGHT) g_next += g_pitch;
    };
    auto codes_at = [&](Bytes p) -> uint32_t {                   // W of them
        if constexpr (W == 8) return *(__attribute__((address_space(1))) const uint32_t*)p;
        else if constexpr (W == 4) return *(__attribute__((address_space(1))) const uint16_t*)p;
        else return *p;
    };
    auto load_q = [&](int u) {
        code[u] = codes_at(at_lane(q_next, q_at));
        scale[u] = at_lane(s_next, s_at)[8 * u];
        q_next += q_pitch;
    };
    auto split_g = [&](int u) {
        if constexpr (WEIGHT) {
            Words<W / 2> v[NP];
            split<TYPE, W / 2>(g[u], v);
#pragma unroll
            for (int p = 0; p < NP; ++p) g_part[p][u] = v[p];
        } else {
            Words<4> v[NP];
            split<TYPE, 4>(g[u], v);
#pragma unroll
            for (int p = 0; p < NP; ++p)
                lds_store(g_to + p * kPart + u * 32 * kRowBytes, u32x4{v[p].w[0], v[p].w[1], v[p].w[2], v[p].w[3]});
        }
    };
    auto store_g = [&](int i) {
#pragma unroll
        for (int p = 0; p < NP; ++p) lds_store(to[i] + p * kPart, transposed(g_part[p], i));
    };
    auto widen_q = [&](int u) {
        // (the conversion takes the scale as a float's exponent: every code is right as it is, 0 and NaN's 255 too)
        const float s = __builtin_bit_cast(float, scale[u] << 23);
        q_wide[u].w[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code[u], s, 0));
        if constexpr (W >= 4) q_wide[u].w[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code[u], s, 1));
        if constexpr (W >= 8) {
            q_wide[u].w[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code[u], s, 2));
            q_wide[u].w[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code[u], s, 3));
        }
    };
    auto store_q = [&](int i) { lds_store(to[i] + NP * kPart, transposed(q_wide, i)); };
    constexpr int kTasksQ = 16 + W, kTasks = kTasksQ + 2 * kGCount + (WEIGHT ? W : 0);
    // task k of bringing in one pass and loading the one aimed at into its registers
    auto task = [&](auto number) {
        constexpr int k = number.value, m = k - kTasksQ;
        if constexpr (k < 8) widen_q(k);
        else if constexpr (k < 16) load_q(k - 8);
        else if constexpr (k < kTasksQ) store_q(k - 16);
        else if constexpr (m < kGCount) split_g(m);
        else if constexpr (m < kTasks - kTasksQ - kGCount) store_g(m - kGCount);
        else load_g(k - (kTasks - kGCount));
    };
    // what a pass in registers has of its first `skip` summation indices becomes zero
    auto leave_out = [&](int skip) {
#pragma unroll
        for (int u = 0; u < 8; ++u)
            if (8 * chunk + u < skip) code[u] = scale[u] = 0u;
#pragma unroll
        for (int u = 0; u < kGCount; ++u)
#pragma unroll
            for (int q = 0; q < kGWords; ++q) {
                if constexpr (WEIGHT) {
                    if (8 * chunk + u < skip) g[u].w[q] = 0u;
                } else if constexpr (TYPE == APB_F32) {
                    if (8 * piece + q < skip) g[u].w[q] = 0u;
                } else {
                    if (8 * piece + 2 * q < skip) g[u].w[q] &= 0xffff0000u;
                    if (8 * piece + 2 * q + 1 < skip) g[u].w[q] = 0u;
                }
            }
    };

    bf16x8 fp[2][NP * F], fq[2][F];
    auto read = [&](int ks, int set, int i) {
        if (i < F) fq[set][i] = lds_load<bf16x8>(q_from[ks] + 32 * i * kRowBytes);
        else fp[set][i - F] = lds_load<bf16x8>(p_from[ks] + (i - F) / F * kPart + (i - F) % F * 32 * kRowBytes);
    };
    auto multiply = [&](int ks, int i) {                         // i: part, x, y
        const int x = i / F % F, y = i % F, set = ks & 1, n = kSums == 1 ? 0 : NP > 1 ? i / (F * F) : ks >> 1;
        sums[n][x][y] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fq[set][y], fp[set][i / F], sums[n][x][y], 0, 0, 0);
    };
    constexpr int kReads = F + NP * F, kProducts = NP * F * F;   // of a step
    constexpr int kLast = kStep / 16 - 1;
    // Loads without checks need whole passes and whole blocks of G.  The last pass is the last 64 indices: of those that it shares
    // with the one before it takes none.
    if (rows_c >= kStep && (!WEIGHT || rows_i == kTile || N % W == 0)) {
        const int passes = (rows_c + kStep - 1) / kStep, rounds = (passes + GROUPS - 1) / GROUPS;
        // of this group's n-th pass: where it begins, and how many of its indices others have
        auto begin = [&](int n) { return min((n * GROUPS + group) * kStep, rows_c - kStep); };
        auto known = [&](int n) { return min((n * GROUPS + group) * kStep - begin(n), kStep); };
        aim(begin(0));
        each<8>([&](auto u) { load_q(u.value); });
        each<kGCount>([&](auto u) { load_g(u.value); });
        if (known(0) > 0) leave_out(known(0));
        aim(begin(1));
        each<kTasks>([&](auto k) { task(k); });
        lds_ready();
        each<kReads>([&](auto i) { read(0, 0, i.value); });
        int turn = kBuffer;                                      // from one buffer to the other: writes are one ahead of reads
#pragma unroll
        for (int i = 0; i < W; ++i) to[i] += turn;
        g_to += turn;
        // A round multiplies one pass of the group's, brings in the next one and loads the one behind it.  (Two passes ahead in registers,
        // by turns in two copies of this loop, cost more in fetching instructions than they saved in waiting: 333 x 1000 x 517 24.2 us
        // instead of 22.5.)
        for (int round = 0; round < rounds; ++round) {
            if (round + 2 == rounds && known(round + 1) > 0) leave_out(known(round + 1));
            aim(begin(round + 2));                               // (beyond the last pass: that again, unread)
            each<kStep / 16>([&](auto step) {
                constexpr int ks = step.value;
                if constexpr (ks == kLast) {
                    lds_ready();
                    p_from[0] += turn;
                    q_from[0] += turn;
                }
                __builtin_amdgcn_sched_barrier(0);
                each<kProducts>([&](auto product) {
                    constexpr int i = product.value;
                    multiply(ks, i);
                    constexpr int r0 = i * kReads / kProducts, r1 = (i + 1) * kReads / kProducts;
                    each<r1 - r0>([&](auto j) { read((ks + 1) & kLast, 1 - (ks & 1), r0 + j.value); });
                    if constexpr (ks < kLast) {
                        constexpr int slot = ks * kProducts + i, kSlots = kLast * kProducts;
                        constexpr int t0 = slot * kTasks / kSlots, t1 = (slot + 1) * kTasks / kSlots;
                        each<t1 - t0>([&](auto j) { task(std::integral_constant<int, t0 + decltype(j)::value>{}); });
                    }
                    __builtin_amdgcn_sched_barrier(0);
                });
            });
#pragma unroll
            for (int ks = 1; ks < kStep / 16; ++ks) {
                p_from[ks] += turn;
                q_from[ks] += turn;
            }
            turn = -turn;
#pragma unroll
            for (int i = 0; i < W; ++i) to[i] += turn;
            g_to += turn;
        }
        rows_c = 0;
    }
    // few summation indices, or blocks of G that N cuts: what lies outside G and Q is zero
    for (int round = 0; round * GROUPS * kStep < rows_c; ++round) {
        const int c = (round * GROUPS + group) * kStep;
#pragma unroll
        for (int u = 0; u < kGCount; ++u) {
            if constexpr (WEIGHT) {
                const int cc = c + 8 * chunk + u;
                g[u] = load_some_words<TYPE, W>(G, (long long)(g_row + cc) * ldg + i0 + block, cc < rows_c ? rows_i - block : 0);
            } else {
                const int row = min(u * 32 + line, rows_i - 1);
                g[u] = load_some_words<TYPE, 8>(G, (long long)(g_row + row) * ldg + g_col + c + 8 * piece, rows_c - c - 8 * piece);
            }
        }
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            const int cc = c + 8 * chunk + u, row = min(cc, rows_c - 1);
            code[u] = codes_at(q_base + (size_t)row * q_pitch + block / 2);
            scale[u] = s_base[(size_t)row * 8 + block / kMxBlock];
            if (cc >= rows_c) code[u] = scale[u] = 0u;
        }
        each<kGCount>([&](auto u) { split_g(u.value); });
        each<8>([&](auto u) { widen_q(u.value); });
        each<W>([&](auto i) {
            if constexpr (WEIGHT) store_g(i.value);
            store_q(i.value);
        });
        lds_ready();
#pragma unroll
        for (int ks = 0; ks < kStep / 16; ++ks) {
#pragma unroll
            for (int i = 0; i < kReads; ++i) read(ks, 0, i);
#pragma unroll
            for (int i = 0; i < kProducts; ++i) multiply(2 * (ks & 1), i);
        }
        lds_ready();
    }
#pragma unroll
    for (int n = 1; n < kSums; ++n)
#pragma unroll
        for (int x = 0; x < F; ++x)
#pragma unroll
            for (int y = 0; y < F; ++y)
#pragma unroll
                for (int q = 0; q < 16; ++q)
                    acc[x][y][q] = fmaf(sums[n][x][y][q], NP < 3 ? 1.0f : n == 1 ? 1.0f / kSecond : 1.0f / (kSecond * kThird), acc[x][y][q]);
    lds_ready();
    if constexpr (GROUPS == 2) {
        static_assert(F * F * 16 * 4 * kGroup <= 2 * kBuffer, "a group's sums fit its buffers");
        float* theirs = reinterpret_cast<float*>(shared) + tid * 4;
#pragma unroll
        for (int i = 0; i < F * F * 4; ++i) {
            const f32x16& a = acc[i / 4 / F][i / 4 % F];
            const int q = 4 * (i & 3);
            if (group == 1) *reinterpret_cast<f32x4*>(theirs + i * 4 * kGroup) = f32x4{a[q], a[q + 1], a[q + 2], a[q + 3]};
        }
        lds_ready();
        if (group == 0)
#pragma unroll
            for (int i = 0; i < F * F * 4; ++i) {
                const f32x4 v = *reinterpret_cast<const f32x4*>(theirs + i * 4 * kGroup);
#pragma unroll
                for (int q = 0; q < 4; ++q) acc[i / 4 / F][i / 4 % F][4 * (i & 3) + q] += v[q];
            }
        lds_ready();
        if (group == 1) return;
    }
    // the 4-bit matrix was the first operand: a lane holds four neighbours of an output row
    static_assert(4 * kTileLds<F> <= 2 * kBuffer, "a wave's tile passes through its share of the buffers");
    store_tile<F>(acc, lds_address(lds) + wave * kTileLds<F>, out, type, out_row + wi, ldo, min(32 * F, rows_i - wi), j0 + wj, K - j0 - wj);
}

// out = the sum of the slices' matrices, in their order; four neighbours to a thread
__global__ __launch_bounds__(kGroup) void k_mx4_join(const float* __restrict__ parts, int slices, int rows, int K, FastDiv by_fours, int type,
                                                     void* __restrict__ out, long long ldo) {
    const uint32_t i = blockIdx.x * kGroup + threadIdx.x;
    const int row = (int)by_fours.div(i), k = 4 * (int)(i - (uint32_t)row * by_fours.d);
    if (row >= rows) return;
    const int have = min(K - k, 4);
    const size_t at = (size_t)row * K + k, step = (size_t)rows * K;
    float sum[4] = {};
    constexpr int kAhead = 8;                                    // slices under way
    for (int s = 0; s < slices; s += kAhead) {
        u32x4 v[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const float* p = parts + min(s + u, slices - 1) * step + at;
            if (have == 4) v[u] = load16_any(p);
            else
#pragma unroll
                for (int q = 0; q < 4; ++q) v[u][q] = q < have ? float_bits(p[q]) : 0u;
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const uint32_t bits = v[u][q];
                if (s + u < slices) sum[q] += __builtin_bit_cast(float, bits);
            }
    }
    store4(out, type, (long long)row * ldo + k, sum, have);
}

template <int TYPE, bool WEIGHT, int F, int GROUPS>
void launch_tiles(const Mx4Plan& plan, const void* G, long long ldg, const Mx& Q, const int32_t* offsets, int E, int M, int N, int K, int type,
                  void* out, long long ldo, hipStream_t s) {
    constexpr int kTile = 64 * F;
    const unsigned tiles_i = (unsigned)(WEIGHT ? (N + kTile - 1) / kTile : max_row_tiles(M, E, offsets != nullptr, kTile));
    const dim3 grid(tiles_i, (unsigned)((K + kTile - 1) / kTile), (unsigned)((WEIGHT ? E : 1) * plan.slices));
    hipLaunchKernelGGL((k_mx4_backward<TYPE, WEIGHT, F, GROUPS>), grid, dim3(kGroup * GROUPS), 0, s, G, ldg, Q, offsets, E, M, N, K,
                       plan.slices, type, out, ldo);
}

template <int TYPE, bool WEIGHT>
void launch_type(const Mx4Plan& plan, const void* G, long long ldg, const Mx& Q, const int32_t* offsets, int E, int M, int N, int K, int type,
                 void* out, long long ldo, hipStream_t s) {
    if constexpr (TYPE == APB_BF16) {
        if (plan.f == 4) return launch_tiles<TYPE, WEIGHT, 4, 1>(plan, G, ldg, Q, offsets, E, M, N, K, type, out, ldo, s);
        if (plan.f == 2 && plan.groups == 2) return launch_tiles<TYPE, WEIGHT, 2, 2>(plan, G, ldg, Q, offsets, E, M, N, K, type, out, ldo, s);
    }
    if (plan.f == 2) return launch_tiles<TYPE, WEIGHT, 2, 1>(plan, G, ldg, Q, offsets, E, M, N, K, type, out, ldo, s);
    launch_tiles<TYPE, WEIGHT, 1, 2>(plan, G, ldg, Q, offsets, E, M, N, K, type, out, ldo, s);
}

template <bool WEIGHT>
size_t workspace_bytes(const Mx4Plan& plan, int E, int M, int N, int K) {
    return plan.slices > 1 ? (size_t)plan.slices * (WEIGHT ? (size_t)E * N : M) * K * sizeof(float) : 0;
}

template <bool WEIGHT>
int launch(const void* G, int g_type, long long ldg, const Mx& Q, const int32_t* offsets, int E, int M, int N, int K, int type,
           void* out, long long ldo, void* workspace, size_t bytes, hipStream_t s) {
    Mx4Plan plan = mx4_gradient_plan<WEIGHT>(g_type, offsets != nullptr, E, M, N, K);
    if (!workspace || bytes < workspace_bytes<WEIGHT>(plan, E, M, N, K)) plan = mx4_gradient_plan<WEIGHT>(g_type, offsets != nullptr, E, M, N, K, false);
    const bool split = plan.slices > 1;
    void* to = split ? workspace : out;
    const int to_type = split ? (int)APB_F32 : type;
    const long long ld = split ? K : ldo;
    if (g_type == APB_F32) launch_type<APB_F32, WEIGHT>(plan, G, ldg, Q, offsets, E, M, N, K, to_type, to, ld, s);
    else if (g_type == APB_BF16) launch_type<APB_BF16, WEIGHT>(plan, G, ldg, Q, offsets, E, M, N, K, to_type, to, ld, s);
    else launch_type<APB_F16, WEIGHT>(plan, G, ldg, Q, offsets, E, M, N, K, to_type, to, ld, s);
    if (split) {
        const int rows = WEIGHT ? E * N : M;
        const uint32_t fours = (uint32_t)(K + 3) / 4;
        const unsigned blocks = (unsigned)(((long long)rows * fours + kGroup - 1) / kGroup);
        hipLaunchKernelGGL(k_mx4_join, dim3(blocks), dim3(kGroup), 0, s, static_cast<const float*>(workspace), plan.slices, rows, K,
                           FastDiv(fours), type, out, ldo);
    }
    APB_HIP(hipGetLastError());
    return APB_OK;
}

int check(const void* G, int g_type, long long ldg, const void* Q, const int32_t* offsets, int E, int M, int N, int K, int type,
          const void* out, long long ldo, const void* workspace) {
    if (!G || !Q || !out) return APB_ERR_NULL;
    if (bad_type(g_type) || bad_type(type)) return APB_ERR_TYPE;
    if (bad_product(E, M, N, K, offsets) || ldg < N || ldg > kMxMaxK || ldo < K) return APB_ERR_SHAPE;
    if (!aligned(G, type_size(g_type)) || !aligned(Q, 16) || !aligned(out, type_size(type)) || !aligned(offsets, 4) ||
        !aligned(workspace, 4))
        return APB_ERR_ALIGN;
    return APB_OK;
}

}  // namespace
}  // namespace apb

using namespace apb;

extern "C" {

size_t apb_mx4_backward_input_workspace_bytes(int g_type, int grouped, int E, int M, int N, int K) {
    const int32_t some = 0;
    if (bad_type(g_type) || bad_product(E, M, N, K, grouped ? &some : nullptr)) return 0;
    return workspace_bytes<false>(mx4_gradient_plan<false>(g_type, grouped != 0, E, M, N, K), E, M, N, K);
}

size_t apb_mx4_backward_weight_workspace_bytes(int g_type, int grouped, int E, int M, int N, int K) {
    const int32_t some = 0;
    if (bad_type(g_type) || bad_product(E, M, N, K, grouped ? &some : nullptr)) return 0;
    return workspace_bytes<true>(mx4_gradient_plan<true>(g_type, grouped != 0, E, M, N, K), E, M, N, K);
}

int apb_mx4_backward_input(const void* G, int g_type, long long ldg, const void* W, const int32_t* offsets, int E, int M,
                           int N, int K, int type, void* dX, long long ldx, void* workspace, size_t workspace_bytes, void* stream) {
    const int rc = check(G, g_type, ldg, W, offsets, E, M, N, K, type, dX, ldx, workspace);
    if (rc != APB_OK) return rc;
    return launch<false>(G, g_type, ldg, mx_view(W, E * N, K), offsets, E, M, N, K, type, dX, ldx, workspace, workspace_bytes,
                         reinterpret_cast<hipStream_t>(stream));
}

int apb_mx4_backward_weight(const void* G, int g_type, long long ldg, const void* X, const int32_t* offsets, int E, int M,
                            int N, int K, int type, void* dW, long long ldw, void* workspace, size_t workspace_bytes, void* stream) {
    const int rc = check(G, g_type, ldg, X, offsets, E, M, N, K, type, dW, ldw, workspace);
    if (rc != APB_OK) return rc;
    return launch<true>(G, g_type, ldg, mx_view(X, M, K), offsets, E, M, N, K, type, dW, ldw, workspace, workspace_bytes,
                        reinterpret_cast<hipStream_t>(stream));
}

}  // extern "C"
