// Routing tokens to experts: the k largest logits of a token, softmax over them, the slots (token, choice) ordered by expert;
// joining the experts' results; and both gradients.
//
// Routing is a few short kernels, each bound by its launch and a chain of dependent steps: 16384 tokens, 8 of 128 experts: choosing
// 9.6 us, the two steps of the order 2.7 and 6.4, the logits' gradient 5.1; one token 3.1 as one kernel, and 1.8.  Joining is bound by
// memory: 8192 tokens, 4 rows of 4096 bfloat16 values each, 336 MB: 65 us (5.2 TB/s); its gradients, 604 MB, 124 us (4.9); a large copy
// runs at 5.1.
//
// The order is that of a stable counting sort by expert.  A token takes an expert once at most, so the slots of an expert
// among 64 tokens are a 64-bit mask, the rank of one the number of mask bits below it, and nothing depends on the order in
// which atomics arrive.
#include "apb_mx4.h"

namespace apb {
namespace {

constexpr int kThreads = 256;
constexpr int kTokens = 64;                   // tokens of a workgroup: bits of a mask
constexpr int kChooseThreads = 1024;          // four waves for a SIMD to switch between: a choice is a chain of dependent steps
constexpr long long kMaxSlots = 1LL << 24;    // a workgroup of 256 lanes per token: the lanes of a launch fit 32 bits

// An order-preserving map of the logits that can be taken to positive whole numbers; -inf and NaN: 0.
__device__ __forceinline__ uint32_t order_key(float v) {
    const uint32_t b = __builtin_bit_cast(uint32_t, v + 0.0f);      // (-0 and 0 are equal)
    if (!(v > -INFINITY)) return 0u;
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float key_value(uint32_t key) {
    return __builtin_bit_cast(float, key & 0x80000000u ? key & 0x7fffffffu : ~key);
}

// Lane permutations of an operand; lanes without a partner take 0.
template <int CTRL>
__device__ __forceinline__ int from_lane(int v) { return __builtin_amdgcn_update_dpp(0, v, CTRL, 0xf, 0xf, false); }

// The best of a group of lanes, 16 (a row of the wave) or all 64, in every one of them: rotations within a row, then exchanges.
template <int LANES, class Best>
__device__ __forceinline__ uint32_t best_of(uint32_t v, Best best) {
    v = best(v, (uint32_t)from_lane<0x128>((int)v));             // by 8, 4, 2, 1
    v = best(v, (uint32_t)from_lane<0x124>((int)v));
    v = best(v, (uint32_t)from_lane<0x122>((int)v));
    v = best(v, (uint32_t)from_lane<0x121>((int)v));
    if (LANES == kWave) {
        v = best(v, (uint32_t)__shfl_xor((int)v, 16, kWave));
        v = best(v, (uint32_t)__shfl_xor((int)v, 32, kWave));
    }
    return v;
}
template <int LANES>
__device__ __forceinline__ float group_sum(float v) {
#pragma unroll
    for (int d = LANES / 2; d > 0; d >>= 1) v += __shfl_xor(v, d, LANES);
    return v;
}
// sum over this lane and those below
__device__ __forceinline__ int wave_prefix(int v) {
    v += from_lane<0x111>(v);
    v += from_lane<0x112>(v);
    v += from_lane<0x114>(v);
    v += from_lane<0x118>(v);
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);      // into rows 1 and 3
    v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);      // into rows 2 and 3
    return v;
}
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
    for (int d = kWave / 2; d > 0; d >>= 1) v += __shfl_xor(v, d, kWave);
    return v;
}

// A group of lanes: the choices of a token.  A lane holds EPL experts, expert LANES * r + lane, and gets the choices lane,
// lane + LANES ... (-1: none) and their weights.  Every choice is two reductions, the largest key and the lowest index that has it.
template <int LANES, int EPL>
__device__ __forceinline__ void choose(const void* logits, int type, long long at, int E, int k, bool there,
                                       int (&mine)[APB_MOE_MAX_K / LANES + 1], float (&weight)[APB_MOE_MAX_K / LANES + 1]) {
    constexpr int kSlots = APB_MOE_MAX_K / LANES + 1;
    const int lane = threadIdx.x & (LANES - 1);
    uint32_t key[EPL], mine_key[kSlots];
#pragma unroll
    for (int r = 0; r < EPL; ++r) {
        const int e = r * LANES + lane;
        key[r] = there && e < E ? order_key(load_f32(logits, type, at + e)) : 0u;
    }
#pragma unroll
    for (int i = 0; i < kSlots; ++i) mine[i] = -1, mine_key[i] = 0u;
    uint32_t top = 0;
    for (int j = 0; j < k; ++j) {
        uint32_t best = key[0];
#pragma unroll
        for (int r = 1; r < EPL; ++r) best = max(best, key[r]);
        best = best_of<LANES>(best, [](uint32_t a, uint32_t b) { return max(a, b); });
        uint32_t not_r = 0;                                      // ~expert, so that the lowest is the largest
#pragma unroll
        for (int r = EPL - 1; r >= 0; --r) not_r = key[r] == best ? ~(uint32_t)(r * LANES + lane) : not_r;
        const uint32_t e = ~best_of<LANES>(not_r, [](uint32_t a, uint32_t b) { return max(a, b); });
#pragma unroll
        for (int r = 0; r < EPL; ++r)
            if (e == (uint32_t)(r * LANES + lane)) key[r] = 0u;
        if (j == 0) top = best;
#pragma unroll
        for (int i = 0; i < kSlots; ++i)
            if (lane + i * LANES == j && best != 0u) mine[i] = (int)e, mine_key[i] = best;
    }
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < kSlots; ++i) {
        weight[i] = mine[i] >= 0 ? expf(key_value(mine_key[i]) - key_value(top)) : 0.0f;
        sum += weight[i];
    }
    sum = group_sum<LANES>(sum);
#pragma unroll
    for (int i = 0; i < kSlots; ++i) weight[i] = mine[i] >= 0 ? weight[i] / sum : 0.0f;
}

// What a workgroup knows of its 64 tokens: mask[e], which of them took expert e; drop[t], how many choices of token t there
// are not.
struct Block {
    unsigned long long mask[APB_MOE_MAX_E];
    int drop[kTokens];
};

__device__ __forceinline__ void clear(Block& b, int E) {
    for (int e = threadIdx.x; e < E; e += blockDim.x) b.mask[e] = 0ull;
    if (threadIdx.x < kTokens) b.drop[threadIdx.x] = 0;
}
__device__ __forceinline__ void note(Block& b, int token, int expert) {
    if (expert >= 0) atomicOr(&b.mask[expert], 1ull << token);
    else atomicAdd(&b.drop[token], 1);
}
// rank of slot (token, j) among the workgroup's slots of its expert (-1: among those without)
__device__ __forceinline__ int rank_of(const Block& b, int token, int expert, int j, int k) {
    if (expert >= 0) return __popcll(b.mask[expert] & ((1ull << token) - 1ull));
    int n = j - (k - b.drop[token]);                             // (a token's missing choices are its last ones)
    for (int i = 0; i < token; ++i) n += b.drop[i];
    return n;
}

// First rows of the experts from how many slots each has; a whole wave.
__device__ __forceinline__ int start_of(int n, int lane, int& before) {
    const int upto = wave_prefix(n);
    const int start = before + upto - n;
    before += __builtin_amdgcn_readlane(upto, kWave - 1);
    return start;
}

// ALONE: one workgroup has all tokens and does everything.  Otherwise count[e][workgroup] is written (e == E: slots without
// an expert) and the scan and placement kernels follow.
template <int LANES, int EPL, bool ALONE>
__global__ __launch_bounds__(kChooseThreads) void k_moe_choose(const void* __restrict__ logits, int type, long long ld, int T, int E,
                                                               int k, int32_t* __restrict__ expert, float* __restrict__ weight,
                                                               int32_t* __restrict__ offsets, int32_t* __restrict__ row_token,
                                                               int32_t* __restrict__ slot_row, int32_t* __restrict__ count) {
    __shared__ Block b;
    __shared__ int start[ALONE ? APB_MOE_MAX_E + 1 : 1];
    clear(b, E);
    __syncthreads();
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const int t0 = blockIdx.x * kTokens;
    for (int first = 0; first < kTokens && t0 + first < T; first += blockDim.x / LANES) {
        const int i = first + threadIdx.x / LANES, t = t0 + i, l = threadIdx.x & (LANES - 1);
        const bool there = i < kTokens && t < T;
        int e[APB_MOE_MAX_K / LANES + 1];
        float w[APB_MOE_MAX_K / LANES + 1];
        choose<LANES, EPL>(logits, type, (long long)t * ld, E, k, there, e, w);
#pragma unroll
        for (int u = 0; u <= APB_MOE_MAX_K / LANES; ++u) {
            const int j = l + u * LANES;
            if (there && j < k) {
                expert[t * k + j] = e[u];
                weight[t * k + j] = w[u];
                note(b, i, e[u]);
            }
        }
    }
    __syncthreads();
    if (!ALONE) {
        for (int e = threadIdx.x; e <= E; e += blockDim.x) {
            int n = 0;
            if (e < E) n = __popcll(b.mask[e]);
            else
                for (int i = 0; i < kTokens; ++i) n += b.drop[i];
            count[(size_t)e * gridDim.x + blockIdx.x] = n;
        }
        return;
    }
    if (wave == 0) {
        int before = 0;
        for (int base = 0; base <= E; base += kWave) {
            const int e = base + lane;
            const int first = start_of(e < E ? __popcll(b.mask[e]) : 0, lane, before);
            if (e <= E) {
                start[e] = first;
                offsets[e] = first;
            }
        }
    }
    __syncthreads();
    for (int s = threadIdx.x; s < T * k; s += blockDim.x) {
        const int t = s / k, e = expert[s];                      // (written by this workgroup, before its barrier)
        const int row = start[e >= 0 ? e : E] + rank_of(b, t, e, s - t * k, k);
        slot_row[s] = row;
        row_token[row] = t;
    }
}

// One wave per expert: count[e][..] becomes the number of slots of e before each workgroup, total[e] that of all of them.
__global__ __launch_bounds__(kWave) void k_moe_scan(int32_t* __restrict__ count, int blocks, int32_t* __restrict__ total) {
    constexpr int kEach = 4;                                     // workgroups to a lane
    const int lane = threadIdx.x;
    int32_t* row = count + (size_t)blockIdx.x * blocks;
    int before = 0;
    for (int base = 0; base < blocks; base += kWave * kEach) {
        const int i0 = base + lane * kEach;
        int n[kEach], sum = 0;
#pragma unroll
        for (int i = 0; i < kEach; ++i) n[i] = i0 + i < blocks ? row[i0 + i] : 0;
#pragma unroll
        for (int i = 0; i < kEach; ++i) sum += n[i];
        int at = start_of(sum, lane, before);
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            if (i0 + i < blocks) row[i0 + i] = at;
            at += n[i];
        }
    }
    if (lane == 0) total[blockIdx.x] = before;
}

__global__ __launch_bounds__(kThreads) void k_moe_place(const int32_t* __restrict__ expert, int T, int E, int k,
                                                        const int32_t* __restrict__ count, const int32_t* __restrict__ total,
                                                        int32_t* __restrict__ offsets, int32_t* __restrict__ row_token,
                                                        int32_t* __restrict__ slot_row) {
    __shared__ Block b;
    __shared__ int start[APB_MOE_MAX_E + 1];
    clear(b, E);
    __syncthreads();
    const int t0 = blockIdx.x * kTokens;
    const int slots = min(kTokens, T - t0) * k;
    for (int s = threadIdx.x; s < slots; s += kThreads) note(b, s / k, expert[t0 * k + s]);
    if (threadIdx.x < kWave) {
        const int lane = threadIdx.x;
        int before = 0;
        for (int base = 0; base <= E; base += kWave) {
            const int e = base + lane;
            const int first = start_of(e < E ? total[e] : 0, lane, before);
            if (e <= E) {
                start[e] = first + count[(size_t)e * gridDim.x + blockIdx.x];
                if (blockIdx.x == 0) offsets[e] = first;
            }
        }
    }
    __syncthreads();
    for (int s = threadIdx.x; s < slots; s += kThreads) {
        const int t = s / k, e = expert[t0 * k + s];
        const int row = start[e >= 0 ? e : E] + rank_of(b, t, e, s - t * k, k);
        slot_row[t0 * k + s] = row;
        row_token[row] = t0 + t;
    }
}

// Sixteen tokens to a workgroup, a row of lanes each; their rows of dlogits are put together in LDS and written as one piece.
constexpr int kRowTokens = kThreads / 16;
__global__ __launch_bounds__(kThreads) void k_moe_route_backward(const int32_t* __restrict__ expert,
                                                                 const float* __restrict__ weight,
                                                                 const float* __restrict__ dweight, int T, int E, int k,
                                                                 int type, void* __restrict__ dlogits, long long ld) {
    extern __shared__ float rows[];                              // [kRowTokens][E in whole fours]
    constexpr int kSlots = APB_MOE_MAX_K / 16;
    const int fours = (E + 3) / 4, t0 = blockIdx.x * kRowTokens;
    for (int i = threadIdx.x; i < kRowTokens * fours; i += kThreads) reinterpret_cast<f32x4*>(rows)[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    __syncthreads();
    const int l = threadIdx.x & 15, t = t0 + threadIdx.x / 16;
    int e[kSlots];
    float w[kSlots], d[kSlots], inner[kSlots] = {};
#pragma unroll
    for (int u = 0; u < kSlots; ++u) {
        const int j = l + 16 * u;
        const bool slot = t < T && j < k;
        e[u] = slot ? expert[t * k + j] : -1;
        if (e[u] >= E) e[u] = -1;
        w[u] = e[u] >= 0 ? weight[t * k + j] : 0.0f;
        d[u] = e[u] >= 0 ? dweight[t * k + j] : 0.0f;
    }
    // d_j - sum w_i d_i = sum w_i (d_j - d_i), as the weights sum to 1: nothing is lost where one of them is nearly that
    for (int i = 0; i < k; ++i) {
        const float wi = __shfl(i < 16 ? w[0] : w[1], i & 15, 16), di = __shfl(i < 16 ? d[0] : d[1], i & 15, 16);
#pragma unroll
        for (int u = 0; u < kSlots; ++u) inner[u] = fmaf(wi, d[u] - di, inner[u]);
    }
#pragma unroll
    for (int u = 0; u < kSlots; ++u)
        if (e[u] >= 0) rows[(threadIdx.x / 16) * 4 * fours + e[u]] = w[u] * inner[u];
    __syncthreads();
    for (int i = threadIdx.x; i < min(kRowTokens, T - t0) * fours; i += kThreads) {
        const int row = i / fours, first = 4 * (i - row * fours);
        const f32x4 v = reinterpret_cast<const f32x4*>(rows)[i];
        const float x[4] = {v[0], v[1], v[2], v[3]};
        store4(dlogits, type, (long long)(t0 + row) * ld + first, x, E - first);
    }
}

// A lane makes eight neighbours of a row of Y.  grid.x: tokens, grid.y: pieces of 2048 columns.
template <int TYPE, bool ONCE>
__global__ __launch_bounds__(kThreads) void k_moe_combine(const void* __restrict__ Z, long long ldz,
                                                          const int32_t* __restrict__ slot_row,
                                                          const float* __restrict__ weight, int T, int k, int N,
                                                          void* __restrict__ Y, long long ldy) {
    const int t = blockIdx.x, n = (blockIdx.y * kThreads + threadIdx.x) * 8;
    if (n >= N) return;
    float acc[8] = {};
    constexpr int kAhead = 4;                                    // rows under way
    for (int j = 0; j < k; j += kAhead) {
        int row[kAhead];
        float w[kAhead];
        Eight<TYPE> v[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            row[u] = j + u < k ? slot_row[t * k + j + u] : -1;
            w[u] = j + u < k ? weight ? weight[t * k + j + u] : 1.0f : 0.0f;
            if (row[u] < 0 || row[u] >= T * k) w[u] = 0.0f;
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
            if (w[u] != 0.0f) v[u] = load_some<TYPE, ONCE>(Z, (long long)row[u] * ldz + n, N - n);
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (w[u] == 0.0f) continue;
            float x[8];
            floats(v[u], x);
#pragma unroll
            for (int q = 0; q < 8; ++q) acc[q] = fmaf(w[u], x[q], acc[q]);
        }
    }
    store8<TYPE>(Y, (long long)t * ldy + n, N - n, acc);
}

// One workgroup per slot: its row of dZ and its dweight.
template <int TYPE, bool ONCE>
__global__ __launch_bounds__(kThreads) void k_moe_combine_backward(const void* __restrict__ dY, long long lddy,
                                                                   const void* __restrict__ Z, long long ldz,
                                                                   const int32_t* __restrict__ slot_row,
                                                                   const float* __restrict__ weight, int slots, FastDiv by_k, int N,
                                                                   void* __restrict__ dZ, long long lddz,
                                                                   float* __restrict__ dweight) {
    __shared__ float sums[kThreads / kWave];
    const int s = blockIdx.x, t = (int)by_k.div((uint32_t)s), row = slot_row[s];
    const float w = weight ? weight[s] : 1.0f;
    if (row < 0 || row >= slots) {
        if (dweight && threadIdx.x == 0) dweight[s] = 0.0f;
        return;
    }
    float dot = 0.0f;
    for (int n = threadIdx.x * 8; n < N; n += kThreads * 8) {
        const Eight<TYPE> a = load_some<TYPE>(dY, (long long)t * lddy + n, N - n);
        float g[8], d[8];
        if (dweight) {
            const Eight<TYPE> b = load_some<TYPE, ONCE>(Z, (long long)row * ldz + n, N - n);
            float z[8];
            floats(a, g);
            floats(b, z);
#pragma unroll
            for (int q = 0; q < 8; ++q) dot = fmaf(g[q], z[q], dot);
        } else {
            floats(a, g);
        }
#pragma unroll
        for (int q = 0; q < 8; ++q) d[q] = w == 0.0f ? 0.0f : w * g[q];
        store8<TYPE>(dZ, (long long)row * lddz + n, N - n, d);
    }
    if (dweight) {
        dot = wave_sum(dot);
        if ((threadIdx.x & (kWave - 1)) == 0) sums[threadIdx.x / kWave] = dot;
        __syncthreads();
        if (threadIdx.x == 0) {
            float all = sums[0];
#pragma unroll
            for (int i = 1; i < kThreads / kWave; ++i) all += sums[i];
            dweight[s] = all;
        }
    }
}

// ALONE: one workgroup has all tokens
template <bool ALONE, int LANES, int EPL, class... Args>
void launch_choose(int blocks, int T, hipStream_t s, Args... args) {
    const dim3 threads(std::min(kChooseThreads, (LANES * T + kWave - 1) / kWave * kWave));
    hipLaunchKernelGGL((k_moe_choose<LANES, EPL, ALONE>), dim3(blocks), threads, 0, s, args...);
}
// The lanes of a token: 16 wherever that leaves more tokens to a wave, all 64 where a workgroup has a wave for every token or a
// lane of 16 would hold too many experts.  Measured, 16 lanes and 64 (us): 16384 tokens, 64, 128, 256, 512 experts 11 and 15, 16
// and 23, 21 and 28, 230 and 43 (of 16 experts each 51); one token, 64, 128, 256 experts 3.8 and 3.5, 5.2 and 4.5, 7.7 and 5.5.
template <bool ALONE, class... Args>
void launch_by_experts(int E, int T, int blocks, hipStream_t s, Args... args) {
    if (E > 512) return launch_choose<ALONE, 64, 16>(blocks, T, s, args...);
    if (E > 256) return launch_choose<ALONE, 64, 8>(blocks, T, s, args...);
    if constexpr (ALONE) {
        if (T <= kChooseThreads / kWave) {
            if (E <= 64) return launch_choose<ALONE, 64, 1>(blocks, T, s, args...);
            if (E <= 128) return launch_choose<ALONE, 64, 2>(blocks, T, s, args...);
            return launch_choose<ALONE, 64, 4>(blocks, T, s, args...);
        }
    }
    if (E <= 64) return launch_choose<ALONE, 16, 4>(blocks, T, s, args...);
    if (E <= 128) return launch_choose<ALONE, 16, 8>(blocks, T, s, args...);
    launch_choose<ALONE, 16, 16>(blocks, T, s, args...);
}

bool bad_route(int T, int E, int k) {
    return T <= 0 || E <= 0 || k <= 0 || k > E || E > APB_MOE_MAX_E || k > APB_MOE_MAX_K || (long long)T * k >= kMaxSlots;
}
// Rows that the last cache (256 MB) would not keep for who reads them next beside what else is in use are read past it.  Measured
// with and without, the join, its gradients, one behind the other (us): 268 MB 59 and 66, 118 and 121, 175 and 196; 134 MB 35 and
// 35, 62 and 62, 96 and 101; 34 MB 9 and 9, 19 and 18, 29 and 26.
bool beyond_caches(int T, int k, int N, int type) { return (long long)T * k * N * type_size(type) >= 128LL << 20; }
int route_blocks(int T) { return (T + kTokens - 1) / kTokens; }

}  // namespace
}  // namespace apb

using namespace apb;

extern "C" {

size_t apb_moe_workspace_bytes(int T, int E, int k) {
    if (bad_route(T, E, k)) return 0;
    return ((size_t)route_blocks(T) + 1) * (E + 1) * sizeof(int32_t);
}

int apb_moe_route(const void* logits, int type, long long ld, int T, int E, int k, int32_t* expert, float* weight,
                  int32_t* offsets, int32_t* row_token, int32_t* slot_row, void* workspace, void* stream) {
    if (!logits || !expert || !weight || !offsets || !row_token || !slot_row || !workspace) return APB_ERR_NULL;
    if (bad_type(type)) return APB_ERR_TYPE;
    if (bad_route(T, E, k) || ld < E) return APB_ERR_SHAPE;
    if (!aligned(logits, type_size(type)) || !aligned(expert, 4) || !aligned(weight, 4) || !aligned(offsets, 4) ||
        !aligned(row_token, 4) || !aligned(slot_row, 4) || !aligned(workspace, 4))
        return APB_ERR_ALIGN;
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    const int blocks = route_blocks(T);
    int32_t* count = static_cast<int32_t*>(workspace);
    if (blocks == 1) {
        launch_by_experts<true>(E, T, blocks, s, logits, type, ld, T, E, k, expert, weight, offsets, row_token, slot_row, count);
    } else {
        launch_by_experts<false>(E, T, blocks, s, logits, type, ld, T, E, k, expert, weight, offsets, row_token, slot_row, count);
        int32_t* total = count + (size_t)blocks * (E + 1);
        hipLaunchKernelGGL(k_moe_scan, dim3(E + 1), dim3(kWave), 0, s, count, blocks, total);
        hipLaunchKernelGGL(k_moe_place, dim3(blocks), dim3(kThreads), 0, s, expert, T, E, k, count, total, offsets, row_token, slot_row);
    }
    APB_HIP(hipGetLastError());
    return APB_OK;
}

int apb_moe_route_backward(const int32_t* expert, const float* weight, const float* dweight, int T, int E, int k, int type,
                           void* dlogits, long long ld, void* stream) {
    if (!expert || !weight || !dweight || !dlogits) return APB_ERR_NULL;
    if (bad_type(type)) return APB_ERR_TYPE;
    if (bad_route(T, E, k) || ld < E) return APB_ERR_SHAPE;
    if (!aligned(expert, 4) || !aligned(weight, 4) || !aligned(dweight, 4) || !aligned(dlogits, type_size(type))) return APB_ERR_ALIGN;
    const size_t lds = (size_t)kRowTokens * ((E + 3) / 4) * 16;
    hipLaunchKernelGGL(k_moe_route_backward, dim3((T + kRowTokens - 1) / kRowTokens), dim3(kThreads), lds,
                       reinterpret_cast<hipStream_t>(stream), expert, weight, dweight, T, E, k, type, dlogits, ld);
    APB_HIP(hipGetLastError());
    return APB_OK;
}

#define APB_LAUNCH(kernel, type, once, grid, ...)                                                                          \
    do {                                                                                                                   \
        if (once) hipLaunchKernelGGL((kernel<type, true>), grid, dim3(kThreads), 0, s, __VA_ARGS__);                       \
        else hipLaunchKernelGGL((kernel<type, false>), grid, dim3(kThreads), 0, s, __VA_ARGS__);                           \
    } while (0)
#define APB_BY_TYPE(kernel, once, grid, ...)                                                                               \
    do {                                                                                                                   \
        if (type == APB_F32) APB_LAUNCH(kernel, APB_F32, once, grid, __VA_ARGS__);                                         \
        else if (type == APB_BF16) APB_LAUNCH(kernel, APB_BF16, once, grid, __VA_ARGS__);                                  \
        else APB_LAUNCH(kernel, APB_F16, once, grid, __VA_ARGS__);                                                         \
    } while (0)

int apb_moe_combine(const void* Z, int type, long long ldz, const int32_t* slot_row, const float* weight, int T, int k,
                    int N, void* Y, long long ldy, void* stream) {
    if (!Z || !slot_row || !Y) return APB_ERR_NULL;
    if (bad_type(type)) return APB_ERR_TYPE;
    if (T <= 0 || k <= 0 || k > APB_MOE_MAX_K || N <= 0 || N > kMxMaxK || (long long)T * k >= kMaxSlots || ldz < N || ldy < N) return APB_ERR_SHAPE;
    if (!aligned(Z, type_size(type)) || !aligned(Y, type_size(type)) || !aligned(slot_row, 4) || !aligned(weight, 4)) return APB_ERR_ALIGN;
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    const dim3 grid((unsigned)T, (unsigned)((N + kThreads * 8 - 1) / (kThreads * 8)));
    APB_BY_TYPE(k_moe_combine, beyond_caches(T, k, N, type), grid, Z, ldz, slot_row, weight, T, k, N, Y, ldy);
    APB_HIP(hipGetLastError());
    return APB_OK;
}

int apb_moe_combine_backward(const void* dY, int type, long long lddy, const void* Z, long long ldz, const int32_t* slot_row,
                             const float* weight, int T, int k, int N, void* dZ, long long lddz, float* dweight,
                             void* stream) {
    if (!dY || (!Z && dweight) || !slot_row || !dZ) return APB_ERR_NULL;
    if (bad_type(type)) return APB_ERR_TYPE;
    if (T <= 0 || k <= 0 || k > APB_MOE_MAX_K || N <= 0 || N > kMxMaxK || (long long)T * k >= kMaxSlots || (Z && ldz < N) || lddy < N || lddz < N)
        return APB_ERR_SHAPE;
    if (!aligned(dY, type_size(type)) || !aligned(Z, type_size(type)) || !aligned(dZ, type_size(type)) || !aligned(slot_row, 4) ||
        !aligned(weight, 4) || !aligned(dweight, 4))
        return APB_ERR_ALIGN;
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    const int slots = T * k;
    const dim3 grid((unsigned)slots);
    APB_BY_TYPE(k_moe_combine_backward, beyond_caches(T, k, N, type), grid, dY, lddy, Z, ldz, slot_row, weight, slots, FastDiv((uint32_t)k), N,
                dZ, lddz, dweight);
    APB_HIP(hipGetLastError());
    return APB_OK;
}

}  // extern "C"
