// Y = Q(X) W^T for few rows, plain or grouped by expert: what bounds it is reading the weights once.  One kernel: a workgroup
// brings its rows of X into LDS as 4-bit blocks (quantizing them on the way) while its first weights are already under way, then
// streams weights through a ring of its own in LDS into the matrix cores.  One row of 4096 through 4096 x 4096 weights, 8.9 MB:
// 5.1 us, of which an empty launch has 2; 16 tokens at 4 of 64 experts of 2048 x 2048, 92 MB of weights: 21 us, 4.3 TB/s.
#include <atomic>
#include <type_traits>

#include "apb_mx4.h"

namespace apb {
namespace {

constexpr int kThreads = 512;
constexpr int kWaves = kThreads / kWave;
constexpr int kRing = 3;                      // segments of 16 rows of weights that a wave has under way
constexpr int kSlot = 16 * kMxSegBytes + 256; // of the ring: 2 KB of codes, 16 rows' scales (twice)
constexpr int kFourBit = 3;                   // "type" of an X that is a 4-bit matrix already
constexpr size_t kMaxLds = 150 * 1024;
constexpr int kMaxDevices = 64;               // devices of one process the launcher keeps state for
constexpr int kWorkgroups = 2048;             // of a launch, at most about: two resident per compute unit, four times over

struct Rows {                                 // the left operand: float rows or a 4-bit matrix
    const void* x;
    long long ld;
    int rows_in;
    const int32_t* rows_from;
    Mx mx;
};

// A wave computes 16 outputs (rows of W) x 16 rows; WK = 2^wk_log2 waves split the segments of a tile
// among them and join their sums through LDS in a fixed order.  Weights go from memory to a ring of the wave's own in LDS, whole
// lines of 128 bytes per row (loaded to registers in the order of the operands they would come in half lines, at half the
// speed), so a wave waits for nobody but its own loads.  Lane (r, g) holds row r; of a segment of 256, step s multiplies blocks
// 4 s .. 4 s + 3.
template <int TYPE>
__global__ __launch_bounds__(kThreads, 4) void k_mx4_few(Rows X, Mx W, const int32_t* __restrict__ offsets, int E, int M, int N,
                                                         int K, int lds_rows, int wk_log2, int type, void* __restrict__ Y,
                                                         long long ldy) {
    extern __shared__ __align__(16) uint8_t lds[];
    const int segs = W.segs;
    const RowTile t = find_row_tile(offsets, E, M, 16, blockIdx.x);
    if (t.rows <= 0) return;
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int tiles_n = (N + 15) / 16;
    const int wk_n = 1 << wk_log2, wn_n = kWaves >> wk_log2;
    if (t.e >= E) {
        const float zero[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        for (int nt = blockIdx.y * kWaves + wave; nt < tiles_n; nt += gridDim.y * kWaves)
            for (int i = lane; i < t.rows * 4; i += kWave) {
                const int n = nt * 16 + (i & 3) * 4;
                store4(Y, type, (long long)(t.row0 + (i >> 2)) * ldy + n, zero, N - n);
            }
        return;
    }
    const int wk = wave & (wk_n - 1), wn = wave >> wk_log2;
    const int r = lane & 15, g = lane >> 4;
    const int step_n = gridDim.y * wn_n;
    const uint32_t pitch = (uint32_t)segs * kMxSegBytes;
    const int nt0 = blockIdx.y * wn_n + wn;
    // what this wave multiplies, in order: segments wk, wk + wk_n, ... of tiles nt0, nt0 + step_n, ...
    const int mine = wk < segs ? (segs - wk + wk_n - 1) / wk_n : 0;
    const int items = nt0 < tiles_n ? ((tiles_n - nt0 + step_n - 1) / step_n) * mine : 0;

    uint8_t* x_scales = lds + (size_t)lds_rows * pitch;
    uint8_t* ring = x_scales + ((size_t)lds_rows * segs * 8 + 15) / 16 * 16;
    float* sums = reinterpret_cast<float*>(ring + kWaves * kRing * kSlot);
    ring += wave * kRing * kSlot;
    const uint32_t ring_at = __builtin_amdgcn_readfirstlane(lds_address(ring));
    int fetch_nt = nt0, fetch_seg = wk, fetch_slot = 0;
    const uint8_t* w_codes = W.codes + (size_t)t.e * N * pitch;
    const uint8_t* w_scales = W.scales + (size_t)t.e * N * 8;
    auto fetch = [&]() {
        const int n0 = fetch_nt * 16, last = N - 1 - n0;         // rows beyond N repeat the last one
        const uint8_t* p = w_codes + (size_t)n0 * pitch + (size_t)fetch_seg * kMxSegBytes;
        const uint8_t* q = w_scales + ((size_t)fetch_seg * W.rows + n0) * 8;
        const uint32_t to = ring_at + fetch_slot * kSlot;
        const int row = lane >> 3, other = row + 8;
        load16_to_lds(to, p, min(row, last) * pitch + 16 * ((lane & 7) ^ (row & 7)));
        load16_to_lds(to + 1024, p, min(other, last) * pitch + 16 * ((lane & 7) ^ (other & 7)));
        load4_to_lds(to + 2048, q, 8 * min((lane >> 1) & 15, last) + 4 * (lane & 1));
        fetch_slot = fetch_slot + 1 == kRing ? 0 : fetch_slot + 1;
        fetch_seg += wk_n;
        if (fetch_seg >= segs) {
            fetch_seg = wk;
            fetch_nt += step_n;
        }
    };
    for (int i = 0; i < min(kRing, items); ++i) fetch();

    // X: row i's 16-byte blocks, permuted by the row's number (no bank is met twice by eight rows), then the scales of all rows
    // A wave takes pieces of 512 values of a row, eight for each lane, four pieces at a time as long as it has as many.
    const int pieces = (segs + 1) / 2, all = t.rows * pieces;
    auto bring = [&](int first, auto count) {
        constexpr int kCount = decltype(count)::value;
        Eight<TYPE == kFourBit ? APB_BF16 : TYPE> v[kCount];
        uint32_t word[kCount], mark[kCount];
        int row[kCount], unit[kCount];
#pragma unroll
        for (int u = 0; u < kCount; ++u) {
            const int i = first + u * kWaves;
            row[u] = i / pieces;
            unit[u] = (i - row[u] * pieces) * kWave + lane;
            if (unit[u] >= segs * 32) unit[u] -= 32;             // (half a piece: the other half does the same again)
            if constexpr (TYPE == kFourBit) {
                const size_t src = (size_t)(t.row0 + row[u]);
                word[u] = *reinterpret_cast<const uint32_t*>(X.mx.codes + src * pitch + 4 * unit[u]);
                mark[u] = X.mx.scales[((size_t)(unit[u] >> 5) * X.mx.rows + src) * 8 + ((unit[u] >> 2) & 7)];
            } else {
                const int src = X.rows_from ? X.rows_from[t.row0 + row[u]] : t.row0 + row[u];
                v[u] = load_some<TYPE>(X.x, (long long)src * X.ld + 8 * unit[u], src >= 0 && src < X.rows_in ? K - 8 * unit[u] : 0);
            }
        }
#pragma unroll
        for (int u = 0; u < kCount; ++u) {
            if constexpr (TYPE != kFourBit) {
                mark[u] = scale_code(top_of_four(top_bits(v[u])));
                word[u] = encode8(v[u], mark[u]);
            }
            *reinterpret_cast<uint32_t*>(lds + row[u] * pitch + 16 * ((unit[u] >> 2) ^ (row[u] & 7)) + 4 * (unit[u] & 3)) = word[u];
            if ((unit[u] & 3) == 0) x_scales[row[u] * segs * 8 + (unit[u] >> 2)] = (uint8_t)mark[u];
        }
    };
    int piece = wave;
    for (; piece + 3 * kWaves < all; piece += 4 * kWaves) bring(piece, std::integral_constant<int, 4>{});
    for (; piece < all; piece += kWaves) bring(piece, std::integral_constant<int, 1>{});
    __syncthreads();

    const int row = min(r, t.rows - 1);
    const uint8_t* x_codes = lds + row * pitch;
    int item = 0, slot = 0, nt = nt0;
    for (int base = blockIdx.y * wn_n; base < tiles_n; base += step_n, nt += step_n) {
        f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
        for (int seg = nt < tiles_n ? wk : segs; seg < segs; seg += wk_n, ++item) {
            // all but the loads of the segments behind this one
            if (item + kRing <= items) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(3 * (kRing - 1)) : "memory");
            else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            const uint8_t* from = ring + slot * kSlot;
            const u32x4 w0 = *reinterpret_cast<const u32x4*>(from + r * kMxSegBytes + 16 * (g ^ (r & 7)));
            const u32x4 w1 = *reinterpret_cast<const u32x4*>(from + r * kMxSegBytes + 16 * ((4 + g) ^ (r & 7)));
            const int sw0 = from[2048 + 8 * r + g], sw1 = from[2048 + 8 * r + 4 + g];
            const uint8_t* sx = x_scales + (row * segs + seg) * 8 + g;
            const u32x4 x0 = *reinterpret_cast<const u32x4*>(x_codes + 16 * ((8 * seg + g) ^ (row & 7)));
            const u32x4 x1 = *reinterpret_cast<const u32x4*>(x_codes + 16 * ((8 * seg + 4 + g) ^ (row & 7)));
            acc = mfma16<0>(w0, x0, acc, sw0, sx[0]);
            acc = mfma16<0>(w1, x1, acc, sw1, sx[4]);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // (this slot has been read)
            if (item + kRing < items) fetch();
            slot = slot + 1 == kRing ? 0 : slot + 1;
        }
        if (wk_n > 1) {
            // (the barrier at the end of the loop keeps this round's readers ahead of the next round's writers)
            *reinterpret_cast<f32x4*>(sums + (wave * kWave + lane) * 4) = acc;
            __syncthreads();
            if (wk == 0)
                for (int w = 1; w < wk_n; ++w) {
                    const f32x4 v = *reinterpret_cast<const f32x4*>(sums + ((wave + w) * kWave + lane) * 4);
#pragma unroll
                    for (int q = 0; q < 4; ++q) acc[q] += v[q];
                }
        }
        if (wk == 0 && nt < tiles_n && r < t.rows) {
            const int n = nt * 16 + 4 * g;
            const float v[4] = {acc[0], acc[1], acc[2], acc[3]};
            store4(Y, type, (long long)(t.row0 + r) * ldy + n, v, N - n);
        }
        if (wk_n > 1) __syncthreads();
    }
}

size_t lds_bytes(int rows, int segs) {
    return (size_t)rows * segs * kMxSegBytes + ((size_t)rows * segs * 8 + 15) / 16 * 16 + (size_t)kWaves * kRing * kSlot +
           (size_t)kWaves * kWave * 16;
}
template <int TYPE>
int launch(const Rows& X, const Mx& W, const int32_t* offsets, int E, int M, int N, int K, int type, void* Y, long long ldy, hipStream_t s) {
    const int lds_rows = std::min(M, 16);
    const size_t lds = lds_bytes(lds_rows, W.segs);
    const long long row_tiles = max_row_tiles(M, E, offsets != nullptr, 16);
    const int tiles_n = (N + 15) / 16;
    // Waves share a tile only where there would be fewer workgroups than compute units without.
    int wk = 0;
    while (wk < 3 && row_tiles * ((tiles_n + (kWaves >> wk) - 1) / (kWaves >> wk)) < 256) ++wk;
    const int groups = (tiles_n + (kWaves >> wk) - 1) / (kWaves >> wk);
    const long long per_row_tile = std::max<long long>(1, kWorkgroups / row_tiles);
    const dim3 grid((unsigned)row_tiles, (unsigned)std::min<long long>(groups, per_row_tile));
    if (lds > 64 * 1024) {                                       // more than a launch gets without asking: once per device
        static std::atomic<bool> asked[kMaxDevices];
        int dev = 0;
        APB_HIP(hipGetDevice(&dev));
        if (dev < 0 || dev >= kMaxDevices) return APB_ERR_SHAPE;
        if (!asked[dev].load(std::memory_order_acquire)) {
            APB_HIP(hipFuncSetAttribute(reinterpret_cast<const void*>(&k_mx4_few<TYPE>), hipFuncAttributeMaxDynamicSharedMemorySize,
                                        (int)kMaxLds));
            asked[dev].store(true, std::memory_order_release);
        }
    }
    hipLaunchKernelGGL((k_mx4_few<TYPE>), grid, dim3(kThreads), lds, s, X, W, offsets, E, M, N, K, lds_rows, wk, type, Y, ldy);
    APB_HIP(hipGetLastError());
    return APB_OK;
}

}  // namespace

// A workgroup quantizes every row it multiplies with, so the rows must be few and short.  Measured against quantization and
// tiles (us): 4096 x 4096, 1 row 5.0 : 11.7, 16 rows 10.4 : 12.2, 32 rows 16.9 : 12.4; 8192 x 8192, 4 rows 12.2 : 19.9, 16 rows
// 20.5 : 20.0; 64 experts of 2048 x 2048, a row each 20.5 : 26.1, 4 rows 33.9 : 36.1, 8 rows 38.4 : 36.8; 16 experts of
// 2048 x 4096, 8 rows each 28.4 : 17.2.  Not measured: experts of K above 8192, which go to tiles with a row each.
bool mx4_few_applies(const int32_t* offsets, int E, int M, int K) {
    const int mean = offsets ? (M + E - 1) / E : M;              // rows of an expert, were they all alike
    return mean <= 16 && (long long)mean * K <= (offsets ? 8192 : 65536) && lds_bytes(std::min(M, 16), mx_segs(K)) <= kMaxLds;
}

int launch_mx4_few(const void* X, int x_type, long long ldx, int rows_in, const int32_t* rows_from, const Mx& W, const int32_t* offsets,
                   int E, int M, int N, int K, int type, void* Y, long long ldy, hipStream_t s) {
    const Rows rows{X, ldx, rows_in, rows_from, Mx{}};
    if (x_type == APB_F32) return launch<APB_F32>(rows, W, offsets, E, M, N, K, type, Y, ldy, s);
    if (x_type == APB_BF16) return launch<APB_BF16>(rows, W, offsets, E, M, N, K, type, Y, ldy, s);
    return launch<APB_F16>(rows, W, offsets, E, M, N, K, type, Y, ldy, s);
}
int launch_mx4_few(const Mx& A, const Mx& W, const int32_t* offsets, int E, int M, int N, int K, int type, void* Y, long long ldy, hipStream_t s) {
    return launch<kFourBit>(Rows{nullptr, 0, 0, nullptr, A}, W, offsets, E, M, N, K, type, Y, ldy, s);
}

}  // namespace apb
