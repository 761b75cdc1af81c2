// Grouped forward products of few rows: a stream over the weights of the experts that have any, bf16 or block-scaled e4m3.
//
// Bound by memory: a pass over an expert's weights serves 16 of its rows.  A workgroup takes 16 * FG features of an expert, its
// wavefronts a share of the contraction each, and the weights go from memory straight to the registers that the matrix
// instructions read: a load covers 16 features x 64 bytes, the next one the other halves of the same lines.  The rows come from the
// caches the same way.  The wavefronts' sums meet in LDS.  (Loads that bypass the caches' replacement are slower: 16 rows through 8
// experts of 14336 x 4096 167 us with them, 153 without.)  6.1 TB/s for that, 2 rows of them 33 us with a part in the memory-side cache.
#include "bf16_utils.h"
#include "products_internal.h"

namespace moe {
namespace products {
namespace {

typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) int i32x4;
typedef __attribute__((ext_vector_type(8))) int i32x8;

constexpr int kLine = 128;   // bytes of a K step
constexpr int kRows = 16;

__device__ inline i32x4 load16(const char* p) { return *reinterpret_cast<const i32x4*>(p); }

template <bool FP8, int FG, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void product_few_rows_kernel(Args a) {
    constexpr int kFeatures = 16 * FG, kThreads = 64 * WAVES;
    __shared__ float sums[WAVES][kRows][kFeatures + 1];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int f_tiles = a.n / kFeatures;
    const int nth = blockIdx.x / f_tiles, f0 = (blockIdx.x - nth * f_tiles) * kFeatures;
    // The nth expert that has rows.
    int first, end;
    expert_rows(a, lane, first, end);
    uint64_t with_rows = __ballot(end > first);
    for (int i = 0; i < nth; ++i) with_rows &= with_rows - 1;
    if (with_rows == 0) return;
    const int e = __ffsll((long long)with_rows) - 1;
    const int row_end = __builtin_amdgcn_readlane(end, e);

    const size_t row_bytes = (size_t)a.k * (FP8 ? 1 : 2);
    const int steps = (int)((row_bytes + kLine - 1) / kLine), begin = steps * wave / WAVES, stop = steps * (wave + 1) / WAVES;
    const int kb = (a.k + 127) / 128, nb = (a.n + 127) / 128;
    const char* w = static_cast<const char*>(a.p) + ((size_t)e * a.n + f0 + lane % 16) * row_bytes + lane / 16 * 16;
    const float* w_scale = FP8 ? a.p_scales + ((size_t)e * nb + f0 / 128) * kb : nullptr;

    for (int row0 = __builtin_amdgcn_readlane(first, e); row0 < row_end; row0 += kRows) {
        const int rows = min(kRows, row_end - row0);
        const size_t row = row0 + min(lane % 16, rows - 1);   // (rows past the end repeat the last one)
        const char* x = static_cast<const char*>(a.q) + row * row_bytes + lane / 16 * 16;
        const float* x_scale = FP8 ? a.q_scales + row * kb : nullptr;
        f32x4 acc[FG];
#pragma unroll
        for (int f = 0; f < FG; ++f) acc[f] = f32x4{0.f, 0.f, 0.f, 0.f};
        auto step = [&](int s, bool second_half) __attribute__((always_inline)) {
            const size_t at = (size_t)s * kLine;
            i32x4 wl[FG], wh[FG];
#pragma unroll
            for (int f = 0; f < FG; ++f) {
                wl[f] = load16(w + f * 16 * row_bytes + at);
                wh[f] = second_half ? load16(w + f * 16 * row_bytes + at + 64) : i32x4{0, 0, 0, 0};
            }
            const i32x4 xl = load16(x + at), xh = second_half ? load16(x + at + 64) : i32x4{0, 0, 0, 0};
            if constexpr (FP8) {
                const float by = x_scale[s] * w_scale[s];
                const i32x8 q = __builtin_shufflevector(xl, xh, 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
                for (int f = 0; f < FG; ++f) {
                    const i32x8 p = __builtin_shufflevector(wl[f], wh[f], 0, 1, 2, 3, 4, 5, 6, 7);
                    const f32x4 d = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(p, q, f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0, 0, 0, 0);
#pragma unroll
                    for (int c = 0; c < 4; ++c) acc[f][c] = fmaf(d[c], by, acc[f][c]);
                }
            } else {
#pragma unroll
                for (int f = 0; f < FG; ++f) {
                    acc[f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, wl[f]), __builtin_bit_cast(bf16x8, xl), acc[f], 0, 0, 0);
                    acc[f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, wh[f]), __builtin_bit_cast(bf16x8, xh), acc[f], 0, 0, 0);
                }
            }
        };
        const bool ragged = FP8 && a.k % kLine != 0 && stop == steps;   // the last block has 64 numbers
        const int whole = ragged ? stop - 1 : stop;
        int s = begin;
        for (; s + 4 <= whole; s += 4) {
#pragma unroll
            for (int i = 0; i < 4; ++i) step(s + i, true);
        }
        for (; s < whole; ++s) step(s, true);
        if (ragged && s < stop) step(s, false);

        // A result: lane l holds row l % 16 and features 4 * (l / 16) + 0 .. 3 of its fragment.
#pragma unroll
        for (int f = 0; f < FG; ++f)
#pragma unroll
            for (int c = 0; c < 4; ++c) sums[wave][lane % 16][f * 16 + lane / 16 * 4 + c] = acc[f][c];
        __syncthreads();
        for (int i = threadIdx.x; i < rows * (kFeatures / 2); i += kThreads) {
            const int row = i / (kFeatures / 2), f = i % (kFeatures / 2) * 2;
            float lo = sums[0][row][f], hi = sums[0][row][f + 1];
#pragma unroll
            for (int v = 1; v < WAVES; ++v) {
                lo += sums[v][row][f];
                hi += sums[v][row][f + 1];
            }
            *reinterpret_cast<uint32_t*>(static_cast<uint16_t*>(a.out) + (size_t)(row0 + row) * a.n + f0 + f) = pack_bf16x2(lo, hi);
        }
        __syncthreads();
    }
}

template <bool FP8, int FG, int WAVES>
hipError_t launch(const Args& a, int active, hipStream_t stream) {
    product_few_rows_kernel<FP8, FG, WAVES><<<dim3((unsigned)(active * (a.n / (16 * FG)))), 64 * WAVES, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace

// Up to 16 rows a pass over the weights of every expert that has any is all that is needed; beyond, as long as the experts have few on average, see the
// times of this kernel / of the tile kernels in us (experts, out, in features, rows): bf16 8, 14336, 4096, 16 154 / 181, 32 171 / 186, 64 188 / 191, 128 259 / 198;
// 8, 4096, 14336, 32 192 / 187, 64 195 / 177; 64, 1408, 2048, 64 44 / 55, 240 68 / 92; 1, 6400, 4096, 16 17 / 22, 64 59 / 30; 8 bits 8, 14336, 4096, 16 80 / 102, 64
// 84 / 106, 128 112 / 111; 16, 6400, 4096, 32 72 / 101; 64, 1408, 2048, 240 35 / 49; 1, 14336, 4096, 32 26 / 25.
bool few_rows(const Args& a, bool fp8) { return a.rows <= kRows || a.rows <= (fp8 ? 8 : 4) * a.experts; }

// Two feature fragments for 8 bits beyond 16 rows: the rows' loads and scales serve both (8, 14336, 4096, 64: 99 -> 84 us; bf16 188 -> 203).
// Eight wavefronts where four would leave the CUs with few and each still has 16 K steps (bf16 8, 4096, 14336, 2: 42 -> 37 us; with less, 8 bits
// 16, 6400, 4096, 2: 12.2 -> 15.4).
hipError_t launch_few_rows(const Args& a, bool fp8, hipStream_t stream) {
    const int active = a.experts < a.rows ? a.experts : a.rows;   // experts with rows, at most
    const bool eight = (long)active * (a.n / 16) <= 4L * compute_units() && a.k / 64 >= 8 * 16;
    if (!fp8) return eight ? launch<false, 1, 8>(a, active, stream) : launch<false, 1, 4>(a, active, stream);
    return a.rows <= kRows ? launch<true, 1, 4>(a, active, stream) : launch<true, 2, 4>(a, active, stream);
}

}  // namespace products
}  // namespace moe
