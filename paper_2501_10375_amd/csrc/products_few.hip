// Grouped forward products of few rows: a stream over the weights of the experts that have any, bf16 or block-scaled e4m3.
//
// Bound by memory: a pass over an expert's weights serves 16 * RF of its rows.  A workgroup takes 16 * FG features of an expert, its
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
constexpr int kRows = 16;    // of a fragment

__device__ inline i32x4 load16(const char* p) { return *reinterpret_cast<const i32x4*>(p); }

template <bool FP8, int RF, int FG, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void product_few_rows_kernel(Args a) {
    constexpr int kFeatures = 16 * FG, kThreads = 64 * WAVES, kPass = RF * kRows;
    __shared__ float sums[WAVES][kPass][kFeatures + 1];
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

    for (int row0 = __builtin_amdgcn_readlane(first, e); row0 < row_end; row0 += kPass) {
        const int rows = min(kPass, row_end - row0);
        const char* x[RF];
        const float* x_scale[RF];
        f32x4 acc[RF][FG];
#pragma unroll
        for (int r = 0; r < RF; ++r) {
            const size_t row = row0 + min(r * kRows + lane % 16, rows - 1);   // (rows past the end repeat the last one)
            x[r] = static_cast<const char*>(a.q) + row * row_bytes + lane / 16 * 16;
            x_scale[r] = FP8 ? a.q_scales + row * kb : nullptr;
#pragma unroll
            for (int f = 0; f < FG; ++f) acc[r][f] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
        auto step = [&](int s, bool second_half) __attribute__((always_inline)) {
            const size_t at = (size_t)s * kLine;
            i32x4 wl[FG], wh[FG], xl[RF], xh[RF];
#pragma unroll
            for (int f = 0; f < FG; ++f) {
                wl[f] = load16(w + f * 16 * row_bytes + at);
                wh[f] = second_half ? load16(w + f * 16 * row_bytes + at + 64) : i32x4{0, 0, 0, 0};
            }
#pragma unroll
            for (int r = 0; r < RF; ++r) {
                xl[r] = load16(x[r] + at);
                xh[r] = second_half ? load16(x[r] + at + 64) : i32x4{0, 0, 0, 0};
            }
#pragma unroll
            for (int r = 0; r < RF; ++r) {
                if constexpr (FP8) {
                    const float by = x_scale[r][s] * w_scale[s];
                    const i32x8 q = __builtin_shufflevector(xl[r], xh[r], 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
                    for (int f = 0; f < FG; ++f) {
                        const i32x8 p = __builtin_shufflevector(wl[f], wh[f], 0, 1, 2, 3, 4, 5, 6, 7);
                        const f32x4 d = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(p, q, f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0, 0, 0, 0);
#pragma unroll
                        for (int c = 0; c < 4; ++c) acc[r][f][c] = fmaf(d[c], by, acc[r][f][c]);
                    }
                } else {
#pragma unroll
                    for (int f = 0; f < FG; ++f) {
                        acc[r][f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, wl[f]), __builtin_bit_cast(bf16x8, xl[r]), acc[r][f], 0, 0, 0);
                        acc[r][f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, wh[f]), __builtin_bit_cast(bf16x8, xh[r]), acc[r][f], 0, 0, 0);
                    }
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

        // A result: lane l holds row l % 16 and features 4 * (l / 16) + 0 .. 3 of its fragments.
#pragma unroll
        for (int r = 0; r < RF; ++r)
#pragma unroll
            for (int f = 0; f < FG; ++f)
#pragma unroll
                for (int c = 0; c < 4; ++c) sums[wave][r * kRows + lane % 16][f * 16 + lane / 16 * 4 + c] = acc[r][f][c];
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

template <bool FP8, int RF, int FG, int WAVES>
hipError_t launch(const Args& a, int active, hipStream_t stream) {
    product_few_rows_kernel<FP8, RF, FG, WAVES><<<dim3((unsigned)(active * (a.n / (16 * FG)))), 64 * WAVES, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_few_rows(const Args& a, bool fp8, hipStream_t stream) {
    const int active = a.experts < a.rows ? a.experts : a.rows;
    const FewRows v = choose_few_rows({a.experts, a.rows, a.n, a.k}, fp8, compute_units());
    if (!fp8) return v.waves == 8 ? launch<false, 1, 1, 8>(a, active, stream) : launch<false, 1, 1, 4>(a, active, stream);
    if (v.row_fragments == 1) return v.feature_fragments == 1 ? launch<true, 1, 1, 4>(a, active, stream) : launch<true, 1, 2, 4>(a, active, stream);
    return v.feature_fragments == 2 ? launch<true, 2, 2, 4>(a, active, stream) : launch<true, 2, 4, 4>(a, active, stream);
}

}  // namespace products
}  // namespace moe
