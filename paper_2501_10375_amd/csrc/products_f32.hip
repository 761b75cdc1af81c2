// Grouped products on the fp32 matrix instructions: the forward product and both gradients of one tile kernel.
//
// A workgroup computes 64 features of up to 64 or 16 rows.  v_mfma_f32_16x16x4_f32 takes one number a lane, row lane % 16 and one of four c by
// lane / 16; which four is free as long as both operands take the same, so instruction m of 16 c takes c = 4 * (lane / 16) + m, and a fragment of 16 c is
// four consecutive numbers a lane.  An operand whose contraction is contiguous goes through LDS as it lies in memory, 16-byte units exchanged
// within a row, and a fragment is one ds_read_b128; one whose rows are (the weights of dgrad, both operands of wgrad) as [c][row], four
// ds_read_b32 whose four c are 16 banks apart.  The features are the instruction's first operand, so that a lane ends up with
// four consecutive ones of a row.
//
// Forward and dgrad: each wavefront 16 features of all rows, so that a ragged tile costs what its groups of 16 rows cost; K steps of 32
// (the forward product of few rows: of 64, a row's 256 bytes at a time).  wgrad: 32 x 32 each; K steps of 16, as its contraction may be a few rows; whole
// rows of the result leave through LDS past the caches.  Two steps are requested ahead.
//
// Large products are bound by the MFMAs (1024 rows, 4096 x 4096: 125 TFLOP/s forward, 127 dgrad, 117 wgrad, which is nine tenths of the cycles at 2.1 GHz; a
// library product of 4096^3 reaches 150), those of few rows by the weights (64 rows, 8 experts of 4096 x 4096: 115 us forward, 4.7 TB/s, 106 dgrad, 5.1), wgrad of few
// rows by its result (64 rows of them: 107 us, 5.0 TB/s), those of about a thousand rows by the unequal shares of some six workgroups a CU (1030 rows, 16
// experts of 1408 x 2048: 75 us each way, of which the MFMAs are half), small ones by the time that a K step takes from its loads to its last MFMA, which
// other workgroups of a CU have to fill: where there are few, the contraction is cut and a second kernel adds the parts (8 rows of 1024 x 1024: 40 ->
// 13 us).
#include <type_traits>

#include "products_internal.h"

namespace moe {
namespace products {
namespace {

typedef __attribute__((ext_vector_type(4))) float f32x4;

constexpr int kThreads = 256, kTileF = 64;
constexpr long kMostWorkgroups = 2048;

__host__ __device__ inline size_t output_size(int form, const Args& a) {
    return form == kWgrad ? (size_t)a.experts * a.n * a.k : (size_t)a.rows * (form == kForward ? a.n : a.k);
}

__device__ inline f32x4 load4(const float* p) { return *reinterpret_cast<const f32x4*>(p); }
__device__ inline void store4(float* p, f32x4 v) { *reinterpret_cast<f32x4*>(p) = v; }

// One operand of a tile.  ROWS: the contraction is contiguous, consecutive rows are `ld` apart; else rows are contiguous and consecutive c are
// `ld` apart.  CUT: the contraction may end inside a K step (the rows of an expert); c from `depth` on count as zeros.
// BK: c of a K step.
template <bool ROWS, int TILE, bool CUT, int BK>
struct Operand {
    static constexpr int kAll = TILE * BK / 4, kEach = kAll < kThreads ? 1 : kAll / kThreads;   // four numbers at a time
    static constexpr int kAcross = ROWS ? BK / 4 : TILE / 4;
    static constexpr int kLd = TILE + 4, kFloats = ROWS ? TILE * BK : BK * kLd;   // of a K step in LDS
    const float* at[kEach];   // this thread's of the next K step that is requested
    const float* base;        // CUT: some that exist
    size_t step;
    int c_left[2];            // CUT: c from the first of them to the end, of the next step in each slot
    f32x4 v[2][kEach];        // K steps on their way, one in each slot

    // What a row's units are exchanged by: the 16 rows of a fragment, read at one unit, are in 64 different banks.
    static __device__ int turn(int row) { return BK == 64 ? row & 15 : BK == 32 ? row / 2 & 7 : row / 4 & 3; }
    // `tile`: its element (row 0, c 0); `limit` rows of it exist (rows behind them repeat the last one); begin: first c, which is the step that goes to `first_slot`.
    __device__ void set(const float* tile, size_t ld, int limit, int begin, int depth, int first_slot) {
#pragma unroll
        for (int n = 0; n < kEach; ++n) {
            const int t = threadIdx.x + n * kThreads;
            const int row = ROWS ? min(t / kAcross, limit - 1) : t % kAcross * 4, c = begin + (ROWS ? t % kAcross * 4 : t / kAcross);
            at[n] = tile + (ROWS ? (size_t)row * ld + c : (size_t)c * ld + row);
        }
        base = tile;
        step = ROWS ? BK : BK * ld;
        const int c = depth - begin - (int)threadIdx.x / kAcross;
        c_left[0] = first_slot == 0 ? c : c - BK;
        c_left[1] = first_slot == 0 ? c - BK : c;
    }
    template <int SLOT>
    __device__ void load() {
#pragma unroll
        for (int n = 0; n < kEach; ++n) {
            v[SLOT][n] = load4(!CUT || c_left[SLOT] > n * (kThreads / kAcross) ? at[n] : base);
            at[n] += step;
        }
        c_left[SLOT] -= 2 * BK;
    }
    template <int SLOT>
    __device__ void stage(float* lds) const {
        if (kAll < kThreads && threadIdx.x >= kAll) return;
#pragma unroll
        for (int n = 0; n < kEach; ++n) {
            const int t = threadIdx.x + n * kThreads, a = t / kAcross, b = t % kAcross;
            const bool there = !CUT || c_left[SLOT] + 2 * BK > n * (kThreads / kAcross);
            *reinterpret_cast<f32x4*>(lds + (ROWS ? a * BK + ((b ^ turn(a)) * 4) : a * kLd + b * 4)) = there ? v[SLOT][n] : f32x4{0.f, 0.f, 0.f, 0.f};
        }
    }
    // This lane's four numbers (c half * 16 + 4 * (lane / 16) + 0 .. 3) of the fragment whose first row is `row`.
    __device__ static f32x4 fragment(const float* lds, int row, int half) {
        const int l = threadIdx.x & 63;
        if constexpr (ROWS) {
            return *reinterpret_cast<const f32x4*>(lds + row * BK + l % 16 * BK + (((l / 16 + half * 4) ^ turn(l % 16)) * 4));
        } else {
            f32x4 f;
#pragma unroll
            for (int m = 0; m < 4; ++m) f[m] = lds[(half * 16 + l / 16 * 4 + m) * kLd + l % 16 + row];
            return f;
        }
    }
};

// HEIGHT: rows of a tile, 64 or 16.  With `parts` > 1 workgroup (x, s) adds up part s of the contraction and stores it as part s of the scratch memory,
// laid out like the output.
template <int FORM, int HEIGHT>
__global__ __launch_bounds__(kThreads, 2) void product_kernel(Args a, int parts, float* scratch) {
    constexpr int kAcross = FORM == kWgrad ? 2 : 4;   // wavefronts across the features
    constexpr int kP = kTileF / 16 / kAcross, kQ = HEIGHT / 16 / (4 / kAcross);   // fragments of a wavefront
    constexpr int kBK = FORM == kWgrad ? 16 : FORM == kForward && HEIGHT == 16 ? 64 : 32;
    using P = Operand<FORM == kForward, kTileF, FORM == kWgrad, kBK>;
    using Q = Operand<FORM != kWgrad, HEIGHT, FORM == kWgrad, kBK>;
    __shared__ __attribute__((aligned(16))) float lds[2][P::kFloats + Q::kFloats];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int features = FORM == kForward ? a.n : a.k;
    const int f_tiles = features / kTileF;
    const int f0 = blockIdx.x % f_tiles * kTileF;
    const int m = blockIdx.x / f_tiles;
    int e, row0, rows, depth;
    P p;
    Q q;
    const float *p_base, *q_base;
    size_t q_ld, out_at;
    if constexpr (FORM == kWgrad) {
        const int n_tiles = a.n / HEIGHT;
        e = m / n_tiles;
        const int n0 = m % n_tiles * HEIGHT;
        int first, end;
        expert_rows(a, lane, first, end);
        first = __builtin_amdgcn_readlane(first, e);
        depth = __builtin_amdgcn_readlane(end, e) - first;
        if (depth == 0 && a.accumulate) return;   // (such an expert's gradient stays as it is; the parts of it are not read)
        rows = HEIGHT;
        q_base = static_cast<const float*>(a.q) + (size_t)first * a.n + n0;
        q_ld = a.n;
        p_base = static_cast<const float*>(a.p) + (size_t)first * a.k + f0;
        out_at = ((size_t)e * a.n + n0) * a.k + f0;
    } else {
        if (!find_row_tile(a, m, HEIGHT, e, row0, rows)) return;
        depth = FORM == kForward ? a.k : a.n;
        q_base = static_cast<const float*>(a.q) + (size_t)row0 * depth;
        q_ld = depth;
        p_base = static_cast<const float*>(a.p) + (size_t)e * a.n * a.k + (FORM == kForward ? (size_t)f0 * a.k : f0);
        out_at = (size_t)row0 * features + f0;
    }
    // This wavefront's part of the tile: row fragments wr, wr + kDown ...
    constexpr int kDown = 4 / kAcross;
    const int wf = wave % kAcross * (16 * kP), wr = wave / kAcross;
    f32x4 acc[kP][kQ];   // [feature fragment][row fragment]
#pragma unroll
    for (int i = 0; i < kP; ++i)
#pragma unroll
        for (int j = 0; j < kQ; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    const int all = (depth + kBK - 1) / kBK;
    const int begin = (int)((long)all * blockIdx.y / parts), steps = (int)((long)all * (blockIdx.y + 1) / parts);
    const int first_slot = steps - begin > 1 ? (steps - begin) & 1 : 0;
    p.set(p_base, a.k, kTileF, begin * kBK, depth, first_slot);
    q.set(q_base, q_ld, rows, begin * kBK, depth, first_slot);
    // All K steps, for `count` fragments of rows that exist.
    auto compute = [&](auto count) __attribute__((always_inline)) {
        constexpr int kCount = decltype(count)::value;
        auto request = [&](auto slot) __attribute__((always_inline)) {
            p.template load<decltype(slot)::value>();
            q.template load<decltype(slot)::value>();
        };
        auto step = [&](auto slot, int s, auto more) __attribute__((always_inline)) {
            float *lp = lds[s & 1], *lq = lp + P::kFloats;
            p.template stage<decltype(slot)::value>(lp);
            q.template stage<decltype(slot)::value>(lq);
            __syncthreads();   // (the other pair of stages is written after the next one, which everybody reaches behind its reads)
            if constexpr (decltype(more)::value) request(slot);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int half = 0; half < kBK / 16; ++half) {
                f32x4 fp[kP], fq[kCount];
#pragma unroll
                for (int i = 0; i < kP; ++i) fp[i] = P::fragment(lp, wf + i * 16, half);
#pragma unroll
                for (int j = 0; j < kCount; ++j) fq[j] = Q::fragment(lq, (wr + j * kDown) * 16, half);
#pragma unroll
                for (int c = 0; c < 4; ++c)
#pragma unroll
                    for (int j = 0; j < kCount; ++j)
#pragma unroll
                        for (int i = 0; i < kP; ++i) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(fp[i][c], fq[j][c], acc[i][j], 0, 0, 0);
            }
        };
        using Zero = std::integral_constant<int, 0>;
        using One = std::integral_constant<int, 1>;
        using Yes = std::true_type;
        using No = std::false_type;
        // Two steps are requested ahead, none behind the last one, and none under a branch: a compiler that has to expect both waits for all of them.
        int s = begin;
        if (steps - begin == 1) {
            request(Zero{});
            step(Zero{}, s, No{});
            return;
        }
        if ((steps - begin) & 1) {
            request(One{});
            request(Zero{});
            step(One{}, s++, Yes{});
        } else {
            request(Zero{});
            request(One{});
        }
        for (; s < steps - 2; s += 2) {
            step(Zero{}, s, Yes{});
            step(One{}, s + 1, Yes{});
        }
        step(Zero{}, s, No{});
        step(One{}, s + 1, No{});
    };
    if (begin < steps) {
        if constexpr (FORM == kWgrad || kQ == 1) {
            compute(std::integral_constant<int, kQ>{});
        } else {
            switch ((rows + 15) / 16) {
                case 1: compute(std::integral_constant<int, 1>{}); break;
                case 2: compute(std::integral_constant<int, 2>{}); break;
                case 3: compute(std::integral_constant<int, 3>{}); break;
                default: compute(std::integral_constant<int, 4>{}); break;
            }
        }
    }
    float* out = static_cast<float*>(a.out) + out_at;
    if (parts > 1) out = scratch + blockIdx.y * output_size(FORM, a) + out_at;
    if constexpr (FORM == kWgrad) {   // through LDS, so that a store is four whole rows
        constexpr int kLd = kTileF + 4;
        static_assert(sizeof(lds) >= HEIGHT * kLd * sizeof(float), "");
        float* const sums = lds[0];
        __syncthreads();
#pragma unroll
        for (int j = 0; j < kQ; ++j)
#pragma unroll
            for (int i = 0; i < kP; ++i) store4(sums + ((wr + j * kDown) * 16 + lane % 16) * kLd + wf + i * 16 + lane / 16 * 4, acc[i][j]);
        __syncthreads();
#pragma unroll
        for (int r = 0; r < HEIGHT; r += kThreads / 16) {
            const int row = r + threadIdx.x / 16, f = threadIdx.x % 16 * 4;
            f32x4* const to = reinterpret_cast<f32x4*>(out + (size_t)row * features + f);
            f32x4 v = load4(sums + row * kLd + f);
            if (parts > 1) {
                *to = v;
            } else {
                if (a.accumulate) v += __builtin_nontemporal_load(to);
                __builtin_nontemporal_store(v, to);
            }
        }
    } else {
#pragma unroll
        for (int j = 0; j < kQ; ++j) {
            const int row = j * 16 + lane % 16;
            if (row >= rows) continue;
#pragma unroll
            for (int i = 0; i < kP; ++i) store4(out + (size_t)row * features + wf + i * 16 + lane / 16 * 4, acc[i][j]);
        }
    }
}

// Adds the parts of everything that the experts have.
template <int FORM>
__global__ __launch_bounds__(kThreads) void join_parts_kernel(Args a, int parts, const float* __restrict__ scratch) {
    const int lane = threadIdx.x & 63;
    int first, end;
    expert_rows(a, lane, first, end);
    const size_t size = output_size(FORM, a), at = ((size_t)blockIdx.x * kThreads + threadIdx.x) * 4;
    if (FORM == kWgrad) {
        if (at >= size) return;
        const int e = (int)(at / ((size_t)a.n * a.k));   // (the same in the whole wavefront: a matrix is a multiple of 4096 numbers)
        if (a.accumulate && __builtin_amdgcn_readlane(end - first, __builtin_amdgcn_readfirstlane(e)) == 0) return;
    } else {
        const size_t features = FORM == kForward ? a.n : a.k;
        // rows from the first expert's first to the last one's end
        const size_t row = at / features;
        if (row < (size_t)__builtin_amdgcn_readlane(first, 0) || row >= (size_t)__builtin_amdgcn_readlane(end, a.experts - 1)) return;
    }
    f32x4 v = load4(scratch + at);
    for (int s = 1; s < parts; ++s) v += load4(scratch + s * size + at);
    float* to = static_cast<float*>(a.out) + at;
    if (FORM == kWgrad && a.accumulate) v += load4(to);
    store4(to, v);
}

template <int FORM, int HEIGHT>
hipError_t launch(const Args& a, float* scratch, hipStream_t stream) {
    const long f_tiles = (FORM == kForward ? a.n : a.k) / kTileF;
    const long m_tiles = FORM == kWgrad ? (long)a.experts * (a.n / HEIGHT) : most_row_tiles(a.rows, a.experts, HEIGHT);
    const long tiles = f_tiles * m_tiles;
    // Eight workgroups a CU, and 16 K steps each: with fewer the second kernel takes as long as what it saves.
    const int depth = FORM == kForward ? a.k : FORM == kDgrad ? a.n : (a.rows + a.experts - 1) / a.experts;
    long parts = kMostWorkgroups / tiles;
    if (parts > depth / 256) parts = depth / 256;
    if (parts > (long)(kScratchFloats / output_size(FORM, a))) parts = (long)(kScratchFloats / output_size(FORM, a));
    if (parts < 1) parts = 1;
    product_kernel<FORM, HEIGHT><<<dim3((unsigned)tiles, (unsigned)parts), dim3(kThreads), 0, stream>>>(a, (int)parts, scratch);
    hipError_t err = hipGetLastError();
    if (err != hipSuccess || parts == 1) return err;
    const size_t size = output_size(FORM, a);
    join_parts_kernel<FORM><<<dim3((unsigned)((size / 4 + kThreads - 1) / kThreads)), dim3(kThreads), 0, stream>>>(a, (int)parts, scratch);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_f32(Form form, const Args& a, void* workspace, hipStream_t stream) {
    float* scratch = static_cast<float*>(workspace);
    const bool low = a.rows <= 16 * a.experts;   // 64 rows, 8 experts of 4096 x 4096: 209 us in tiles of 64, 141 in tiles of 16
    switch (form) {
        case kForward: return low ? launch<kForward, 16>(a, scratch, stream) : launch<kForward, 64>(a, scratch, stream);
        case kDgrad: return low ? launch<kDgrad, 16>(a, scratch, stream) : launch<kDgrad, 64>(a, scratch, stream);
        default: return launch<kWgrad, 64>(a, scratch, stream);
    }
}

}  // namespace products
}  // namespace moe
