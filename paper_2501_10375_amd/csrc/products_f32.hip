// Grouped products on the fp32 matrix instructions: the forward product and both gradients of one tile kernel.
//
// A workgroup computes 64 features of up to 64 or 16 rows.  v_mfma_f32_16x16x4_f32 takes one number a lane, row lane % 16 and one of four c by
// lane / 16; which four is free as long as both operands take the same, so instruction m of 16 c takes c = 4 * (lane / 16) + m, and a fragment of 16 c is
// four consecutive numbers a lane.  An operand whose contraction is contiguous goes through LDS as it lies in memory, 16-byte units exchanged
// within a row, and a fragment is one ds_read_b128; one whose rows are (the weights of dgrad, both operands of wgrad) as [c][row], four
// ds_read_b32 whose four c are 16 banks apart.  The features are the instruction's first operand, so that a lane ends up with
// four consecutive ones of a row.
//
// Forward and dgrad: each wavefront 16 features of all rows, so that a ragged tile costs what its groups of 16 rows cost; K steps of 32, two requested ahead
// (the forward product of few rows: of 64, a row's 256 bytes at a time: 64 rows, 8 experts of 4096 x 4096 136 -> 121 us).  wgrad: 32 x 32 each; K steps of 16, four
// ahead, as its contraction may be a few rows; whole rows of the result leave through LDS past the caches.
//
// Large products are bound by the MFMAs (1024 rows, 4096 x 4096: 113 TFLOP/s forward, 120 dgrad, 110 wgrad; a library product of 4096^3 reaches 150), those of
// few rows by the weights (8 rows, 8 experts of 4096 x 4096: 117 us forward, 102 dgrad, 5.2 TB/s), wgrad of few rows by its result (64 rows of them: 111 us,
// 4.8 TB/s), small ones by the time that a K step takes from its loads to its last MFMA, which
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
// BK: c of a K step, AHEAD: steps that are requested ahead.
template <bool ROWS, int TILE, bool CUT, int BK, int AHEAD>
struct Operand {
    static constexpr int kAll = TILE * BK / 4, kEach = kAll < kThreads ? 1 : kAll / kThreads;   // four numbers at a time
    static constexpr int kAcross = ROWS ? BK / 4 : TILE / 4;
    static constexpr int kLd = TILE + 4, kFloats = ROWS ? TILE * BK : BK * kLd;   // of a K step in LDS
    const float* at[kEach];   // this thread's of the next K step that is requested
    size_t step;
    int c_left;               // CUT: c from the first of them to the end
    f32x4 v[AHEAD][kEach];    // K steps on their way

    // What a row's units are exchanged by: the 16 rows of a fragment, read at one unit, are in 64 different banks.
    static __device__ int turn(int row) { return BK == 64 ? row & 15 : BK == 32 ? row / 2 & 7 : row / 4 & 3; }
    // `base`: element (row 0, c 0) of the tile, of which `limit` rows exist (rows behind them repeat the last one), begin: first c.
    __device__ void set(const float* base, size_t ld, int limit, int begin, int depth) {
#pragma unroll
        for (int n = 0; n < kEach; ++n) {
            const int t = threadIdx.x + n * kThreads;
            const int row = ROWS ? min(t / kAcross, limit - 1) : t % kAcross * 4, c = begin + (ROWS ? t % kAcross * 4 : t / kAcross);
            at[n] = base + (ROWS ? (size_t)row * ld + c : (size_t)c * ld + row);
        }
        step = ROWS ? BK : BK * ld;
        c_left = depth - begin - threadIdx.x / kAcross;
    }
    template <int SLOT>
    __device__ void load() {
#pragma unroll
        for (int n = 0; n < kEach; ++n) {
            v[SLOT][n] = f32x4{0.f, 0.f, 0.f, 0.f};
            if ((!CUT || c_left > n * (kThreads / kAcross)) && (kAll >= kThreads || threadIdx.x < kAll)) v[SLOT][n] = load4(at[n]);
            at[n] += step;
        }
        if (CUT) c_left -= BK;
    }
    template <int SLOT>
    __device__ void stage(float* lds) const {
        if (kAll < kThreads && threadIdx.x >= kAll) return;
#pragma unroll
        for (int n = 0; n < kEach; ++n) {
            const int t = threadIdx.x + n * kThreads, a = t / kAcross, b = t % kAcross;
            *reinterpret_cast<f32x4*>(lds + (ROWS ? a * BK + ((b ^ turn(a)) * 4) : a * kLd + b * 4)) = v[SLOT][n];
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
    constexpr bool kFew = FORM == kForward && HEIGHT == 16;
    constexpr int kBK = FORM == kWgrad ? 16 : kFew ? 64 : 32, kAhead = FORM == kWgrad ? 4 : 2;
    using P = Operand<FORM == kForward, kTileF, FORM == kWgrad, kBK, kAhead>;
    using Q = Operand<FORM != kWgrad, HEIGHT, FORM == kWgrad, kBK, kAhead>;
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
    int fragments = FORM == kWgrad ? kQ : (rows + 15) / 16;   // of rows that exist
    // (not a constant for the compiler: the branch keeps the MFMAs of one fragment ahead of the reads of the next, 4 % of wgrad's time)
    if (FORM == kWgrad) asm("" : "+s"(fragments));
    f32x4 acc[kP][kQ];   // [feature fragment][row fragment]
#pragma unroll
    for (int i = 0; i < kP; ++i)
#pragma unroll
        for (int j = 0; j < kQ; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    const int all = (depth + kBK - 1) / kBK;
    const int begin = (int)((long)all * blockIdx.y / parts), steps = (int)((long)all * (blockIdx.y + 1) / parts);
    p.set(p_base, a.k, kTileF, begin * kBK, depth);
    q.set(q_base, q_ld, rows, begin * kBK, depth);
    auto request = [&](auto slot, int s) __attribute__((always_inline)) {
        if (s >= steps) return;
        p.template load<decltype(slot)::value>();
        q.template load<decltype(slot)::value>();
    };
    auto step = [&](auto slot, int s) __attribute__((always_inline)) {
        float *lp = lds[s & 1], *lq = lp + P::kFloats;
        p.template stage<decltype(slot)::value>(lp);
        q.template stage<decltype(slot)::value>(lq);
        __syncthreads();   // (the other pair of stages is written after the next one, which everybody reaches behind its reads)
        request(slot, s + kAhead);
#pragma unroll
        for (int half = 0; half < kBK / 16; ++half) {
            f32x4 fp[kP], fq[kQ];
#pragma unroll
            for (int i = 0; i < kP; ++i) fp[i] = P::fragment(lp, wf + i * 16, half);
#pragma unroll
            for (int j = 0; j < kQ; ++j) fq[j] = Q::fragment(lq, (wr + j * kDown) * 16, half);
#pragma unroll
            for (int j = 0; j < kQ; ++j) {
                if (j >= fragments) break;
#pragma unroll
                for (int c = 0; c < 4; ++c)
#pragma unroll
                    for (int i = 0; i < kP; ++i) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(fp[i][c], fq[j][c], acc[i][j], 0, 0, 0);
            }
        }
    };
    using std::integral_constant;
    request(integral_constant<int, 0>{}, begin);
    request(integral_constant<int, 1>{}, begin + 1);
    if constexpr (kAhead == 4) {
        request(integral_constant<int, 2>{}, begin + 2);
        request(integral_constant<int, 3>{}, begin + 3);
    }
    for (int s = begin; s < steps; s += kAhead) {
        step(integral_constant<int, 0>{}, s);
        if (s + 1 < steps) step(integral_constant<int, 1>{}, s + 1);
        if constexpr (kAhead == 4) {
            if (s + 2 < steps) step(integral_constant<int, 2>{}, s + 2);
            if (s + 3 < steps) step(integral_constant<int, 3>{}, s + 3);
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
