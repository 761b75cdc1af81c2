// Grouped products of small size: the forward product and both gradients in bf16, the forward product in block-scaled e4m3; a workgroup for each tile of
// 64 features x 64 rows.
//
// The same operands as in the large tiles (products_bf16.h, products_fp8.hip): K steps of 128 bytes straight from memory to LDS, as rows or, transposed by the
// reads, as lines of 64 features, through buffer descriptors behind whose end lie zeros.  Four wavefronts take 32 x 32 each.  What counts here is the
// time from a call to its first load and the latency of a K step: nothing is planned, two or three steps are on their way while one is computed, and a
// step has one barrier.
//
// A K step takes 0.17 us, whether a CU has one workgroup or two: its 32 KB read from and 16 KB written to the LDS are 380 cycles.  (Tiles of 128 x 128, which
// read half as much for an MFMA, take 0.7 us, with one workgroup a CU.)  64 x 64 tiles of 32 steps on every CU: 9.5 us, the large tiles need 24.
#include "products_tiles.h"

namespace moe {
namespace products {
namespace {

using gg::bf16x8;

constexpr int kTile64 = 64, kStepC = 64, kThreads = 256, kStages = 4;
constexpr uint32_t kOperand = kTile64 * 128, kStage = 2 * kOperand;   // of a K step

typedef __attribute__((address_space(3))) const unsigned char* lds_ptr;
typedef __attribute__((ext_vector_type(4))) short i16x4;
typedef __attribute__((ext_vector_type(4))) int i32x4;
typedef __attribute__((ext_vector_type(8))) int i32x8;

// 16 bytes a lane from the buffer to LDS address `to` + lane * 16.
__device__ GG_INLINE void load_to(uint32_t to, u32x4 d, uint32_t off) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(to), "v"(off), "s"(d) : "memory");
}

// One operand of a tile: 64 rows whose contraction is contiguous, or (COLUMNS) lines of 64 rows, one for each c.  Either way 64 x 128 bytes a K step, two
// loads of 16 bytes a lane.
template <bool COLUMNS>
struct Operand {
    Buffer buffer;
    uint32_t off[2];

    // Rows: position p of row r holds piece p ^ (r / 2 % 8).  Columns: 32-byte units are exchanged, unit u of line c at u ^ exchange(c), so that the 32
    // lanes that a transposing read serves at a time (eight c, 32 bytes each: c % 8 < 4 of two neighbouring eights) find theirs in different banks.
    static __device__ GG_INLINE uint32_t exchange(int c) { return (uint32_t)((c >> 1 & 1) | (c >> 3 & 1) << 1); }
    // `rows`: that exist; ld: bytes from one row (c) to the next; steps, and c left (columns).
    __device__ GG_INLINE void set(const void* tile, int rows, uint32_t ld, int steps, int depth) {
#pragma unroll
        for (int n = 0; n < 2; ++n) {
            const int r = n * 32 + threadIdx.x / 8, piece = threadIdx.x % 8;
            off[n] = (uint32_t)r * ld + (COLUMNS ? (uint32_t)piece ^ exchange(r) << 1 : (uint32_t)gg::swizzled(r, piece)) * 16u;
        }
        if constexpr (COLUMNS) buffer.template set_columns<kStepC>(tile, depth, ld, ld - kTile64 * 2u, steps);
        else buffer.set_rows(tile, (int64_t)rows * ld, steps);
    }
    __device__ GG_INLINE void request(uint32_t to) {
        const uint32_t at = to + (uint32_t)uniform((int)threadIdx.x >> 6) * 1024;
#pragma unroll
        for (int n = 0; n < 2; ++n) load_to(at + n * 4096, buffer.d, off[n]);
        if constexpr (COLUMNS) buffer.template next_columns<kStepC>();
        else buffer.next_rows(128);
    }
    // Fragment of 16 rows from `row` on x 32 c (half `half` of the step): lane l holds row l % 16, c (l / 16) * 8 + 0 .. 7.
    static __device__ GG_INLINE bf16x8 fragment(lds_ptr lds, int row, int half) {
        const int lane = threadIdx.x & 63, i = lane & 15, block = lane >> 4;
        if constexpr (COLUMNS) {
            // lane i of a block fetches c i / 4 (of four), rows 4 (i % 4) .. + 3, and receives row i
            bf16x8 f;
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const int c = half * 32 + block * 8 + r * 4 + (i >> 2);
                const uint32_t at = (uint32_t)c * 128 + (((uint32_t)(row >> 4) ^ exchange(c)) << 5) + (uint32_t)(i & 3) * 8;
                reinterpret_cast<i16x4*>(&f)[r] =
                    __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4*)(uintptr_t)(uint32_t)(uintptr_t)(lds + at));
            }
            return f;
        } else {
            const int r = row + i;
            return *reinterpret_cast<__attribute__((address_space(3))) const bf16x8*>(lds + r * 128 + gg::swizzled(r, half * 4 + block) * 16);
        }
    }
};

// Results to LDS and from there to memory, so that a store is whole rows.  A result: lane l holds row l % 16 and features 4 * (l / 16) + 0 .. 3 of its fragment.
template <bool OUT32>
__device__ GG_INLINE void store_tile(const Args& a, unsigned char* lds, const f32x4 (&acc)[2][2], int wf, int wr, int rows, int features, size_t out_at) {
    constexpr int kLd = kTile64 + 4;
    const int lane = threadIdx.x & 63;
    gg::wait_vmcnt<0>();   // (no load may be on its way to LDS)
    gg::lds_barrier();
    float* const sums = reinterpret_cast<float*>(lds);
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int i = 0; i < 2; ++i) *reinterpret_cast<f32x4*>(sums + (wr + j * 16 + (lane & 15)) * kLd + wf + i * 16 + (lane >> 4) * 4) = acc[i][j];
    gg::lds_barrier();
    constexpr int kWide = OUT32 ? 4 : 8, kPass = kThreads * kWide / kTile64;   // features of a thread, rows of a pass
#pragma unroll
    for (int r = 0; r < kTile64; r += kPass) {
        const int row = r + threadIdx.x * kWide / kTile64, f = threadIdx.x * kWide % kTile64;
        if (row >= rows) break;
        const float* const from = sums + row * kLd + f;
        const size_t to = out_at + (size_t)row * features + f;
        f32x4 v = *reinterpret_cast<const f32x4*>(from);
        if constexpr (OUT32) {
            f32x4* const o = reinterpret_cast<f32x4*>(static_cast<float*>(a.out) + to);
            if (a.accumulate) v += __builtin_nontemporal_load(o);
            __builtin_nontemporal_store(v, o);
        } else {
            const f32x4 w = *reinterpret_cast<const f32x4*>(from + 4);
            const u32x4 pk = {pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(w[0], w[1]), pack_bf16x2(w[2], w[3])};
            __builtin_nontemporal_store(pk, reinterpret_cast<u32x4*>(static_cast<uint16_t*>(a.out) + to));
        }
    }
}

template <int FORM, bool OUT32>
__global__ __launch_bounds__(kThreads, 2) void product_small_kernel(Args a) {
    using P = Operand<FORM != kForward>;
    using Q = Operand<FORM == kWgrad>;
    __shared__ __attribute__((aligned(1024))) unsigned char lds[kStages * kStage];
    const lds_ptr lds3 = (lds_ptr)lds;
    const uint32_t lds0 = (uint32_t)(uintptr_t)lds3;
    const int lane = threadIdx.x & 63, wave = uniform((int)threadIdx.x >> 6);
    const int N = a.n, K = a.k, features = FORM == kForward ? N : K;
    const int f_tiles = features / kTile64, m = blockIdx.x / f_tiles, f0 = (blockIdx.x - m * f_tiles) * kTile64;
    const uint16_t *pm = static_cast<const uint16_t*>(a.p), *qm = static_cast<const uint16_t*>(a.q);
    P p;
    Q q;
    int e, row0, rows, depth, steps;
    size_t out_at;
    if constexpr (FORM == kWgrad) {
        const int n_tiles = N / kTile64;
        e = m / n_tiles;
        row0 = (m - e * n_tiles) * kTile64;
        rows = kTile64;
        int first, end;
        expert_rows(a, lane, first, end);
        first = __builtin_amdgcn_readlane(first, e);
        depth = __builtin_amdgcn_readlane(end, e) - first;
        if (depth == 0 && a.accumulate) return;   // (such an expert's gradient stays as it is)
        steps = (depth + kStepC - 1) / kStepC;
        p.set(pm + (size_t)first * K + f0, kTile64, K * 2, steps, depth);
        q.set(qm + (size_t)first * N + row0, kTile64, N * 2, steps, depth);
        out_at = ((size_t)e * N + row0) * K + f0;
    } else {
        if (!find_row_tile(a, m, kTile64, e, row0, rows)) return;
        depth = FORM == kForward ? K : N;
        steps = depth / kStepC;
        p.set(pm + (size_t)e * N * K + (FORM == kForward ? (size_t)f0 * K : (size_t)f0), kTile64, K * 2, steps, depth);
        q.set(qm + (size_t)row0 * depth, rows, depth * 2, steps, depth);
        out_at = (size_t)row0 * features + f0;
    }
    const int wf = (wave >> 1) * 32, wr = (wave & 1) * 32;
    f32x4 acc[2][2];   // [feature fragment][row fragment]
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < kStages - 1; ++s) {
        p.request(lds0 + s * kStage);
        q.request(lds0 + s * kStage + kOperand);
    }
    uint32_t at = 0, to = (kStages - 1) * kStage;
    for (int s = 0; s < steps; ++s) {
        gg::wait_vmcnt<8>();   // two steps behind this one (requests behind the last step return zeros)
        gg::lds_barrier();     // everybody's loads are there, and everybody has read the step before
        p.request(lds0 + to);
        q.request(lds0 + to + kOperand);
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            bf16x8 fp[2], fq[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) fp[i] = P::fragment(lds3 + at, wf + i * 16, half);
#pragma unroll
            for (int j = 0; j < 2; ++j) fq[j] = Q::fragment(lds3 + at + kOperand, wr + j * 16, half);
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int i = 0; i < 2; ++i) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fp[i], fq[j], acc[i][j], 0, 0, 0);
        }
        to = at;
        at = at == (kStages - 1) * kStage ? 0u : at + kStage;
    }
    store_tile<OUT32>(a, lds, acc, wf, wr, rows, features, out_at);
}

// acc += scales * block sums, K steps of a block of 128.  The scales of the whole tile go to LDS first.
__global__ __launch_bounds__(kThreads, 2) void product_small_fp8_kernel(Args a) {
    constexpr int kStages8 = 3;
    __shared__ __attribute__((aligned(1024))) unsigned char lds[kStages8 * kStage];
    __shared__ float x_scales[kMostSmallBlocks * kTile64], w_scales[kMostSmallBlocks];   // [block][row]
    const lds_ptr lds3 = (lds_ptr)lds;
    const uint32_t lds0 = (uint32_t)(uintptr_t)lds3;
    const int lane = threadIdx.x & 63, wave = uniform((int)threadIdx.x >> 6);
    const int N = a.n, K = a.k, steps = (K + 127) / 128;
    const int f_tiles = N / kTile64, m = blockIdx.x / f_tiles, f0 = (blockIdx.x - m * f_tiles) * kTile64;
    int e, row0, rows;
    if (!find_row_tile(a, m, kTile64, e, row0, rows)) return;
    Operand<false> p, q;
    p.set(static_cast<const uint8_t*>(a.p) + ((size_t)e * N + f0) * K, kTile64, K, steps, K);
    q.set(static_cast<const uint8_t*>(a.q) + (size_t)row0 * K, rows, K, steps, K);
#pragma unroll
    for (int s = 0; s < kStages8 - 1; ++s) {
        p.request(lds0 + s * kStage);
        q.request(lds0 + s * kStage + kOperand);
    }
    {
        const int row = threadIdx.x / 4;
        const float* const from = a.q_scales + (size_t)(row0 + min(row, rows - 1)) * steps;
        for (int s = threadIdx.x % 4; s < steps; s += 4) x_scales[s * kTile64 + row] = from[s];
        if ((int)threadIdx.x < steps) w_scales[threadIdx.x] = a.p_scales[((size_t)e * ((N + 127) / 128) + f0 / 128) * steps + threadIdx.x];
    }
    const int wf = (wave >> 1) * 32, wr = (wave & 1) * 32;
    f32x4 acc[2][2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    uint32_t at = 0, to = (kStages8 - 1) * kStage;
    for (int s = 0; s < steps; ++s) {
        gg::wait_vmcnt<4>();
        gg::lds_barrier();   // (the first one also for the scales)
        p.request(lds0 + to);
        q.request(lds0 + to + kOperand);
        // Fragment: 16 rows x 128 bytes, lane l holds row l % 16, pieces l / 16 and l / 16 + 4 (any 32 bytes do, if both operands take the same).  What
        // lies behind a last block of 64 is cleared.
        const bool half_block = s == steps - 1 && K % 128 != 0;
        auto fragment = [&](uint32_t operand, int row) GG_LAMBDA {
            const int r = row + (lane & 15), piece = lane >> 4;
            typedef __attribute__((address_space(3))) const i32x4* piece_ptr;
            const i32x4 lo = *reinterpret_cast<piece_ptr>(lds3 + at + operand + r * 128 + gg::swizzled(r, piece) * 16);
            i32x4 hi = *reinterpret_cast<piece_ptr>(lds3 + at + operand + r * 128 + gg::swizzled(r, piece + 4) * 16);
            if (half_block) hi = i32x4{0, 0, 0, 0};
            return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        };
        i32x8 fp[2], fq[2];
        float by[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) fp[i] = fragment(0, wf + i * 16);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            fq[j] = fragment(kOperand, wr + j * 16);
            by[j] = x_scales[s * kTile64 + wr + j * 16 + (lane & 15)] * w_scales[s];
        }
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const f32x4 d = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fp[i], fq[j], f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0, 0, 0, 0);
#pragma unroll
                for (int c = 0; c < 4; ++c) acc[i][j][c] = fmaf(d[c], by[j], acc[i][j][c]);
            }
        to = at;
        at = at == (kStages8 - 1) * kStage ? 0u : at + kStage;
    }
    store_tile<false>(a, lds, acc, wf, wr, rows, N, (size_t)row0 * N + f0);
}

template <int FORM, bool OUT32>
hipError_t launch(const Args& a, hipStream_t stream) {
    const long f_tiles = (FORM == kForward ? a.n : a.k) / kTile64;
    const long m_tiles = FORM == kWgrad ? (long)a.experts * (a.n / kTile64) : most_row_tiles(a.rows, a.experts, kTile64);
    product_small_kernel<FORM, OUT32><<<dim3((unsigned)(f_tiles * m_tiles)), kThreads, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_small_fp8(const Args& a, hipStream_t stream) {
    product_small_fp8_kernel<<<dim3((unsigned)(a.n / kTile64 * most_row_tiles(a.rows, a.experts, kTile64))), kThreads, 0, stream>>>(a);
    return hipGetLastError();
}

hipError_t launch_small(Form form, const Args& a, bool out_f32, hipStream_t stream) {
    switch (form) {
        case kForward: return launch<kForward, false>(a, stream);
        case kDgrad: return launch<kDgrad, false>(a, stream);
        default: return out_f32 ? launch<kWgrad, true>(a, stream) : launch<kWgrad, false>(a, stream);
    }
}

}  // namespace products
}  // namespace moe
