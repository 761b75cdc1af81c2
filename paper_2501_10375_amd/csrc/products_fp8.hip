// Grouped products of block-scaled e4m3 matrices on the CDNA4 matrix cores.
//
// y[row, feature] = sum over blocks b of 128 c of x_scale(row, b) * w_scale(feature / 128, b) * (sum over c in b of x(row, c) * w(feature, c)).
//
// A K step is a block, 128 bytes of a row, so that operand tiles look like those of the bf16 products (rows of 128 bytes,
// pieces of 16 exchanged so that reads are free of bank conflicts, straight from memory to LDS).  One v_mfma_f32_16x16x128_f8f6f4 is the sum
// over a block, which leaves its scale as the only thing to do between two of them: with the weights as the first operand a
// lane holds four features of one row, and as a wavefront's features are of one block of weights, one factor a lane serves
// all MFMAs of a row fragment.  Four fused multiply-adds an MFMA take 16 of its 32 cycles, on the SIMD's other pipe.  The instruction aligns eight
// products at a time to the largest one and keeps 13 bits behind its exponent (moe_products.h has the bound); the bf16 instruction, which would
// keep all, takes twice the cycles for the same products, and its operands would have to be converted first.
//
// That they are vector instructions sets the tile: their accumulators cannot be in AGPRs.  Eight wavefronts of 64 features x 96 rows (a
// tile of 256 x 192), two on a SIMD: 96 accumulators, the weights' fragments of this and the next K step and some of the rows' are the
// 256 registers that each has, and one's MFMAs run under the other's additions.
//
// LDS: three stages of weights, whose lines come from memory, two of rows, two of the scales of four K steps (of 192 rows and two blocks of
// weights).  A row's scales are 16 bytes of a line of their own, which cost the load path as much as a whole line of operands: four K steps'
// at a time they are a tenth of its work, one by one they were three tenths.
//
// What bounds it: MFMAs, additions and LDS reads alone run at 3.1 PFLOP/s, at 1.5 GHz on numbers with all their bits in use; with the lines
// on their way to LDS as well it is 2.3 at 6144 x 6144 x 16384 (538 us), 64 % of the cycles MFMAs at 1.7 GHz: the board is at its power limit, and what moves
// data costs clock.  (A tile of 256 x 160, which leaves room for three stages of rows: 1.99 at 60 % and 1.62 GHz.)  Few rows are a stream over the weights:
// 154 rows, 8 experts of 14336 x 4096 in 104 us, 4.6 TB/s.
#include "products_tiles.h"

namespace moe {
namespace products {
namespace {

typedef __attribute__((ext_vector_type(8))) int i32x8;
typedef __attribute__((ext_vector_type(4))) int i32x4;

constexpr int kStepC = 128, kTallest = 192;

struct Fp8Kernel {
    static constexpr int kThreads = 512;
    static constexpr int kF = 4;                       // fragments of 16 features a wavefront
    static constexpr int kPStage = 32768, kQStage = kTallest * 128, kSStage = 4096;
    static constexpr uint32_t kQBase = 3 * kPStage, kSBase = kQBase + 2 * kQStage;
    static constexpr int kLdsBytes = kSBase + 2 * kSStage;
    static constexpr uint32_t kNowhere = 0xc0000000u;  // a lane offset behind the end of every buffer
    static constexpr int kLate = 3;                    // MFMAs between one and the addition of its result

    typedef __attribute__((address_space(3))) const unsigned char* lds_ptr;

    static __device__ GG_INLINE void set_lds_target(uint32_t a) { asm volatile("s_mov_b32 m0, %0\n\ts_nop 0" ::"s"(a) : "memory"); }
    static __device__ GG_INLINE void load16(u32x4 d, uint32_t off) { asm volatile("buffer_load_dwordx4 %0, %1, 0 offen lds" ::"v"(off), "s"(d) : "memory"); }
    // d = the block's sum.  An asm statement keeps its place among the others and its result in VGPRs.  What the compiler does not know
    // is that it is an MFMA: a result is not touched for kLate MFMAs and the additions between them, 15 instructions (12 are
    // needed behind these eight passes), and settle() stands before the last ones; tests/test_products_isa.py reads the built kernel for it.
    static __device__ GG_INLINE void block_sum(f32x4& d, i32x8 a, i32x8 b) {
        asm volatile("v_mfma_f32_16x16x128_f8f6f4 %0, %1, %2, 0" : "=&v"(d) : "v"(a), "v"(b));
    }
    // acc += d * by (an asm statement as well: the compiler moves additions away from the MFMA whose registers they free)
    static __device__ GG_INLINE void add_scaled(float& acc, float d, float by) { asm volatile("v_fmac_f32 %0, %1, %2" : "+v"(acc) : "v"(d), "v"(by)); }
    static __device__ GG_INLINE void settle() { asm volatile("s_nop 15" ::: "memory"); }

    static constexpr int kStreamed = 2;   // cache policy of results: not kept in favour of operands
    // Waits for the first two K steps of an item, which were requested before the `stores` of the item before.
    static __device__ GG_INLINE void wait_first(int stores) {
        switch (stores) {
            case 0: gg::wait_vmcnt<0>(); break;
            case 2: gg::wait_vmcnt<2>(); break;
            case 4: gg::wait_vmcnt<4>(); break;
            case 6: gg::wait_vmcnt<6>(); break;
            case 8: gg::wait_vmcnt<8>(); break;
            case 10: gg::wait_vmcnt<10>(); break;
            case 12: gg::wait_vmcnt<12>(); break;
            case 16: gg::wait_vmcnt<16>(); break;
            case 20: gg::wait_vmcnt<20>(); break;
            default: gg::wait_vmcnt<24>(); break;
        }
    }

    template <class Decode>
    static __device__ GG_INLINE void run(const Args& a, float* scratch, Told* told, int piece_units, unsigned char* lds, Item cur, const Decode& decode) {
        const int N = a.n, K = a.k, kb = (K + 127) / 128, nb = (N + 127) / 128;
        const lds_ptr lds3 = (lds_ptr)lds;
        const uint32_t lds0 = (uint32_t)(uintptr_t)lds3;
        const int wave = uniform((int)threadIdx.x >> 6);
        const int wt = wave & 1, wq = wave >> 1;       // row group, feature group
        const uint32_t wave_lds = lds0 + (uint32_t)wave * 1024;
        auto next_of_3 = [](uint32_t s) GG_LAMBDA { return s == 2 ? 0u : s + 1; };

        // Load n of wavefront w covers rows n * 64 + w * 8 .. + 7, lane l the 16-byte piece that belongs at position l % 8 of row l / 8.
        // Scales: wavefronts 0 to 2 those of 64 rows each, 3 the weights' two.  (A load takes dwords at any dword's address, and checks each for the end.)
        uint32_t off[4];   // of both operands
        Buffer p, q, s;
        const int lane0 = threadIdx.x & 63;
#pragma unroll
        for (int n = 0; n < 4; ++n) {
            const int row = n * 64 + wave * 8 + (lane0 >> 3);
            off[n] = (uint32_t)row * (uint32_t)K + (uint32_t)gg::swizzled(row, lane0 & 7) * 16u;
        }
        const uint32_t s_off = wave < 3 || lane0 < 2 ? (uint32_t)((wave < 3 ? wave * 64 : 0) + lane0) * (uint32_t)kb * 4u : kNowhere;
        auto p_load = [&](uint32_t stage, int n) GG_LAMBDA {
            set_lds_target(wave_lds + stage * kPStage + n * 8192);
            load16(p.d, off[n]);
        };
        auto q_load = [&](uint32_t stage, int n) GG_LAMBDA {
            set_lds_target(wave_lds + kQBase + stage * kQStage + n * 8192);
            load16(q.d, off[n]);
        };
        auto s_load = [&](uint32_t stage) GG_LAMBDA {   // of the next four steps
            if (wave >= 4) return;
            set_lds_target(wave_lds + kSBase + stage * kSStage);
            load16(s.d, s_off);
            s.next_rows(16);
        };
        auto p_next = [&]() GG_LAMBDA { p.next_rows(kStepC); };
        auto q_next = [&]() GG_LAMBDA { q.next_rows(kStepC); };
        auto p_stage = [&](uint32_t stage) GG_LAMBDA {
#pragma unroll
            for (int n = 0; n < 4; ++n) p_load(stage, n);
            p_next();
        };
        auto q_stage = [&](uint32_t stage, int rows) GG_LAMBDA {
#pragma unroll
            for (int n = 0; n < 3; ++n)
                if (n * 64 + wave * 8 < rows) q_load(stage, n);
            q_next();
        };
        // The first two steps of an item.
        auto request_first = [&](const Item& t) GG_LAMBDA {
            const int block = t.c0 / kStepC;
            const uint8_t *pm = static_cast<const uint8_t*>(a.p), *qm = static_cast<const uint8_t*>(a.q);
            const int64_t at = (int64_t)t.f0 * K + t.c0;   // in the expert's matrix
            p.set_rows(pm + (size_t)t.expert * N * K + at, (int64_t)min(kTile, N - t.f0) * K - t.c0, t.k_steps);
            q.set_rows(qm + (size_t)t.row0 * K + t.c0, (int64_t)t.rows * K - t.c0, t.k_steps);
            const int f_block = t.f0 / 128;
            const float* sm = wave < 3 ? a.q_scales + (size_t)t.row0 * kb : a.p_scales + ((size_t)t.expert * nb + f_block) * kb;
            s.set_rows(sm + block, ((int64_t)(wave < 3 ? t.rows : min(2, nb - f_block)) * kb - block) * 4, (t.k_steps + 3) / 4);
            s_load(0);
            q_stage(0, t.rows);
            p_stage(0);
            q_stage(1, t.rows);
            p_stage(1);
        };

        int stores = 0;   // of the item before
        request_first(cur);
        for (int n = 1;; ++n) {
        int tid = threadIdx.x;   // (opaque: lane addresses are computed where they are used)
        asm volatile("" : "+v"(tid));
        const int lane = tid & 63;
        wait_first(stores);
        gg::lds_barrier();   // (the results of the item before went through the third stage, too)
        p_stage(2);

        // Fragments: 16 rows x 128 bytes.  Lane l holds row l % 16, pieces l / 16 and l / 16 + 4 (any 32 bytes of the block do, if both operands
        // take the same), at r * 128 + ((piece ^ ((r >> 1) & 7)) << 4).  Feature fragment j: features wq * 64 + j * 16; row fragment i: rows (2 i + wt) * 16.
        const int frow = lane & 15, fpiece = lane >> 4;
        const uint32_t in_row = (uint32_t)(frow * 128 + ((((frow >> 1) & 7) ^ fpiece) << 4));
        const uint32_t p_read = (uint32_t)(wq * 64) * 128 + in_row, q_read = kQBase + (uint32_t)wt * 2048 + in_row;
        const uint32_t x_read = kSBase + (uint32_t)(wt * 16 + frow) * 16, w_read = kSBase + 3 * 1024 + (uint32_t)(wq >> 1) * 16;
        auto fragment = [&](uint32_t at, int rows) GG_LAMBDA {
            typedef __attribute__((address_space(3))) const i32x4* piece;
            const i32x4 lo = *reinterpret_cast<piece>(lds3 + at + rows * 128), hi = *reinterpret_cast<piece>(lds3 + (at ^ 64u) + rows * 128);
            return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        };
        auto number = [&](uint32_t at) GG_LAMBDA { return *reinterpret_cast<__attribute__((address_space(3))) const float*>(lds3 + at); };

        Item next;
        bool more_items = false;
        auto tile = [&](auto tfe_c) GG_LAMBDA {
            constexpr int TFE = decltype(tfe_c)::value;
            constexpr int kM = kF * TFE;
            // Fragments of rows that a step begins with, those that it reads in its first part, and all that it reads in its second (of the next step).
            constexpr int kHeld = TFE < 2 ? TFE : 2, kFirst = TFE - kHeld, kSecond = kF + kHeld;
            constexpr int kTurn = kM * kFirst / (kFirst + kSecond);   // the slot at which the second part begins
            float acc[kF][TFE][4];
#pragma unroll
            for (int j = 0; j < kF; ++j)
#pragma unroll
                for (int i = 0; i < TFE; ++i)
#pragma unroll
                    for (int c = 0; c < 4; ++c) acc[j][i][c] = 0.f;
            i32x8 pf[2][kF], qf[2][TFE];
            float xs[2][TFE], ws[2];   // scales
            f32x4 d[kLate + 1];        // results that are not added yet
#pragma unroll
            for (int i = 0; i <= kLate; ++i) d[i] = f32x4{0.f, 0.f, 0.f, 0.f};

            // The last block of a row may have 64 numbers: what was loaded behind them (pieces 4 to 7) is cleared.
            const bool ragged = cur.depth < cur.k_steps * kStepC;
            int left = cur.k_steps;   // steps that are not computed yet
            auto clear_second_halves = [&](uint32_t p_at, uint32_t q_at) GG_LAMBDA {
                for (int x = tid; x < (kTile + kTallest) * 4; x += kThreads) {
                    const int row = x >> 2;   // weights, then rows (kTile is a multiple of the swizzle's period)
                    unsigned char* stage = lds + (row < kTile ? p_at * kPStage : kQBase + q_at * kQStage - kTile * 128);
                    *reinterpret_cast<u32x4*>(stage + row * 128 + gg::swizzled(row, 4 + (x & 3)) * 16) = u32x4{0, 0, 0, 0};
                }
                gg::lds_barrier();
            };
            auto add = [&](int m, float by) GG_LAMBDA {   // the result of the MFMA of slot m
#pragma unroll
                for (int c = 0; c < 4; ++c) add_scaled(acc[m % kF][m / kF][c], d[m % (kLate + 1)][c], by);
            };
            float by[TFE], by_before = 0.f;   // scales of the rows times those of the weights; of the last rows in the step before
            // Step kt: its MFMAs out of fragment buffer B, between them the reads of what is left of the step's rows, then, when step kt + 1 is there,
            // of its weights and first rows, and the requests of the rows and scales of kt + 2 and of the weights of kt + 3.
            uint32_t p_at = 0, q_at = 0, s_at = 0;   // stages of step kt; where its scales are behind those of step 0
            auto k_step = [&](auto buf) GG_LAMBDA {
                constexpr int B = decltype(buf)::value;
                const uint32_t p1 = next_of_3(p_at), q1 = q_at ^ 1;
                // four steps in a stage of scales
                const uint32_t s1 = B == 0 ? s_at + 4 : (s_at & 12) == 12 ? (s_at ^ kSStage) - 12 : s_at + 4;
                constexpr int kRowLoads = (TFE + 1) / 2, kLoads = kRowLoads + kF, kRest = kM - kTurn;
#pragma unroll
                for (int m = 0; m < kM; ++m) {
                    if (m == kTurn) {
                        // Outstanding, oldest first: weights of kt + 1, rows and scales of kt + 1, weights of kt + 2 (four loads).  At step 0 the stores of
                        // the item before come ahead of the last ones, and what is needed is there already.
                        if (left < cur.k_steps) gg::wait_vmcnt<4>();
                        gg::lds_barrier();
                        if (ragged && left == 2) clear_second_halves(p1, q1);
                    }
                    block_sum(d[m % (kLate + 1)], pf[B][m % kF], qf[B][m / kF]);
                    // (behind the last step there may be another row's scale, and zero times that need not be zero)
                    if (m % kF == 0) by[m / kF] = B == 0 || left > 0 ? xs[B][m / kF] * ws[B] : 0.f;
                    if (m >= kLate) add(m - kLate, by[(m - kLate) / kF]);
                    else add(m - kLate + kM, by_before);
                    if (m < kTurn) {
#pragma unroll
                        for (int x = 0; x < kFirst; ++x)
                            if (x * kTurn / (kFirst > 0 ? kFirst : 1) == m) {
                                qf[B][kHeld + x] = fragment(q_read + q_at * kQStage, (kHeld + x) * 32);
                                xs[B][kHeld + x] = number(x_read + s_at + (kHeld + x) * 512);
                            }
                    } else {
#pragma unroll
                        for (int x = 0; x < kSecond; ++x) {
                            if (kTurn + x * (kRest - 1) / kSecond != m) continue;
                            if (x < kF) {
                                pf[1 - B][x] = fragment(p_read + p1 * kPStage, x * 16);
                            } else {
                                qf[1 - B][x - kF] = fragment(q_read + q1 * kQStage, (x - kF) * 32);
                                xs[1 - B][x - kF] = number(x_read + s1 + (x - kF) * 512);
                                if (x == kF) ws[1 - B] = number(w_read + s1);
                            }
                        }
#pragma unroll
                        for (int x = 0; x < kLoads; ++x) {
                            if (kTurn + x * kRest / kLoads != m) continue;
                            if (x < kRowLoads) {
                                if (x * 2 + 2 <= TFE || wave < 4) q_load(q_at, x);   // 64 rows, or the last 32
                            } else {
                                if (B == 0 && x == kRowLoads && (s_at & 12) == 0) s_load(s_at == 0 ? 1u : 0u);
                                p_load(p_at, x - kRowLoads);
                            }
                        }
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
                by_before = by[TFE - 1];   // (the last MFMAs of this step are added in the next)
                --left;
                q_next();
                p_next();
                p_at = p1;
                q_at = q1;
                s_at = s1;
            };
            // step 0's weights and first rows
            if (ragged && left == 1) clear_second_halves(0, 0);
#pragma unroll
            for (int j = 0; j < kF; ++j) pf[0][j] = fragment(p_read, j * 16);
#pragma unroll
            for (int i = 0; i < kHeld; ++i) {
                qf[0][i] = fragment(q_read, i * 32);
                xs[0][i] = number(x_read + i * 512);
            }
            ws[0] = number(w_read);
            do {   // (two steps at a time, for the two fragment buffers; a step behind the last one adds zeros)
                k_step(std::integral_constant<int, 0>{});
                k_step(std::integral_constant<int, 1>{});
            } while (left > 0);
            settle();
#pragma unroll
            for (int m = kM - kLate; m < kM; ++m) add(m, by_before);

            // ---- the next item's first operands are requested before this one's results are stored
            more_items = decode(n, next);
            gg::wait_vmcnt<0>();
            gg::lds_barrier();   // every wavefront is done reading operand tiles; no load is outstanding
            if (more_items) request_first(next);

            // ---- epilogue: through LDS (4 KB a wavefront in the third stage of weights, which is requested later), so that stores are whole lines.
            // Every store is issued (what does not exist lies behind the end of the buffer), so that wait_first() can count them.
            unsigned char* own = lds + 2 * kPStage + wave * 4096;
            if (cur.piece < 0) {
                // [16 rows][64 features] bf16, rows of 128 bytes, 16-byte unit u of row r at swizzled(r, u)
                const int f = cur.f0 + wq * 64 + (lane & 7) * 8;
                const uint32_t stride = (uint32_t)N * 2u;
                const __amdgpu_buffer_rsrc_t out = __builtin_amdgcn_make_buffer_rsrc(static_cast<uint16_t*>(a.out) + (size_t)cur.row0 * N, 0,
                                                                                    (int)((uint32_t)cur.rows * stride), 0x00020000);
                const uint32_t to = f < N ? (uint32_t)(wt * 16 + (lane >> 3)) * stride + (uint32_t)f * 2u : kNowhere;
#pragma unroll
                for (int i = 0; i < TFE; ++i) {
#pragma unroll
                    for (int j = 0; j < kF; ++j) {
                        const uint2 pk = make_uint2(pack_bf16x2(acc[j][i][0], acc[j][i][1]), pack_bf16x2(acc[j][i][2], acc[j][i][3]));
                        *reinterpret_cast<uint2*>(own + frow * 128 + gg::swizzled(frow, j * 2 + (fpiece >> 1)) * 16 + (fpiece & 1) * 8) = pk;
                    }
                    gg::wave_order();
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const int lr = h * 8 + (lane >> 3);
                        const u32x4 v = *reinterpret_cast<const u32x4*>(own + lr * 128 + gg::swizzled(lr, lane & 7) * 16);
                        __builtin_amdgcn_raw_buffer_store_b128(v, out, to + (uint32_t)(i * 32 + h * 8) * stride, 0, kStreamed);
                    }
                    gg::wave_order();
                }
                stores = 2 * TFE;
            } else {
                // [16 rows][64 features] fp32, rows of 256 bytes, 16-byte unit u of row r at u ^ r
                const int col = wq * 64 + frow * 4;
                tell_cut(told, cur, (int64_t)cur.row0 * N + cur.f0, N);
                const __amdgpu_buffer_rsrc_t out = __builtin_amdgcn_make_buffer_rsrc(scratch + (size_t)cur.piece * piece_units * kUnitFloats, 0,
                                                                                    cur.rows * kTile * 4, 0x00020000);
                const uint32_t to = cur.f0 + col < N ? (uint32_t)((wt * 16 + fpiece) * kTile + col) * 4u : kNowhere;
#pragma unroll
                for (int i = 0; i < TFE; ++i) {
#pragma unroll
                    for (int j = 0; j < kF; ++j)
                        *reinterpret_cast<f32x4*>(own + frow * 256 + (((j * 4 + fpiece) ^ frow) << 4)) = f32x4{acc[j][i][0], acc[j][i][1], acc[j][i][2], acc[j][i][3]};
                    gg::wave_order();
#pragma unroll
                    for (int h = 0; h < 4; ++h) {
                        const int lr = h * 4 + fpiece;
                        const u32x4 v = *reinterpret_cast<const u32x4*>(own + lr * 256 + ((frow ^ lr) << 4));
                        __builtin_amdgcn_raw_buffer_store_b128(v, out, to + (uint32_t)((i * 32 + h * 4) * kTile) * 4u, 0, 0);
                    }
                    gg::wave_order();
                }
                stores = 4 * TFE;
            }
        };
        switch (uniform((cur.rows + 31) / 32)) {
            case 1: tile(std::integral_constant<int, 1>{}); break;
            case 2: tile(std::integral_constant<int, 2>{}); break;
            case 3: tile(std::integral_constant<int, 3>{}); break;
            case 4: tile(std::integral_constant<int, 4>{}); break;
            case 5: tile(std::integral_constant<int, 5>{}); break;
            default: tile(std::integral_constant<int, 6>{}); break;
        }
        if (!more_items) break;
        cur = next;
        }
    }
};

__global__ __launch_bounds__(Fp8Kernel::kThreads, 1) void product_fp8_kernel(Args a, float* scratch, Told* told) {
    __shared__ __attribute__((aligned(1024))) unsigned char lds[Fp8Kernel::kLdsBytes];
    Tiles<kForward, kStepC> list(a);
    const Plan plan = choose_tiles(list, gridDim.x, {kTallest, 60, 13});
    list.build(plan.height);
    const Items<kForward, kStepC> items(list, plan);
    if (blockIdx.x == 0 && threadIdx.x == 0) told->plan = items.plan;
    const Hand<kForward, kStepC> hand(list, items);
    Item item;
    if (!hand(0, item)) return;
    Fp8Kernel::run(a, scratch, told, plan.piece_units, lds, item, hand);
}

}  // namespace

hipError_t launch_fp8(const Args& a, void* workspace, hipStream_t stream) {
    float* scratch = static_cast<float*>(workspace);
    Told* told = reinterpret_cast<Told*>(static_cast<char*>(workspace) + kScratchBytes);
    const int grid = persistent_grid();
    product_fp8_kernel<<<grid, Fp8Kernel::kThreads, 0, stream>>>(a, scratch, told);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || !may_cut(kForward, a, kStepC, grid)) return e;
    join_pieces_kernel<false><<<kJoinWorkgroups, 256, 0, stream>>>(a.out, a.n, 0, scratch, told);
    return hipGetLastError();
}

}  // namespace products
}  // namespace moe
