// Grouped products of bf16 matrices on the CDNA4 matrix cores (device code): the forward product and both gradients.
//
// out[row, feature] = sum over c of q(row, c) * p(feature, c), see Form.  The kernel is built like the one of the expert GEMMs
// (grouped_gemm_bf16.h: tiles of 256 x 256 on four wavefronts of 128 x 128, accumulators in the AGPRs, 16x16x32 MFMAs with at most two other
// instructions between them, operand tiles straight from memory to LDS, three stages of p and two of q, 64 c a K step), for
// operands that lie in memory either way:
//   rows     the contraction is contiguous (x, dy and the weights of the forward product): a K step is 256 rows of 128 bytes, a
//            fragment of 16 rows x 32 c is read with ds_read_b128
//   columns  the rows are contiguous and c goes down the memory (the weights of dgrad, both operands of wgrad): a K step is 64
//            lines of 512 bytes, and a fragment is read with two ds_read_b64_tr_b16, in which 16 lanes hand 4 x 16 numbers
//            over transposed: nothing is transposed in memory, and a line of LDS is a line of memory
// Both are loaded through buffer descriptors that begin at the K step and end at the last byte of the tile's operand, so
// that what lies behind it (rows of a ragged tile, the end of an expert's rows in wgrad) arrives as zeros without being read.
//
// What bounds it: large products the MFMAs at the board's power limit (8192^3: forward and dgrad 704 us, 1.56 PFLOP/s, wgrad into fp32 755 us; a library
// product 1.63 and, of the dgrad form, 1.40), a skewed prompt also its ragged tiles (8192 rows, 8 experts of 4096 x 14336: 725 us, 1.33 PFLOP/s, MFMAs 73 % of
// the cycles at 1.78 GHz).  Few rows: the weights (512 rows, 8 experts of 14336 x 4096: 182 us, 5.2 TB/s).  wgrad: its result, where there are few rows (64 each,
// 8 experts of 14336 x 4096, fp32: 335 us, 5.6 TB/s); with 1024 rows (915 us) a tile's 256 KB, which its CU's part of the L2 takes in some 10 000 cycles
// after 16 K steps of 2 900, hold the CU up for a fifth of the time.  (Workgroups that begin at different times, so that fewer store at once, make no
// difference: the time that they save comes back as clock.)
#pragma once

#include "products_tiles.h"

namespace moe {
namespace products {

using gg::bf16x8;

constexpr int kStepC = 64;

// One tile at a time, see the top of this file.  OUT32: whole tiles are stored in fp32 (wgrad), else in bf16.
template <int FORM, bool OUT32>
struct TileKernel {
    static constexpr bool kPCols = FORM != kForward, kQCols = FORM == kWgrad;
    static constexpr int kThreads = 256;
    static constexpr int kF = 8;                      // fragments of 16 features a wavefront
    static constexpr int kStage = 32768;              // a K step of one operand
    static constexpr uint32_t kQBase = 3 * kStage;    // p: three stages from 0, q: two from here
    static constexpr int kLdsBytes = 5 * kStage;

    typedef __attribute__((address_space(3))) const unsigned char* lds_ptr;
    typedef __attribute__((ext_vector_type(4))) short i16x4;
    using Yes = std::true_type;
    using No = std::false_type;

    // M0 (the LDS address of the load that follows behind some other instruction) ...
    static __device__ GG_INLINE void set_lds_target(uint32_t to) { asm volatile("s_mov_b32 m0, %0" ::"s"(to) : "memory"); }
    // ... and the load itself: 16 bytes a lane from the buffer to M0 + lane * 16.
    static __device__ GG_INLINE void load_lane(u32x4 d, uint32_t off) { asm volatile("buffer_load_dwordx4 %0, %1, 0 offen lds" ::"v"(off), "s"(d) : "memory"); }
    static __device__ GG_INLINE void load_to(uint32_t to, u32x4 d, uint32_t off) {
        set_lds_target(to);
        asm volatile("s_nop 0" ::: "memory");
        load_lane(d, off);
    }
    static constexpr uint32_t kNowhere = 0xc0000000u;  // a lane offset behind the end of every buffer
    // Cache policy of results (the nt bit): they are not kept in favour of operands.  wgrad of 8 x 14336 x 4096: 512 rows an expert in fp32 691 ->
    // 630 us, 64 rows in bf16 244 -> 198.
    static constexpr int kStreamed = 2;
    // Waits for the first two K steps of an item, which were requested before the `stores` of the item before.
    // (The counter has six bits: with 64 behind them, what it can wait for is enough.)
    static __device__ GG_INLINE void wait_first(int stores) {
        switch (stores) {
            case 0: gg::wait_vmcnt<0>(); break;
            case 4: gg::wait_vmcnt<4>(); break;
            case 8: gg::wait_vmcnt<8>(); break;
            case 12: gg::wait_vmcnt<12>(); break;
            case 16: gg::wait_vmcnt<16>(); break;
            case 20: gg::wait_vmcnt<20>(); break;
            case 24: gg::wait_vmcnt<24>(); break;
            case 32: gg::wait_vmcnt<32>(); break;
            case 40: gg::wait_vmcnt<40>(); break;
            case 48: gg::wait_vmcnt<48>(); break;
            case 56: gg::wait_vmcnt<56>(); break;
            default: gg::wait_vmcnt<63>(); break;
        }
    }
    // See Gemm::mfma_acc() of the expert GEMMs for why the MFMAs are asm statements, and settle() and pin() around them.
    static __device__ GG_INLINE void mfma_acc(f32x4& acc, bf16x8 a, bf16x8 b) {
        asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(acc) : "v"(a), "v"(b));
    }
    static __device__ GG_INLINE void settle() { asm volatile("s_nop 15\n\ts_nop 15" ::: "memory"); }
    template <int TFE>
    static __device__ GG_INLINE void pin(f32x4 (&acc)[kF][TFE]) {
#pragma unroll
        for (int j = 0; j < kF; ++j)
#pragma unroll
            for (int i = 0; i < TFE; ++i) asm volatile("" : "+a"(acc[j][i]));
    }
    static __device__ GG_INLINE float from_acc(float a) {
        float v;
        asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(v) : "a"(a));
        return v;
    }

    // Half a fragment (4 c of 16 rows) out of a column stage.
    static __device__ GG_INLINE i16x4 read_turned(lds_ptr p) {
        return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4*)(uintptr_t)(uint32_t)(uintptr_t)p);
    }

    // decode(n, Item&): this workgroup's n-th item, false if it has fewer.
    template <class Decode>
    static __device__ GG_INLINE void run(const Args& a, float* scratch, Told* told, int piece_units, unsigned char* lds, Item cur, const Decode& decode) {
        const int N = a.n, K = a.k;
        const int features = FORM == kForward ? N : K;
        const lds_ptr lds3 = (lds_ptr)lds;
        const uint32_t lds0 = (uint32_t)(uintptr_t)lds3;
        const int wave = uniform((int)threadIdx.x >> 6);
        const int wt = wave & 1, wq = wave >> 1;      // row group, feature group
        const uint32_t wave_lds = lds0 + (uint32_t)wave * 1024;

        // ---- staging.  Rows: load n of wavefront w covers rows n * 32 + w * 8 .. + 7, lane l the 16-byte piece that belongs at
        // position l % 8 of row l / 8.  Columns: c n * 8 + w * 2 and the next one, lane l the piece that belongs at position l % 32 of
        // line l / 32; there 32-byte units are exchanged, unit u of line c at u ^ (c % 4 + 4 (c / 8 % 2)), so that the 32 lanes that a
        // transposing read serves at a time (eight c, 32 bytes each) find their units in different banks.
        const uint32_t p_ld = (uint32_t)K * 2u, q_ld = (uint32_t)(FORM == kForward ? K : N) * 2u;
        uint32_t p_off[8], q_off[8];
        {
            const int lane = threadIdx.x & 63;
#pragma unroll
            for (int n = 0; n < 8; ++n) {
                const int row = n * 32 + wave * 8 + (lane >> 3), c = n * 8 + wave * 2 + (lane >> 5);
                const uint32_t in_row = (uint32_t)gg::swizzled(row, lane & 7) * 16u;
                const uint32_t in_line = (uint32_t)((lane & 31) ^ (((c & 3) | ((c >> 3) & 1) << 2) << 1)) * 16u;
                p_off[n] = kPCols ? (uint32_t)c * p_ld + in_line : (uint32_t)row * p_ld + in_row;
                q_off[n] = kQCols ? (uint32_t)c * q_ld + in_line : (uint32_t)row * q_ld + in_row;
            }
        }
        Buffer p, q;
        auto p_next = [&]() GG_LAMBDA {
            if constexpr (kPCols) p.template next_columns<kStepC>();
            else p.next_rows(kStepC * 2);
        };
        auto q_next = [&]() GG_LAMBDA {
            if constexpr (kQCols) q.template next_columns<kStepC>();
            else q.next_rows(kStepC * 2);
        };
        auto p_stage = [&](uint32_t stage) GG_LAMBDA {
#pragma unroll
            for (int n = 0; n < 8; ++n) load_to(wave_lds + stage + n * 4096, p.d, p_off[n]);
            p_next();
        };
        auto q_stage = [&](uint32_t stage, int rows) GG_LAMBDA {
#pragma unroll
            for (int n = 0; n < 8; ++n)
                if (kQCols || n * 32 < rows) load_to(wave_lds + kQBase + stage + n * 4096, q.d, q_off[n]);
            q_next();
        };
        // The first two K steps of an item, in four parts.
        auto request = [&](int part, const Item& t) GG_LAMBDA {
            if (part == 0) {
                const uint16_t *pm = static_cast<const uint16_t*>(a.p), *qm = static_cast<const uint16_t*>(a.q);
                if constexpr (FORM == kWgrad) {
                    p.template set_columns<kStepC>(pm + (size_t)t.c0 * K + t.f0, t.depth, p_ld, (uint32_t)t.f0 * 2u, t.k_steps);
                    q.template set_columns<kStepC>(qm + (size_t)t.c0 * N + t.row0, t.depth, q_ld, (uint32_t)t.row0 * 2u, t.k_steps);
                } else {
                    const uint16_t* matrix = pm + (size_t)t.expert * N * K;
                    if constexpr (kPCols) p.template set_columns<kStepC>(matrix + (size_t)t.c0 * K + t.f0, t.depth, p_ld, (uint32_t)t.f0 * 2u, t.k_steps);
                    else p.set_rows(matrix + (size_t)t.f0 * K + t.c0, ((int64_t)min(kTile, N - t.f0) * K - t.c0) * 2, t.k_steps);
                    const int ld = FORM == kForward ? K : N;
                    q.set_rows(qm + (size_t)t.row0 * ld + t.c0, ((int64_t)t.rows * ld - t.c0) * 2, t.k_steps);
                }
            }
            if (part % 2 == 0) p_stage(part / 2 * kStage);
            else q_stage(part / 2 * kStage, t.rows);
        };
        auto request_first = [&](const Item& t) GG_LAMBDA {
#pragma unroll
            for (int part = 0; part < 4; ++part) request(part, t);
        };

        int stores = 0;   // of the item before, behind the requests of this one
        request_first(cur);
        for (int n = 1;; ++n) {
        int tid = threadIdx.x;   // (opaque: lane addresses are computed where they are used)
        asm volatile("" : "+v"(tid));
        const int lane = tid & 63;
        wait_first(stores);
        gg::lds_barrier();

        // ---- fragments.  Rows: 16 rows x 32 c, lane l holds row l % 16, piece l / 16 of the half K step, at r * 128 + ((piece ^ ((r >> 1) & 7))
        // << 4).  Columns: in each of two reads, block l / 16 of lanes takes 4 c of the half K step, c = (l / 16) * 8 + 4 * read; lane i of it fetches
        // c i / 4, rows 4 * (i % 4) .. + 3 and receives row i.  Feature fragment j: features wq * 128 + j * 16; row fragment i: rows (2 i + wt) * 16.
        const int frow = lane & 15, fpiece = lane >> 4;
        const uint32_t in_row = (uint32_t)(frow * 128 + ((((frow >> 1) & 7) ^ fpiece) << 4));
        const uint32_t in_cols = (uint32_t)((fpiece * 8 + (frow >> 2)) * 512 + (frow & 3) * 8) + (uint32_t)(((frow >> 2) | (fpiece & 1) << 2) << 5);
        const uint32_t p_read = kPCols ? in_cols ^ (uint32_t)(wq << 8) : (uint32_t)(wq * 128) * 128 + in_row;
        const uint32_t q_read = kQCols ? in_cols ^ (uint32_t)(wt << 5) : (uint32_t)wt * 2048 + in_row;
        auto fragment = [&](auto cols, uint32_t read, uint32_t stage, int half, int row16) GG_LAMBDA {
            if constexpr (decltype(cols)::value) {
                const lds_ptr at = lds3 + ((read ^ (uint32_t)(row16 << 5)) + stage);
                const i16x4 lo = read_turned(at + half * 16384), hi = read_turned(at + half * 16384 + 2048);
                bf16x8 f;
                reinterpret_cast<i16x4*>(&f)[0] = lo;
                reinterpret_cast<i16x4*>(&f)[1] = hi;
                return f;
            } else {
                return *reinterpret_cast<__attribute__((address_space(3))) const bf16x8*>(lds3 + ((read ^ (uint32_t)(half << 6)) + stage) + row16 * 2048);
            }
        };

        Item next;
        bool more_items = false;
        // The whole tile for TFE valid groups of 32 rows, from the accumulators to the stores (see the expert GEMMs).
        auto tile = [&](auto tfe_c) GG_LAMBDA {
            constexpr int TFE = decltype(tfe_c)::value;
            f32x4 acc[kF][TFE];  // [feature fragment][row fragment]
#pragma unroll
            for (int j = 0; j < kF; ++j)
#pragma unroll
                for (int i = 0; i < TFE; ++i) acc[j][i] = f32x4{0.f, 0.f, 0.f, 0.f};
            pin(acc);
            settle();

            constexpr int kM = kF * TFE, kR = kF + TFE, kQLoads = kQCols ? 8 : TFE, kLoads = kQLoads + 8;
            bf16x8 pf[2][kF], qf[2][TFE];
            // Half a K step: the MFMAs of fragment buffer mbuf, between them the LDS reads of half `half` of the stages p_at and q_at
            // into buffer 1 - mbuf, and the loads of one operand (LOADS 1: q, 2: p) for a later K step into the stage `to`.
            auto half_step = [&](auto mfma, auto mbuf_c, auto reads, int half, uint32_t p_at, uint32_t q_at, auto loads, uint32_t to) GG_LAMBDA {
                constexpr int mbuf = decltype(mbuf_c)::value, rbuf = 1 - mbuf, LOADS = decltype(loads)::value;
                constexpr int n_loads = LOADS == 1 ? kQLoads : 8;
                constexpr int read_slots = kM - kM / 8;   // the last reads get some MFMAs' time before they are used
#pragma unroll
                for (int m = 0; m < kM; ++m) {
                    // x of n things over `of` slots goes into slot x * of / n: a load at most, up to two reads
                    const int l = (m * n_loads + kM - 1) / kM, r = (m * kR + read_slots - 1) / read_slots;
                    const bool load = LOADS != 0 && l < n_loads && l * kM / n_loads == m;
                    if (load) set_lds_target(wave_lds + (LOADS == 1 ? kQBase : 0) + to + l * 4096);
                    if constexpr (decltype(mfma)::value) mfma_acc(acc[m % kF][m / kF], pf[mbuf][m % kF], qf[mbuf][m / kF]);
                    auto read = [&](int x) GG_LAMBDA {
                        if (!decltype(reads)::value || x >= kR || x * read_slots / kR != m) return;
                        if (x < kF) pf[rbuf][x] = fragment(std::bool_constant<kPCols>{}, p_read, p_at, half, x);
                        else qf[rbuf][x - kF] = fragment(std::bool_constant<kQCols>{}, q_read, q_at + kQBase, half, (x - kF) * 2);
                    };
                    read(r);
                    read(r + 1);
                    if (load) {
                        load_lane(LOADS == 1 ? q.d : p.d, LOADS == 1 ? q_off[l] : p_off[l]);
                        if (l == n_loads - 1) {
                            if constexpr (LOADS == 1) q_next();
                            else p_next();
                        }
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
            };
            using Buf0 = std::integral_constant<int, 0>;
            using Buf1 = std::integral_constant<int, 1>;
            using None = std::integral_constant<int, 0>;
            using LoadQ = std::integral_constant<int, 1>;
            using LoadP = std::integral_constant<int, 2>;

            // First and second halves of the K steps in turn; while one is computed the next is read.  p of a step is requested in the first half of the one
            // two before it, q in the second half.
            uint32_t p_at = 0, q_at = 0, p_to = 2 * kStage;           // stages of K step kt, and where p of kt + 2 goes
            half_step(No{}, Buf1{}, Yes{}, 0, p_at, q_at, None{}, 0u);
            half_step(Yes{}, Buf0{}, Yes{}, 1, p_at, q_at, LoadP{}, p_to);
            gg::lds_barrier();   // (step 1 is there: the stores of the item before are not waited for yet)
            for (int kt = 0; kt < cur.k_steps - 1; ++kt) {
                const uint32_t p1 = p_at == 2 * kStage ? 0u : p_at + kStage, q1 = q_at ^ kStage;
                p_to = p_at;     // nobody reads step kt's stages any more
                half_step(Yes{}, Buf1{}, Yes{}, 0, p1, q1, LoadQ{}, q_at);
                half_step(Yes{}, Buf0{}, Yes{}, 1, p1, q1, LoadP{}, p_to);
                // Outstanding, oldest first: p of kt + 2, q of kt + 2, p of kt + 3 (eight loads).
                gg::wait_vmcnt<8>();
                gg::lds_barrier();
                p_at = p1;
                q_at = q1;
            }
            half_step(Yes{}, Buf1{}, No{}, 0, 0u, 0u, None{}, 0u);
            settle();
            pin(acc);

            more_items = decode(n, next);
            gg::wait_vmcnt<0>();
            gg::lds_barrier();   // every wavefront is done reading operand tiles; no load is outstanding

            // ---- epilogue: through LDS (8 KB a wavefront in the third stage of p, which is requested later), so that stores are whole lines.
            // An MFMA result: lane l holds row l % 16 of its fragment and features 4 * (l / 16) + 0 .. 3.  Every store is issued, whether its rows
            // exist or not (what does not lies behind the end of the buffer), so that wait_first() can count those behind the last request.
            unsigned char* own = lds + 2 * kStage + wave * 8192;
            if (!OUT32 && cur.piece < 0) {
                // [16 rows][128 features] bf16, rows of 256 bytes, 16-byte unit u of row r at u ^ r, in two places in turn.  The next item's first operands are
                // requested a part ahead of each of the first four fragments' stores.  (All ahead of the first one, and one place, wgrad of 64 experts of
                // 1408 x 2048: 64 rows each 88 us, 128 rows 101; like this 82 and 97.  In fp32, twice the bytes, it makes no difference.)
                const int f = cur.f0 + wq * 128 + frow * 8;
                const uint32_t stride = (uint32_t)features * 2u;
                const __amdgpu_buffer_rsrc_t out = __builtin_amdgcn_make_buffer_rsrc(
                    static_cast<uint16_t*>(a.out) + (FORM == kWgrad ? (size_t)cur.expert * N * K : (size_t)0) + (size_t)cur.row0 * features, 0,
                    (int)((uint32_t)cur.rows * stride), 0x00020000);
                const uint32_t to = f < features ? (uint32_t)(wt * 16 + fpiece) * stride + (uint32_t)f * 2u : kNowhere;
                auto put = [&](int i) GG_LAMBDA {
#pragma unroll
                    for (int j = 0; j < kF; ++j) {
                        uint2 pk;
                        pk.x = pack_bf16x2(from_acc(acc[j][i][0]), from_acc(acc[j][i][1]));
                        pk.y = pack_bf16x2(from_acc(acc[j][i][2]), from_acc(acc[j][i][3]));
                        *reinterpret_cast<uint2*>(own + i % 2 * 4096 + frow * 256 + (((j * 2 + (fpiece >> 1)) ^ frow) << 4) + (fpiece & 1) * 8) = pk;
                    }
                };
                constexpr int kWith = TFE < 4 ? TFE : 4;   // fragments with requests
                put(0);
#pragma unroll
                for (int i = 0; i < TFE; ++i) {
                    __builtin_amdgcn_sched_barrier(0);  // one fragment's values in registers at a time
                    if (more_items && i < kWith) {
#pragma unroll
                        for (int part = i * 4 / kWith; part < (i + 1) * 4 / kWith; ++part) request(part, next);
                    }
                    gg::wave_order();
                    u32x4 v[4];
#pragma unroll
                    for (int h = 0; h < 4; ++h) {
                        const int lr = h * 4 + fpiece;
                        v[h] = *reinterpret_cast<const u32x4*>(own + i % 2 * 4096 + lr * 256 + ((frow ^ lr) << 4));
                    }
                    if (i + 1 < TFE) put(i + 1);
#pragma unroll
                    for (int h = 0; h < 4; ++h) __builtin_amdgcn_raw_buffer_store_b128(v[h], out, to + (uint32_t)(i * 32 + h * 4) * stride, 0, kStreamed);
                    gg::wave_order();
                }
                stores = 4 * (TFE - kWith + 1);
            } else {
                if (more_items) request_first(next);
                // [16 rows][128 features] fp32, rows of 512 bytes, 16-byte unit u of row r at u ^ r
                const int unit = lane & 31, col = wq * 128 + unit * 4;
                const bool piece = cur.piece >= 0;
                tell_cut(told, cur, ((int64_t)(FORM == kWgrad ? cur.expert * (int64_t)N : 0) + cur.row0) * features + cur.f0, features);
                const uint32_t stride = (uint32_t)(piece ? kTile : features) * 4u;
                float* const tile_out = piece ? scratch + (size_t)cur.piece * piece_units * kUnitFloats
                                              : static_cast<float*>(a.out) + (size_t)cur.expert * N * K + (size_t)cur.row0 * features + cur.f0;
                // (the last row of a ragged feature tile ends before the next tile's memory)
                const uint32_t bytes = (uint32_t)cur.rows * stride - (piece ? 0u : (uint32_t)cur.f0 * 4u);
                const __amdgpu_buffer_rsrc_t out = __builtin_amdgcn_make_buffer_rsrc(tile_out, 0, (int)bytes, 0x00020000);
                const uint32_t to = cur.f0 + col < features ? (uint32_t)(wt * 16 + (lane >> 5)) * stride + (uint32_t)col * 4u : kNowhere;
                const bool adds = OUT32 && !piece && a.accumulate;
                u32x4 old[OUT32 ? 2 : 1][8];   // what is there already, two fragments ahead
                auto fetch = [&](int i) GG_LAMBDA {
#pragma unroll
                    for (int h = 0; h < 8; ++h) old[OUT32 ? i % 2 : 0][h] = __builtin_amdgcn_raw_buffer_load_b128(out, to + (uint32_t)(i * 32 + h * 2) * stride, 0, kStreamed);
                };
                if (adds) {
                    fetch(0);
                    if (TFE > 1) fetch(1);
                }
#pragma unroll
                for (int i = 0; i < TFE; ++i) {
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int j = 0; j < kF; ++j) {
                        f32x4 v;
#pragma unroll
                        for (int c = 0; c < 4; ++c) v[c] = from_acc(acc[j][i][c]);
                        *reinterpret_cast<f32x4*>(own + frow * 512 + (((j * 4 + fpiece) ^ frow) << 4)) = v;
                    }
                    gg::wave_order();
                    f32x4 v[8];
#pragma unroll
                    for (int h = 0; h < 8; ++h) {
                        const int lr = h * 2 + (lane >> 5);
                        v[h] = *reinterpret_cast<const f32x4*>(own + lr * 512 + ((unit ^ lr) << 4));
                    }
                    if (adds) {
#pragma unroll
                        for (int h = 0; h < 8; ++h) v[h] += __builtin_bit_cast(f32x4, old[OUT32 ? i % 2 : 0][h]);
                        if (i + 2 < TFE) fetch(i + 2);
                    }
#pragma unroll
                    for (int h = 0; h < 8; ++h)
                        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, v[h]), out, to + (uint32_t)(i * 32 + h * 2) * stride, 0, kStreamed);
                    gg::wave_order();
                }
                stores = 8 * TFE;
            }
        };
        const int groups = uniform((cur.rows + 31) / 32);
        if constexpr (FORM == kWgrad) {   // (rows are features here: multiples of 64)
            switch (groups) {
                case 1: case 2: tile(std::integral_constant<int, 2>{}); break;
                case 3: case 4: tile(std::integral_constant<int, 4>{}); break;
                case 5: case 6: tile(std::integral_constant<int, 6>{}); break;
                default: tile(std::integral_constant<int, 8>{}); break;
            }
        } else {
            switch (groups) {
                case 1: tile(std::integral_constant<int, 1>{}); break;
                case 2: tile(std::integral_constant<int, 2>{}); break;
                case 3: tile(std::integral_constant<int, 3>{}); break;
                case 4: tile(std::integral_constant<int, 4>{}); break;
                case 5: tile(std::integral_constant<int, 5>{}); break;
                case 6: tile(std::integral_constant<int, 6>{}); break;
                case 7: tile(std::integral_constant<int, 7>{}); break;
                default: tile(std::integral_constant<int, 8>{}); break;
            }
        }
        if (!more_items) break;
        cur = next;
        gg::lds_barrier();   // (the results went through the stage that is requested next)
        }
    }
};

template <int FORM, bool OUT32>
__global__ __launch_bounds__(256, 1) void product_gemm_kernel(Args a, float* scratch, Told* told) {
    using Kernel = TileKernel<FORM, OUT32>;
    __shared__ __attribute__((aligned(1024))) unsigned char lds[Kernel::kLdsBytes];
    Tiles<FORM, kStepC> list(a);
    Plan plan;
    if constexpr (FORM == kWgrad) {
        list.build(kTile);
        plan = choose_chunk(list, gridDim.x, a.n);
    } else {
        plan = choose_tiles(list, gridDim.x, {kTile, 90, 6});
        list.build(plan.height);
    }
    const Items<FORM, kStepC> items(list, plan);
    if (blockIdx.x == 0 && threadIdx.x == 0) told->plan = items.plan;
    const Hand<FORM, kStepC> hand(list, items);
    Item item;
    if (!hand(0, item)) return;
    Kernel::run(a, scratch, told, plan.piece_units, lds, item, hand);
}

}  // namespace products
}  // namespace moe
