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
#pragma once

#include "grouped_gemm_bf16.h"
#include "products_internal.h"

namespace moe {
namespace products {

using gg::bf16x8;
using gg::f32x4;
using gg::u32x4;
using gg::uniform;

constexpr int kTile = 256, kStepC = 64;
constexpr int kXcds = gg::kXcds;

// Scratch memory for the pieces of tiles that are cut along c, in units of 32 rows of 256 columns, and the plan behind it.
constexpr int kUnitRows = 32, kScratchUnits = 255 * 8;
constexpr size_t kUnitFloats = (size_t)kUnitRows * kTile;
constexpr int kMinPartSteps = 3;   // fewest K steps of a piece

// What a launch does, the same in every wavefront: chosen when its kernel starts and left in the workspace for the one that
// joins the pieces.
struct Plan {
    int height;        // rows of a tile
    int n_whole;       // forward, dgrad: tiles that are not cut; they come first
    int parts;         // forward, dgrad: pieces of the others
    int chunk;         // wgrad: K steps of a piece
    int piece_units;   // units of scratch of a piece
};

// The tiles of a launch, expert by expert in descending order of rows; lane r holds the expert of rank r.  Within an expert
// row tiles in groups of at most eight of nearly equal size, within a group feature tile by feature tile: 32 consecutive tiles are
// what the CUs of an XCD work on at a time, and share operand lines through its L2.
template <int FORM>
struct Tiles {
    static constexpr int kGroup = 8;
    int n_ft, rank_expert, first, depth, count;   // depth: c of the expert; count: its output rows (wgrad: out_features)
    int height, total, first_tile;                // after build()

    __device__ GG_INLINE explicit Tiles(const Args& a) {
        const int lane = threadIdx.x & 63;
        int f, end;
        expert_rows(a, lane, f, end);
        const int rows = lane < a.experts ? end - f : -1;
        int rank = lane < a.experts ? 0 : lane;
        for (int i = 0; i < a.experts; ++i) {
            const int ri = __builtin_amdgcn_readlane(rows, i);
            if (lane < a.experts) rank += (ri > rows || (ri == rows && i < lane)) ? 1 : 0;
        }
        rank_expert = __builtin_amdgcn_ds_permute(rank * 4, lane);
        first = __builtin_amdgcn_ds_permute(rank * 4, f);
        const int own = __builtin_amdgcn_ds_permute(rank * 4, rows);
        const int features = FORM == kForward ? a.n : a.k;
        n_ft = (features + kTile - 1) / kTile;
        depth = FORM == kWgrad ? own : FORM == kForward ? a.k : a.n;
        count = FORM != kWgrad ? own : own < 0 || (own == 0 && a.accumulate) ? 0 : a.n;
        height = total = first_tile = 0;
    }
    __device__ GG_INLINE int row_tiles(int h) const { return count > 0 ? (count + h - 1) / h : 0; }
    __device__ GG_INLINE int steps() const { return depth > 0 ? (depth + kStepC - 1) / kStepC : 1; }  // (no rows: one step of zeros)

    // wgrad: pieces of a tile of this lane's expert.
    __device__ GG_INLINE int parts_of(int chunk) const { return (steps() + chunk - 1) / chunk; }

    __device__ GG_INLINE void build(int h) {
        height = h;
        const int tiles = row_tiles(h) * n_ft;
        const int sum = gg::wave_inclusive_sum(tiles);
        first_tile = sum - tiles;
        total = __builtin_amdgcn_readlane(sum, 63);
    }
    // Tile `id`: rank of its expert, first row within the expert, rows, feature tile.
    __device__ GG_INLINE void find(int id, int& r, int& row, int& rows, int& ft) const {
        r = __popcll(__ballot(first_tile <= id && count > 0)) - 1;
        const int c = __builtin_amdgcn_readlane(count, r);
        const int local = id - __builtin_amdgcn_readlane(first_tile, r);
        const int mt = (c + height - 1) / height;
        const int groups = (mt + kGroup - 1) / kGroup;
        const int size = mt / groups, big = mt - size * groups;   // `big` groups of size + 1 row tiles, then groups of `size`
        const int in_big = big * (size + 1) * n_ft;
        const bool b = local < in_big;
        const int gs = b ? size + 1 : size;
        const int in = b ? local : local - in_big;
        const int g = in / (gs * n_ft);
        const int in_grp = in - g * (gs * n_ft);
        ft = in_grp / gs;
        const int m = (b ? 0 : big * (size + 1)) + g * gs + in_grp - ft * gs;
        row = m * height;
        rows = min(height, c - row);
    }
};

// Height of the tiles and pieces of the leftover ones (forward, dgrad), like choose_plan() of the expert GEMMs: lane l prices one
// of 30 plans (heights 256 - 32 * (l / 6), l % 6 + 1 pieces) in 10 ns, as the larger of
//   full rounds x (K steps x (90 + 6 x height / 32) + 400) and the same for the rounds of pieces       (MFMAs)
//   the weights of the experts with rows at 6.6 TB/s + 600 a round                                   (memory)
// + 300 + 2 a unit of pieces, if there are any; the first of the cheapest is taken.
template <int FORM>
__device__ GG_INLINE Plan choose_tiles(const Tiles<FORM>& list, int features, int grid) {
    const int lane = threadIdx.x & 63;
    const int i = min(lane / 6, 4), p = lane - lane / 6 * 6 + 1, h = kTile - 32 * i;
    int sums[5];
#pragma unroll
    for (int n = 0; n < 5; ++n) sums[n] = list.row_tiles(kTile - 32 * n);
    const int most = __builtin_amdgcn_readlane(list.count, 0);
    const int active = __popcll(__ballot(list.count > 0));
    const int steps = __builtin_amdgcn_readlane(list.steps(), 0);
    gg::wave_totals(sums);
    int tiles = sums[0];
#pragma unroll
    for (int n = 1; n < 5; ++n) tiles = i == n ? sums[n] : tiles;
    tiles *= list.n_ft;
    const int full = tiles / grid, left = tiles - full * grid;
    const int units = (min(h, most) + kUnitRows - 1) / kUnitRows;
    const int rounds = (left * p + grid - 1) / grid;
    const bool allowed = p == 1 || (left > 0 && left * p * units <= kScratchUnits && steps >= p * kMinPartSteps);
    const float step = 90 + 6 * min(h, (most + 31) / 32 * 32) / 32;
    const float work = full * (steps * step + 400.f) + rounds * ((steps + p - 1) / p * step + 400.f);
    const float stream = active * (float)features * steps * (1.f / 516.f) + (full + rounds) * 600.f;
    float cost = fmaxf(work, stream) + (p > 1 ? 300.f + 2.f * left * units * p : 0.f);
    if (lane >= 30 || !allowed) cost = INFINITY;
    float best = cost;
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) best = fminf(best, __shfl_xor(best, d, 64));
    const int winner = __ffsll((long long)__ballot(cost == best)) - 1;
    Plan plan;
    plan.height = __builtin_amdgcn_readlane(h, winner);
    plan.parts = __builtin_amdgcn_readlane(p, winner);
    plan.n_whole = __builtin_amdgcn_readlane(plan.parts > 1 ? full * grid : tiles, winner);
    plan.piece_units = __builtin_amdgcn_readlane(units, winner);
    plan.chunk = 0;
    return plan;
}

// Pieces of wgrad's tiles: where they are less than a round of the chip, lane l prices cutting every expert's rows into chunks of the
// longest one's K steps / (l + 1), as rounds of chunks plus the pieces written and read.
__device__ GG_INLINE Plan choose_chunk(const Tiles<kWgrad>& list, int grid, int n) {
    Plan plan;
    plan.height = kTile;
    plan.parts = 1;
    plan.n_whole = list.total;
    plan.piece_units = (min(kTile, n) + kUnitRows - 1) / kUnitRows;
    const int longest = __builtin_amdgcn_readlane(list.steps(), 0);
    plan.chunk = longest;
    if (list.total >= grid || longest < 2 * kMinPartSteps) return plan;
    const int lane = threadIdx.x & 63;
    const int chunk = max(kMinPartSteps, (longest + lane) / (lane + 1));
    int pieces = 0, cut = 0;
    const int steps = list.steps(), tiles = list.row_tiles(kTile) * list.n_ft;
    for (int r = 0; r < 64; ++r) {
        const int t = __builtin_amdgcn_readlane(tiles, r);
        if (t == 0) continue;
        const int parts = (__builtin_amdgcn_readlane(steps, r) + chunk - 1) / chunk;
        pieces += t * parts;
        cut += parts > 1 ? t * parts : 0;
    }
    float cost = (float)((pieces + grid - 1) / grid) * (chunk * 138.f + 400.f) + (cut > 0 ? 300.f + 2.f * cut * plan.piece_units : 0.f);
    if (cut * plan.piece_units > kScratchUnits) cost = INFINITY;
    float best = cost;
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) best = fminf(best, __shfl_xor(best, d, 64));
    plan.chunk = __builtin_amdgcn_readlane(chunk, __ffsll((long long)__ballot(cost == best)) - 1);
    return plan;
}

// Pieces and tiles in the order in which they are worked on.  forward, dgrad: the whole tiles, then the pieces of the others, first
// all first ones.  wgrad: the tiles expert by expert, the pieces of an expert's tiles with all first ones first.
template <int FORM>
struct Items {
    const Tiles<FORM>& list;
    Plan plan;
    int total, left;
    int first_item, parts, first_piece;   // wgrad, lane r

    __device__ GG_INLINE Items(const Tiles<FORM>& l, const Plan& p) : list(l), plan(p) {
        first_item = parts = first_piece = 0;
        if constexpr (FORM == kWgrad) {
            const int tiles = list.row_tiles(list.height) * list.n_ft;
            parts = list.parts_of(plan.chunk);
            const int sum = gg::wave_inclusive_sum(tiles * parts), cut = gg::wave_inclusive_sum(parts > 1 ? tiles * parts : 0);
            first_item = sum - tiles * parts;
            first_piece = cut - (parts > 1 ? tiles * parts : 0);
            total = __builtin_amdgcn_readlane(sum, 63);
            left = 0;
        } else {
            left = list.total - plan.n_whole;
            total = plan.n_whole + left * plan.parts;
        }
    }
    // Item `id`: its tile, the K steps [begin, end) of it, and the number of its piece (-1: it is a whole tile).
    __device__ GG_INLINE void find(int id, int& tile, int& begin, int& end, int& piece) const {
        int part = 0, of = 1, steps;
        piece = -1;
        if constexpr (FORM == kWgrad) {
            const int r = __popcll(__ballot(first_item <= id && list.count > 0)) - 1;
            of = __builtin_amdgcn_readlane(parts, r);
            const int first = __builtin_amdgcn_readlane(list.first_tile, r), local = id - __builtin_amdgcn_readlane(first_item, r);
            const int tiles = __builtin_amdgcn_readlane(list.row_tiles(list.height) * list.n_ft, r);
            part = local / tiles;
            tile = first + local - part * tiles;
            steps = __builtin_amdgcn_readlane(list.steps(), r);
            if (of > 1) piece = __builtin_amdgcn_readlane(first_piece, r) + (tile - first) * of + part;
        } else {
            tile = id;
            steps = __builtin_amdgcn_readlane(list.steps(), 0);
            if (id >= plan.n_whole && plan.parts > 1) {
                of = plan.parts;
                part = (id - plan.n_whole) / left;
                const int t = id - plan.n_whole - part * left;
                tile = plan.n_whole + t;
                piece = t * of + part;
            }
        }
        begin = steps * part / of;
        end = steps * (part + 1) / of;
    }
};

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

    struct Item {
        int expert, row0, rows, f0, k_steps, depth;   // row0: first output row (forward, dgrad: of the matrix; wgrad: of the expert's)
        int c0;                                       // first c: wgrad: row of the matrix, else of the contraction
        int piece;
    };

    // Memory from `p` on, `bytes` of it; what lies behind reads as zero.
    struct Buffer {
        uint64_t at;
        int64_t left;
        u32x4 d;
        __device__ GG_INLINE void describe() {
            d[0] = (uint32_t)at;
            d[1] = (uint32_t)(at >> 32) & 0xffffu;
            d[2] = left < 0 ? 0u : left > 0xffffffffll ? 0xffffffffu : (uint32_t)left;
        }
        __device__ GG_INLINE void set(const void* p, int64_t bytes) {
            at = reinterpret_cast<uint64_t>(p);
            at = (uint64_t)(uint32_t)uniform((int)(at >> 32)) << 32 | (uint32_t)uniform((int)(uint32_t)at);
            left = (int64_t)((uint64_t)(uint32_t)uniform((int)(bytes >> 32)) << 32 | (uint32_t)uniform((int)(uint32_t)bytes));
            d[3] = 0x00020000u;
            describe();
            asm volatile("s_nop 4" : "+s"(d)::"memory");   // (a scalar register that a vector instruction wrote, before a load reads it)
        }
        __device__ GG_INLINE void advance(uint32_t bytes) {
            at += bytes;
            left -= bytes;
            describe();
        }
    };

    static __device__ GG_INLINE void set_lds_target(uint32_t a) { asm volatile("s_mov_b32 m0, %0" ::"s"(a) : "memory"); }
    static __device__ GG_INLINE void load_lane(u32x4 d, uint32_t off) {
        asm volatile("buffer_load_dwordx4 %0, %1, 0 offen lds" ::"v"(off), "s"(d) : "memory");
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
    static __device__ GG_INLINE void wait_state() { asm volatile("s_nop 0" ::: "memory"); }

    // Half a fragment (4 c of 16 rows) out of a column stage.
    static __device__ GG_INLINE i16x4 read_turned(lds_ptr p) {
        return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4*)(uintptr_t)(uint32_t)(uintptr_t)p);
    }

    // decode(n, Item&): this workgroup's n-th item, false if it has fewer.
    template <class Decode>
    static __device__ GG_INLINE void run(const Args& a, float* scratch, int piece_units, unsigned char* lds, Item cur, const Decode& decode) {
        const int N = a.n, K = a.k;
        const int features = FORM == kForward ? N : K;
        const lds_ptr lds3 = (lds_ptr)lds;
        const uint32_t lds0 = (uint32_t)(uintptr_t)lds3;
        const int wave = uniform((int)threadIdx.x >> 6);
        const int wt = wave & 1, wq = wave >> 1;      // row group, feature group
        const uint32_t wave_lds = lds0 + (uint32_t)wave * 1024;
        auto next_w = [](uint32_t s) GG_LAMBDA { return s == 2 * kStage ? 0u : s + kStage; };

        // ---- staging.  Rows: load n of wavefront w covers rows n * 32 + w * 8 .. + 7, lane l the 16-byte piece that belongs at
        // position l % 8 of row l / 8.  Columns: c n * 8 + w * 2 and the next one, lane l the piece that belongs at position l % 32 of
        // line l / 32; there 32-byte units are exchanged, unit u of line c at u ^ (c % 4 + 4 (c / 8 % 2)), so that the 32 lanes that a
        // transposing read serves at a time (eight c, 32 bytes each) find their units in different banks.
        const uint32_t p_ld = (uint32_t)K * 2u, q_ld = (uint32_t)(FORM == kForward ? K : N) * 2u;
        const uint32_t p_step = kPCols ? kStepC * p_ld : kStepC * 2u, q_step = kQCols ? kStepC * q_ld : kStepC * 2u;
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
        auto p_load = [&](int n) GG_LAMBDA { load_lane(p.d, p_off[n]); };
        auto q_load = [&](int n) GG_LAMBDA { load_lane(q.d, q_off[n]); };
        auto q_loads = [](int rows) GG_LAMBDA { return kQCols ? 8 : (rows + 31) / 32; };
        auto p_stage = [&](uint32_t stage) GG_LAMBDA {
#pragma unroll
            for (int n = 0; n < 8; ++n) {
                set_lds_target(wave_lds + stage + n * 4096);
                wait_state();
                p_load(n);
            }
            p.advance(p_step);
        };
        auto q_stage = [&](uint32_t stage, int loads) GG_LAMBDA {
#pragma unroll
            for (int n = 0; n < 8; ++n) {
                if (n >= loads) break;
                set_lds_target(wave_lds + kQBase + stage + n * 4096);
                wait_state();
                q_load(n);
            }
            q.advance(q_step);
        };
        // First requests of an item, into p stage w0 and q stage 0.
        auto request_first = [&](const Item& t, uint32_t w0) GG_LAMBDA {
            const uint16_t *pm = static_cast<const uint16_t*>(a.p), *qm = static_cast<const uint16_t*>(a.q);
            if constexpr (FORM == kWgrad) {
                p.set(pm + (size_t)t.c0 * K + t.f0, ((int64_t)t.depth * K - t.f0) * 2);
                q.set(qm + (size_t)t.c0 * N + t.row0, ((int64_t)t.depth * N - t.row0) * 2);
            } else {
                const int64_t at = FORM == kForward ? (int64_t)t.f0 * K + t.c0 : (int64_t)t.c0 * K + t.f0;   // in the expert's matrix
                p.set(pm + (size_t)t.expert * N * K + at, ((int64_t)N * K - at) * 2);
                const int ld = FORM == kForward ? K : N;
                q.set(qm + (size_t)t.row0 * ld + t.c0, ((int64_t)t.rows * ld - t.c0) * 2);
            }
            p_stage(w0);
            q_stage(0, q_loads(t.rows));
        };

        uint32_t w0 = 0;   // p stage of an item's first K step
        request_first(cur, w0);
        for (int n = 1;; ++n) {
        int tid = threadIdx.x;   // (opaque: lane addresses are computed where they are used)
        asm volatile("" : "+v"(tid));
        const int lane = tid & 63;
        const int KT = cur.k_steps;
        if (KT > 1) {
            p_stage(next_w(w0));
            gg::wait_vmcnt<8>();
        } else {
            gg::wait_vmcnt<0>();
        }
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

            constexpr int kM = kF * TFE, kR = kF + TFE, kQLoads = kQCols ? 8 : TFE;
            bf16x8 pf[2][kF], qf[2][TFE];
            // Half a K step: the MFMAs of fragment buffer mbuf, between them the LDS reads of half `half` of the stages
            // into buffer 1 - mbuf, and the loads of one operand (LOADS 1: q, 2: p) for a later K step.
            auto half_step = [&](auto mfma, auto mbuf_c, auto read, int half, uint32_t p_at, uint32_t q_at, auto loads, uint32_t target) GG_LAMBDA {
                constexpr int mbuf = decltype(mbuf_c)::value, rbuf = 1 - mbuf;
                constexpr int LOADS = decltype(loads)::value;
                constexpr int n_loads = LOADS == 1 ? kQLoads : LOADS == 2 ? 8 : 1;
                constexpr int gap = kM / n_loads;
                constexpr int read_slots = kM - kM / 8;   // the last reads get some MFMAs' time before they are used
#pragma unroll
                for (int m = 0; m < kM; ++m) {
                    if constexpr (decltype(mfma)::value) {
                        const int i = m / kF, j = m % kF;
                        mfma_acc(acc[j][i], pf[mbuf][j], qf[mbuf][i]);
                    }
                    if constexpr (decltype(read)::value) {
#pragma unroll
                        for (int x = 0; x < kR; ++x) {
                            if (x * read_slots / kR != m) continue;
                            if (x < kF) pf[rbuf][x] = fragment(std::bool_constant<kPCols>{}, p_read, p_at, half, x);
                            else qf[rbuf][x - kF] = fragment(std::bool_constant<kQCols>{}, q_read, q_at + kQBase, half, (x - kF) * 2);
                        }
                    }
                    if constexpr (LOADS != 0) {
                        const int l = m / gap;
                        if (l < n_loads) {
                            if (m % gap == 0) {
                                set_lds_target(target + l * 4096);
                                if (gap == 1) wait_state();
                            }
                            if (m % gap == gap / 2) {
                                if constexpr (LOADS == 1) q_load(l);
                                else p_load(l);
                            }
                        }
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
                if constexpr (LOADS == 1) q.advance(q_step);
                if constexpr (LOADS == 2) p.advance(p_step);
            };
            using Buf0 = std::integral_constant<int, 0>;
            using Buf1 = std::integral_constant<int, 1>;
            using None = std::integral_constant<int, 0>;
            using LoadQ = std::integral_constant<int, 1>;
            using LoadP = std::integral_constant<int, 2>;

            // first half of K step 0 into buffer 0; q of K step 1 requested
            uint32_t p_at = w0, q_at = 0;                      // stages of K step kt
            half_step(No{}, Buf1{}, Yes{}, 0, p_at, q_at, None{}, 0u);
            if (KT > 1) q_stage(kStage, kQLoads);
            auto k_step = [&](auto more) GG_LAMBDA {  // second half of K step kt, first half of K step kt + 1
                const uint32_t w1 = next_w(p_at), w2 = next_w(w1), q1 = q_at ^ kStage;
                // Stage w2 held K step kt - 1, which every wavefront had read before the last barrier.
                half_step(Yes{}, Buf0{}, Yes{}, 1, p_at, q_at, std::conditional_t<decltype(more)::value, LoadP, None>{}, wave_lds + w2);
                // Outstanding, oldest first: p of K step kt + 1, its q, p of K step kt + 2.
                if constexpr (decltype(more)::value) gg::wait_vmcnt<8>();
                else gg::wait_vmcnt<0>();
                gg::lds_barrier();
                half_step(Yes{}, Buf1{}, Yes{}, 0, w1, q1, std::conditional_t<decltype(more)::value, LoadQ, None>{}, wave_lds + kQBase + q_at);
                p_at = w1;
                q_at = q1;
            };
            for (int kt = 0; kt < KT - 2; ++kt) k_step(Yes{});
            if (KT > 1) k_step(No{});
            half_step(Yes{}, Buf0{}, Yes{}, 1, p_at, q_at, None{}, 0u);
            half_step(Yes{}, Buf1{}, No{}, 0, 0u, 0u, None{}, 0u);
            settle();
            pin(acc);

            // ---- the next item's first operands are requested before this one's results are stored.
            more_items = decode(n, next);
            gg::lds_barrier();   // every wavefront is done reading operand tiles; no load is outstanding
            w0 = next_w(p_at);
            if (more_items) request_first(next, w0);

            // ---- epilogue: through LDS (8 KB a wavefront in q stage 1, which is requested later), so that stores are whole lines.
            // An MFMA result: lane l holds row l % 16 of its fragment and features 4 * (l / 16) + 0 .. 3.
            unsigned char* own = lds + kQBase + kStage + wave * 8192;
            if (!OUT32 && cur.piece < 0) {
                // [16 rows][128 features] bf16, rows of 256 bytes, 16-byte unit u of row r at u ^ r
                const int f = cur.f0 + wq * 128 + frow * 8;
                uint16_t* out = static_cast<uint16_t*>(a.out) + (FORM == kWgrad ? (size_t)cur.expert * N * K : (size_t)0) + (size_t)cur.row0 * features + f;
#pragma unroll
                for (int i = 0; i < TFE; ++i) {
                    __builtin_amdgcn_sched_barrier(0);  // one fragment's values in registers at a time
#pragma unroll
                    for (int j = 0; j < kF; ++j) {
                        uint2 pk;
                        pk.x = pack_bf16x2(from_acc(acc[j][i][0]), from_acc(acc[j][i][1]));
                        pk.y = pack_bf16x2(from_acc(acc[j][i][2]), from_acc(acc[j][i][3]));
                        *reinterpret_cast<uint2*>(own + frow * 256 + (((j * 2 + (fpiece >> 1)) ^ frow) << 4) + (fpiece & 1) * 8) = pk;
                    }
                    gg::wave_order();
#pragma unroll
                    for (int h = 0; h < 4; ++h) {
                        const int lr = h * 4 + fpiece;
                        const int row = (2 * i + wt) * 16 + lr;
                        const u32x4 v = *reinterpret_cast<const u32x4*>(own + lr * 256 + ((frow ^ lr) << 4));
                        if (row < cur.rows && f < features) *reinterpret_cast<u32x4*>(out + (size_t)row * features) = v;
                    }
                    gg::wave_order();
                }
            } else {
                // [16 rows][128 features] fp32, rows of 512 bytes, 16-byte unit u of row r at u ^ r
                const int unit = lane & 31, col = wq * 128 + unit * 4;
                const bool piece = cur.piece >= 0;
                float* out = piece ? scratch + (size_t)cur.piece * piece_units * kUnitFloats + col
                                   : static_cast<float*>(a.out) + (size_t)cur.expert * N * K + (size_t)cur.row0 * features + cur.f0 + col;
                const size_t stride = piece ? kTile : features;
                const bool stores = cur.f0 + col < features;
                const bool adds = OUT32 && !piece && a.accumulate;
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
#pragma unroll
                    for (int h = 0; h < 8; ++h) {
                        const int lr = h * 2 + (lane >> 5);
                        const int row = (2 * i + wt) * 16 + lr;
                        f32x4 v = *reinterpret_cast<const f32x4*>(own + lr * 512 + ((unit ^ lr) << 4));
                        if (row < cur.rows && stores) {
                            f32x4* to = reinterpret_cast<f32x4*>(out + (size_t)row * stride);
                            if (adds) v += *to;
                            *to = v;
                        }
                    }
                    gg::wave_order();
                }
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
        }
    }
};

// Persistent, one workgroup a CU.  Workgroup b belongs to XCD b % 8 (the hardware deals them out round-robin); a round is 32 consecutive
// items for each XCD, the last one what is left in equal shares.
template <int FORM, bool OUT32>
__global__ __launch_bounds__(256, 1) void product_gemm_kernel(Args a, float* scratch, Plan* told) {
    using Kernel = TileKernel<FORM, OUT32>;
    __shared__ __attribute__((aligned(1024))) unsigned char lds[Kernel::kLdsBytes];
    Tiles<FORM> list(a);
    const int grid = gridDim.x;   // a multiple of the XCDs
    Plan plan;
    if constexpr (FORM == kWgrad) {
        list.build(kTile);
        plan = choose_chunk(list, grid, a.n);
    } else {
        plan = choose_tiles<FORM>(list, FORM == kForward ? a.n : a.k, grid);
        list.build(plan.height);
    }
    if (blockIdx.x == 0 && threadIdx.x == 0) *told = plan;
    const Items<FORM> items(list, plan);
    const int xcd = blockIdx.x % kXcds, member = blockIdx.x / kXcds, members = grid / kXcds;
    const int full = items.total / grid, rest = items.total - full * grid;
    const int share = (rest + kXcds - 1) / kXcds;
    auto decode = [&](int n, typename Kernel::Item& t) GG_LAMBDA {
        int id = (n * kXcds + xcd) * members + member;
        if (n >= full) {
            if (n > full || member >= share) return false;
            id = full * grid + xcd * share + member;
            if (id >= items.total) return false;
        }
        int tile, begin, end, r, row, ft;
        items.find(id, tile, begin, end, t.piece);
        list.find(tile, r, row, t.rows, ft);
        t.expert = __builtin_amdgcn_readlane(list.rank_expert, r);
        const int first = __builtin_amdgcn_readlane(list.first, r);
        const int depth = __builtin_amdgcn_readlane(list.depth, r);
        t.k_steps = uniform(end - begin);
        t.rows = uniform(t.rows);
        t.f0 = uniform(ft * kTile);
        t.piece = uniform(t.piece);
        t.row0 = uniform(FORM == kWgrad ? row : first + row);
        t.c0 = uniform(begin * kStepC + (FORM == kWgrad ? first : 0));
        t.depth = uniform(max(0, depth - begin * kStepC));
        return true;
    };
    typename Kernel::Item item;
    if (!decode(0, item)) return;
    Kernel::run(a, scratch, plan.piece_units, lds, item, decode);
}

// Adds the pieces of the tiles that were cut: 32 rows of one of them for each workgroup.
template <int FORM, bool OUT32>
__global__ __launch_bounds__(256) void join_pieces_kernel(Args a, const float* __restrict__ scratch, const Plan* told) {
    const Plan plan = *told;
    if (FORM != kWgrad && plan.parts <= 1) return;
    const int cut = blockIdx.x / 8, unit = blockIdx.x % 8;   // number of the cut tile, and which rows of it
    Tiles<FORM> list(a);
    list.build(plan.height);
    const Items<FORM> items(list, plan);
    int tile, r, row, rows, ft, parts, piece;
    if constexpr (FORM == kWgrad) {
        const int cut_tiles = items.parts > 1 ? list.row_tiles(list.height) * list.n_ft : 0;
        const int sum = gg::wave_inclusive_sum(cut_tiles);
        if (cut >= __builtin_amdgcn_readlane(sum, 63)) return;
        const int owner = __popcll(__ballot(sum <= cut));   // (experts that are cut come first: they have most rows)
        const int local = cut - __builtin_amdgcn_readlane(sum - cut_tiles, owner);
        tile = __builtin_amdgcn_readlane(list.first_tile, owner) + local;
        parts = __builtin_amdgcn_readlane(items.parts, owner);
        piece = __builtin_amdgcn_readlane(items.first_piece, owner) + local * parts;
    } else {
        if (cut >= items.left) return;
        tile = plan.n_whole + cut;
        parts = plan.parts;
        piece = cut * parts;
    }
    list.find(tile, r, row, rows, ft);
    const int features = FORM == kForward ? a.n : a.k;
    const int expert = __builtin_amdgcn_readlane(list.rank_expert, r);
    const int64_t row0 = (FORM == kWgrad ? (int64_t)expert * a.n : (int64_t)__builtin_amdgcn_readlane(list.first, r)) + row;
    const int col = threadIdx.x % 64 * 4, f = ft * kTile + col;
    if (f >= features) return;
    const size_t piece_floats = (size_t)plan.piece_units * kUnitFloats;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int at = unit * kUnitRows + i * 4 + threadIdx.x / 64;
        if (at >= rows) break;
        const float* from = scratch + (size_t)piece * piece_floats + (size_t)at * kTile + col;
        f32x4 v = *reinterpret_cast<const f32x4*>(from);
        for (int s = 1; s < parts; ++s) v += *reinterpret_cast<const f32x4*>(from + s * piece_floats);
        const size_t to = (size_t)(row0 + at) * features + f;
        if constexpr (OUT32) {
            f32x4* o = reinterpret_cast<f32x4*>(static_cast<float*>(a.out) + to);
            if (a.accumulate) v += *o;
            *o = v;
        } else {
            *reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.out) + to) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
        }
    }
}

}  // namespace products
}  // namespace moe
