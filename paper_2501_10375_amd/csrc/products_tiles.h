// How the grouped products are cut into tiles and pieces and dealt to the workgroups, and how pieces are joined (device code of
// products_bf16.h and products_fp8.h).
#pragma once

#include "grouped_gemm_bf16.h"
#include "products_internal.h"

namespace moe {
namespace products {

using gg::f32x4;
using gg::u32x4;
using gg::uniform;

constexpr int kTile = 256;   // features of a tile, and its rows at most
constexpr int kXcds = gg::kXcds;

// Scratch memory for the pieces of tiles that are cut along c, in units of 32 rows of 256 columns, and the plan behind it.
constexpr int kUnitRows = 32, kScratchUnits = 255 * 8;
constexpr size_t kUnitFloats = (size_t)kUnitRows * kTile;
constexpr size_t kScratchBytes = kScratchUnits * kUnitFloats * sizeof(float);
constexpr int kMostCutTiles = 255;   // (the leftover tiles of a round of at most 256)
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
// STEP: c of a K step.
template <int FORM, int STEP>
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
    __device__ GG_INLINE int steps() const { return depth > 0 ? (depth + STEP - 1) / STEP : 1; }  // (no rows: one step of zeros)

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

// What a K step of a tile costs, in 10 ns: base + per_group for each 32 rows.
struct Price {
    int tallest, base, per_group;
};

// Height of the tiles and pieces of the leftover ones (forward, dgrad), like choose_plan() of the expert GEMMs: lane l prices one
// of 30 plans (the tallest tile - 32 * (l / 6) rows, l % 6 + 1 pieces) in 10 ns, as the larger of
//   full rounds x (K steps x their price + 400) and the same for the rounds of pieces                  (MFMAs)
//   the weights of the experts with rows at 6.6 TB/s + 600 a round                                   (memory)
// + 300 + 2 a unit of pieces, if there are any; the first of the cheapest is taken.
template <class List>
__device__ GG_INLINE Plan choose_tiles(const List& list, int features, int grid, Price price) {
    const int lane = threadIdx.x & 63;
    const int i = min(lane / 6, 4), p = lane - lane / 6 * 6 + 1, h = price.tallest - 32 * i;
    int sums[5];
#pragma unroll
    for (int n = 0; n < 5; ++n) sums[n] = list.row_tiles(price.tallest - 32 * n);
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
    const float step = price.base + price.per_group * min(h, (most + 31) / 32 * 32) / 32;
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
template <class List>
__device__ GG_INLINE Plan choose_chunk(const List& list, int grid, int n) {
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
template <int FORM, int STEP>
struct Items {
    const Tiles<FORM, STEP>& list;
    Plan plan;
    int total, left;
    int first_item, parts, first_piece;   // wgrad, lane r

    __device__ GG_INLINE Items(const Tiles<FORM, STEP>& l, const Plan& p) : list(l), plan(p) {
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

// A work item: a tile or a piece of one.
struct Item {
    int expert, row0, rows, f0, k_steps, depth;   // row0: first output row (forward, dgrad: of the matrix; wgrad: of the expert's)
    int c0;                                       // first c: wgrad: row of the matrix, else of the contraction; depth: c from there on
    int piece;                                    // number of the piece, -1: a whole tile
};

// A workgroup's items.  The launch is persistent, one workgroup a CU.  Workgroup b belongs to XCD b % 8 (the hardware deals them out
// round-robin); a round is 32 consecutive items for each XCD, the last one what is left in equal shares.
template <int FORM, int STEP>
struct Hand {
    const Tiles<FORM, STEP>& list;
    const Items<FORM, STEP>& items;
    int grid, xcd, member, full, share;

    __device__ GG_INLINE Hand(const Tiles<FORM, STEP>& l, const Items<FORM, STEP>& i) : list(l), items(i) {
        grid = gridDim.x;
        xcd = blockIdx.x % kXcds;
        member = blockIdx.x / kXcds;
        full = items.total / grid;
        share = (items.total - full * grid + kXcds - 1) / kXcds;
    }
    // This workgroup's n-th item; false if it has fewer.
    __device__ GG_INLINE bool operator()(int n, Item& t) const {
        int id = (n * kXcds + xcd) * (grid / kXcds) + member;
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
        t.c0 = uniform(begin * STEP + (FORM == kWgrad ? first : 0));
        t.depth = uniform(max(0, depth - begin * STEP));
        return true;
    }
};

// A buffer descriptor of the memory from a K step of an operand on.  What lies behind its end reads as zero, and behind the last step
// everything does.
struct Buffer {
    u32x4 d;
    int steps;   // left, this one included
    // COLUMNS: lines of `line` bytes, a line for each c, of which c_left are left; the operand begins `skipped` bytes into a line.
    int c_left;
    uint32_t line, skipped;

    __device__ GG_INLINE void begin_at(const void* p, int k_steps) {
        const uint64_t at = reinterpret_cast<uint64_t>(p);
        d[0] = (uint32_t)uniform((int)(uint32_t)at);
        d[1] = (uint32_t)uniform((int)((uint32_t)(at >> 32) & 0xffffu));
        d[3] = 0x00020000u;
        steps = uniform(k_steps);
    }
    __device__ GG_INLINE void settle() { asm volatile("s_nop 4" : "+s"(d)::"memory"); }   // (a load reads what a vector instruction wrote)
    // Rows whose contraction is contiguous: `bytes` to the end of the last one (at most 256 rows of 4 MiB).
    __device__ GG_INLINE void set_rows(const void* p, int64_t bytes, int k_steps) {
        begin_at(p, k_steps);
        d[2] = (uint32_t)uniform((int)bytes);
        settle();
    }
    template <int STEP>
    __device__ GG_INLINE void set_columns(const void* p, int c, uint32_t line_bytes, uint32_t skipped_bytes, int k_steps) {
        begin_at(p, k_steps);
        c_left = uniform(c);
        line = line_bytes;
        skipped = (uint32_t)uniform((int)skipped_bytes);
        bound_columns<STEP>();
        settle();
    }
    template <int STEP>
    __device__ GG_INLINE void bound_columns() { d[2] = c_left > 0 ? (uint32_t)min(c_left, STEP) * line - skipped : 0u; }
    __device__ GG_INLINE void move(uint32_t bytes) {
        const uint64_t at = ((uint64_t)d[1] << 32 | d[0]) + bytes;   // (an address has 48 bits: nothing moves into the fields above)
        d[0] = (uint32_t)at;
        d[1] = (uint32_t)(at >> 32);
    }
    // On to the next K step.
    __device__ GG_INLINE void next_rows(uint32_t bytes) {
        move(bytes);
        --steps;
        d[2] = steps > 0 ? d[2] - bytes : 0u;
    }
    template <int STEP>
    __device__ GG_INLINE void next_columns() {
        move(STEP * line);
        --steps;
        c_left = steps > 0 ? c_left - STEP : 0;
        bound_columns<STEP>();
    }
};

// Adds the pieces of the tiles that were cut: 32 rows of one of them for each workgroup.
template <int FORM, int STEP, bool OUT32>
__global__ __launch_bounds__(256) void join_pieces_kernel(Args a, const float* __restrict__ scratch, const Plan* told) {
    const Plan plan = *told;
    if (FORM != kWgrad && plan.parts <= 1) return;
    const int cut = blockIdx.x / 8, unit = blockIdx.x % 8;   // number of the cut tile, and which rows of it
    Tiles<FORM, STEP> list(a);
    list.build(plan.height);
    const Items<FORM, STEP> items(list, plan);
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
