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
constexpr int kMostCutTiles = 255;   // (the leftover tiles of a round of at most 256 workgroups)
constexpr int kMinPartSteps = 3;   // fewest K steps of a piece

// What a launch does, the same in every wavefront: chosen when its kernel starts and left in the workspace for the one that
// joins the pieces.
struct Plan {
    int height;        // rows of a tile
    int n_whole;       // forward, dgrad: tiles that are not cut; they come first
    int parts;         // forward, dgrad: pieces of the others
    int chunk;         // wgrad: K steps of a piece
    int piece_units;   // units of scratch of a piece
    int n_cuts;        // tiles that are cut
};

// A tile that was cut, for the kernel that joins its pieces.
struct Cut {
    int64_t out_at;         // element of the output of its first row and feature
    int rows, columns;      // that exist
    int first_piece, parts;
};
// What a launch leaves behind its pieces.
struct Told {
    Plan plan;
    Cut cuts[kMostCutTiles];
};
constexpr size_t kWorkspaceBytes = (kScratchBytes + sizeof(Told) + 255) / 256 * 256;

template <int CTRL, int ROWS>
__device__ GG_INLINE float least_before(float v) { return fminf(v, __int_as_float(lanes_before<CTRL, ROWS>(0x7f800000, __float_as_int(v)))); }
__device__ GG_INLINE float wave_min(float v) {   // like wave_sums()
    v = least_before<0x111, 0xf>(v);
    v = least_before<0x112, 0xf>(v);
    v = least_before<0x114, 0xf>(v);
    v = least_before<0x118, 0xf>(v);
    v = least_before<0x142, 0xa>(v);
    v = least_before<0x143, 0xc>(v);
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}

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
        // Rows first, lower experts first among equals, lanes without an expert last.  (Four in a step: one has to wait for the other.)
        const int key = lane < a.experts ? rows * 64 + 63 - lane : -lane;
        int rank = 0;
        for (int i = 0; i < a.experts; i += 4)
#pragma unroll
            for (int j = 0; j < 4; ++j) rank += __builtin_amdgcn_readlane(key, i + j) > key ? 1 : 0;
        rank = lane < a.experts ? rank : lane;
        rank_expert = __builtin_amdgcn_ds_permute(rank * 4, lane);
        first = __builtin_amdgcn_ds_permute(rank * 4, f);
        const int own = __builtin_amdgcn_ds_permute(rank * 4, rows);
        const int features = FORM == kForward ? a.n : a.k;
        n_ft = (features + kTile - 1) / kTile;
        depth = FORM == kWgrad ? own : FORM == kForward ? a.k : a.n;
        count = FORM != kWgrad ? own : own < 0 || (own == 0 && a.accumulate) ? 0 : a.n;
        height = total = first_tile = 0;
    }
    __device__ GG_INLINE int row_tiles(int h) const { return count > 0 ? (int)((uint32_t)(count + h - 1) / (uint32_t)h) : 0; }
    __device__ GG_INLINE int steps() const { return depth > 0 ? (depth + STEP - 1) / STEP : 1; }  // (no rows: one step of zeros)

    // wgrad: pieces of a tile of this lane's expert.
    __device__ GG_INLINE int parts_of(int chunk) const { return (steps() + chunk - 1) / chunk; }

    __device__ GG_INLINE void build(int h) {
        height = h;
        const int tiles = row_tiles(h) * n_ft;
        const int sum = wave_sums(tiles);
        first_tile = sum - tiles;
        total = __builtin_amdgcn_readlane(sum, 63);
    }
    // Tile `id`: rank of its expert, first row within the expert, rows, feature tile.
    __device__ GG_INLINE void find(int id, int& r, int& row, int& rows, int& ft) const {
        r = __popcll(__ballot(first_tile <= id && count > 0)) - 1;
        const int c = __builtin_amdgcn_readlane(count, r);
        const int local = id - __builtin_amdgcn_readlane(first_tile, r);
        const uint32_t mt = (uint32_t)(c + height - 1) / (uint32_t)height;
        const uint32_t groups = (mt + kGroup - 1) / kGroup;
        const int size = (int)(mt / groups), big = mt - size * groups;   // `big` groups of size + 1 row tiles, then groups of `size`
        const int in_big = big * (size + 1) * n_ft;
        const bool b = local < in_big;
        const int gs = b ? size + 1 : size;
        const int in = b ? local : local - in_big;
        const int g = (int)((uint32_t)in / (uint32_t)(gs * n_ft));
        const int in_grp = in - g * (gs * n_ft);
        ft = (int)((uint32_t)in_grp / (uint32_t)gs);
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
// of 60 plans (the tallest tile - 32 * (l / 12) rows; 1 to 6, 8, 10, 12, 16, 20 or 24 pieces) in 10 ns as the rounds, K steps x the price of one + 400 each
// (full ones at the rows of the hottest expert's tiles, those of the pieces, which are the coldest, at an average tile's), + 300 + 2 for each 32 rows
// of pieces, if there are any.  A K step does not take less than the memory needs for the weights that the workgroups of a round ask for: 32 KB each
// at 6.4 TB/s, a line of which the row tiles of an expert share.  The first of the cheapest plans is taken.
// (Prices of the hottest tiles for the pieces too, and one sum of the weights' time instead of the steps', left 1.5 rounds uncut: 64 experts of 1408 x 2048,
// 3000 rows 103 -> 95 us; 1, 4096 x 4096, 300 rows 28 -> 26.5; 8, 14336 x 4096, 512 rows 200 -> 182.)
template <class List>
__device__ GG_INLINE Plan choose_tiles(const List& list, int grid, Price price) {
    const int lane = threadIdx.x & 63;
    const int i = min(lane / 12, 4), n = lane - lane / 12 * 12, h = price.tallest - 32 * i;
    const int p = n < 6 ? n + 1 : n < 9 ? 2 * n - 4 : 4 * n - 20;
    int sums[5];
#pragma unroll
    for (int t = 0; t < 5; ++t) sums[t] = __builtin_amdgcn_readlane(wave_sums(list.row_tiles(price.tallest - 32 * t)), 63);
    const int most = __builtin_amdgcn_readlane(list.count, 0);
    const int active = __popcll(__ballot(list.count > 0));
    const int steps = __builtin_amdgcn_readlane(list.steps(), 0);
    int tiles = sums[0];
#pragma unroll
    for (int t = 1; t < 5; ++t) tiles = i == t ? sums[t] : tiles;
    // groups of 32 rows of an average tile
    const float groups = (float)__builtin_amdgcn_readlane(wave_sums(list.row_tiles(kUnitRows)), 63) / (float)max(tiles, 1);
    tiles *= list.n_ft;
    const int full = (int)((uint32_t)tiles / (uint32_t)grid), left = tiles - full * grid;
    const int units = (min(h, most) + kUnitRows - 1) / kUnitRows;
    const int rounds = (int)((uint32_t)(left * p + grid - 1) / (uint32_t)grid);
    const bool allowed = p == 1 || (left > 0 && left * p * units <= kScratchUnits && steps >= p * kMinPartSteps);
    const float memory = 130.f * active * list.n_ft / (float)max(tiles, 1);   // of a K step of all workgroups
    const float step = fmaxf(price.base + price.per_group * min(h, (most + 31) / 32 * 32) / 32, memory);
    const float step_left = fmaxf(price.base + price.per_group * groups, memory * (left * p) / (float)max(rounds * grid, 1));
    float cost = full * (steps * step + 400.f) + rounds * ((uint32_t)(steps + p - 1) / (uint32_t)p * step_left + 400.f);
    if (p > 1) cost += 300.f + 2.f * left * groups * p;
    if (lane >= 60 || !allowed) cost = INFINITY;
    const float best = wave_min(cost);
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
    const float best = wave_min(cost);
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
    int first_item, parts, first_piece, first_cut;   // wgrad, lane r

    __device__ GG_INLINE Items(const Tiles<FORM, STEP>& l, const Plan& p) : list(l), plan(p) {
        first_item = parts = first_piece = first_cut = 0;
        if constexpr (FORM == kWgrad) {
            const int tiles = list.row_tiles(list.height) * list.n_ft;
            parts = list.parts_of(plan.chunk);
            const int cut = parts > 1 ? tiles : 0;
            const int sum = wave_sums(tiles * parts), pieces = wave_sums(cut * parts), cuts = wave_sums(cut);
            first_item = sum - tiles * parts;
            first_piece = pieces - cut * parts;
            first_cut = cuts - cut;
            total = __builtin_amdgcn_readlane(sum, 63);
            left = 0;
            plan.n_cuts = __builtin_amdgcn_readlane(cuts, 63);
        } else {
            left = list.total - plan.n_whole;
            total = plan.n_whole + left * plan.parts;
            plan.n_cuts = plan.parts > 1 ? left : 0;
        }
    }
    // Item `id`: its tile, the K steps [begin, end) of it, the number of its piece (-1: it is a whole tile), which part of how many that is, and the number of
    // its tile among those that are cut.
    __device__ GG_INLINE void find(int id, int& tile, int& begin, int& end, int& piece, int& part, int& of, int& cut) const {
        int steps;
        part = 0;
        of = 1;
        piece = cut = -1;
        if constexpr (FORM == kWgrad) {
            const int r = __popcll(__ballot(first_item <= id && list.count > 0)) - 1;
            of = __builtin_amdgcn_readlane(parts, r);
            const int first = __builtin_amdgcn_readlane(list.first_tile, r), local = id - __builtin_amdgcn_readlane(first_item, r);
            const int tiles = __builtin_amdgcn_readlane(list.row_tiles(list.height) * list.n_ft, r);
            part = (int)((uint32_t)local / (uint32_t)tiles);
            tile = first + local - part * tiles;
            steps = __builtin_amdgcn_readlane(list.steps(), r);
            if (of > 1) {
                cut = __builtin_amdgcn_readlane(first_cut, r) + tile - first;
                piece = __builtin_amdgcn_readlane(first_piece, r) + (tile - first) * of + part;
            }
        } else {
            tile = id;
            steps = __builtin_amdgcn_readlane(list.steps(), 0);
            if (id >= plan.n_whole && plan.parts > 1) {
                of = plan.parts;
                part = (int)((uint32_t)(id - plan.n_whole) / (uint32_t)left);
                cut = id - plan.n_whole - part * left;
                tile = plan.n_whole + cut;
                piece = cut * of + part;
            }
        }
        begin = of > 1 ? (int)((uint32_t)(steps * part) / (uint32_t)of) : 0;
        end = of > 1 ? (int)((uint32_t)(steps * (part + 1)) / (uint32_t)of) : steps;
    }
};

// A work item: a tile or a piece of one.
struct Item {
    int expert, row0, rows, f0, k_steps, depth;   // row0: first output row (forward, dgrad: of the matrix; wgrad: of the expert's)
    int c0;                                       // first c: wgrad: row of the matrix, else of the contraction; depth: c from there on
    int piece;                                    // number of the piece, -1: a whole tile
    int cut, parts;                               // first piece of a tile that is cut: which one that is (else -1), and its pieces
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
        full = (int)((uint32_t)items.total / (uint32_t)grid);
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
        int tile, begin, end, r, row, ft, part;
        items.find(id, tile, begin, end, t.piece, part, t.parts, t.cut);
        t.cut = uniform(part == 0 ? t.cut : -1);
        t.parts = uniform(t.parts);
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

// The first piece of a tile tells the kernel that joins them where it belongs (out_at: element of its first row and feature).
__device__ GG_INLINE void tell_cut(Told* told, const Item& t, int64_t out_at, int features) {
    if (t.cut >= 0 && threadIdx.x == 0) told->cuts[t.cut] = Cut{out_at, t.rows, min(kTile, features - t.f0), t.piece, t.parts};
}

// Whether a launch of `grid` workgroups may cut tiles, as far as the host can tell: a piece has kMinPartSteps K steps at least, and wgrad cuts where its tiles
// are fewer than the workgroups (accumulating, tiles of experts without rows do not count, which the host does not know).  Where it cannot, nothing is to be
// joined: wgrad of 64 experts of 1408 x 2048 with 128 rows 105 -> 101 us.
inline bool may_cut(Form form, const Args& a, int step, int grid) {
    const int depth = form == kForward ? a.k : form == kDgrad ? a.n : a.rows;
    if ((depth + step - 1) / step < 2 * kMinPartSteps) return false;
    const long tiles = (long)a.experts * ((a.n + kTile - 1) / kTile) * ((a.k + kTile - 1) / kTile);
    return form != kWgrad || a.accumulate || tiles < grid;
}

// Adds the pieces of the tiles that were cut: four rows of one of them at a time for each workgroup, a thread four columns of a row.
constexpr int kJoinWorkgroups = 1024;
template <bool OUT32>
__global__ __launch_bounds__(256) void join_pieces_kernel(void* out, int features, int accumulate, const float* __restrict__ scratch, const Told* __restrict__ told) {
    const int units = told->plan.piece_units, groups = units * (kUnitRows / 4), total = told->plan.n_cuts * groups;
    const size_t piece_floats = (size_t)units * kUnitFloats;
    const int col = threadIdx.x % 64 * 4;
    for (int g = blockIdx.x; g < total; g += kJoinWorkgroups) {
        const Cut cut = told->cuts[g / groups];
        const int row = g % groups * 4 + threadIdx.x / 64;
        if (row >= cut.rows || col >= cut.columns) continue;
        const float* from = scratch + (size_t)cut.first_piece * piece_floats + (size_t)row * kTile + col;
        f32x4 v = *reinterpret_cast<const f32x4*>(from);
#pragma unroll 8
        for (int s = 1; s < cut.parts; ++s) v += *reinterpret_cast<const f32x4*>(from + s * piece_floats);
        const size_t to = (size_t)cut.out_at + (size_t)row * features + col;
        if constexpr (OUT32) {
            f32x4* o = reinterpret_cast<f32x4*>(static_cast<float*>(out) + to);
            if (accumulate) v += *o;
            *o = v;
        } else {
            *reinterpret_cast<uint2*>(static_cast<uint16_t*>(out) + to) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
        }
    }
}

}  // namespace products
}  // namespace moe
