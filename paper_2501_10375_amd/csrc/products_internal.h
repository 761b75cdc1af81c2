// Shared by the translation units of the grouped products (include/moe_products.h): arguments, launchers and how a workgroup
// finds its tile.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "moe_internal.h"
#include "moe_products.h"
#include "products_rules.h"

namespace moe {
namespace products {

struct Args {
    const void *q, *p;
    void* out;
    const int32_t* offsets;           // [E + 1], or null: one expert with all rows
    int experts, rows, n, k;          // n = out_features, k = in_features
    const float *q_scales, *p_scales; // 8-bit operands, else null
    int accumulate;                   // kWgrad
};

// Inclusive sums over a wavefront by DPP: shifts within rows of 16 lanes, then the last lane of a row (of two rows) to the next one.  (Some ten
// cycles a step; by __shfl_up, which goes through LDS, more than a hundred, all of them ahead of a launch's first load.)
template <int CTRL, int ROWS>
__device__ inline int lanes_before(int other, int v) { return __builtin_amdgcn_update_dpp(other, v, CTRL, ROWS, 0xf, false); }
__device__ inline int wave_sums(int v) {
    v += lanes_before<0x111, 0xf>(0, v);
    v += lanes_before<0x112, 0xf>(0, v);
    v += lanes_before<0x114, 0xf>(0, v);
    v += lanes_before<0x118, 0xf>(0, v);
    v += lanes_before<0x142, 0xa>(0, v);
    v += lanes_before<0x143, 0xc>(0, v);
    return v;
}

// First and one past the last row of lane `lane`'s expert, inside [0, rows] whatever the table holds.
__device__ inline void expert_rows(const Args& a, int lane, int& first, int& end) {
    first = end = 0;
    if (lane < a.experts) {
        first = a.offsets == nullptr ? 0 : min(max(a.offsets[lane], 0), a.rows);
        end = a.offsets == nullptr ? a.rows : min(max(a.offsets[lane + 1], first), a.rows);
    }
}

// Row tiles of at most `height` rows that a call can have, which the host knows without the table: every expert's last one may be ragged.
inline long most_row_tiles(int rows, int experts, int height) {
    return (rows + height - 1) / height + (experts - 1 < rows ? experts - 1 : rows);
}

// Row tile `tile` of `height` rows (the same in all lanes; expert by expert): its expert, first row and rows; false if there is none.
__device__ inline bool find_row_tile(const Args& a, int tile, int height, int& expert, int& row0, int& rows) {
    const int lane = threadIdx.x & 63;
    int first, end;
    expert_rows(a, lane, first, end);
    const int tiles = (end - first + height - 1) / height;
    const int sum = wave_sums(tiles);
    if (tile >= __builtin_amdgcn_readlane(sum, 63)) return false;
    expert = __popcll(__ballot(sum <= tile));
    const int m = tile - __builtin_amdgcn_readlane(sum - tiles, expert);
    const int end_row = __builtin_amdgcn_readlane(end, expert);
    row0 = __builtin_amdgcn_readlane(first, expert) + m * height;
    rows = min(height, end_row - row0);
    return true;
}

// Workgroups of a persistent launch: one a CU, a multiple of the 8 XCDs.
inline int persistent_grid() {
    const int n = compute_units() / 8 * 8;
    return n < 8 ? 8 : n > 256 ? 256 : n;
}

// Each enqueues a whole product and returns hipGetLastError().  `workspace`: product_workspace_bytes() of scratch.
constexpr size_t kScratchFloats = (size_t)8 << 20;   // parts of fp32 products
hipError_t launch_f32(Form form, const Args& a, void* workspace, hipStream_t stream);
hipError_t launch_bf16(Form form, const Args& a, bool out_f32, void* workspace, hipStream_t stream);
hipError_t launch_fp8(const Args& a, void* workspace, hipStream_t stream);
// Small products, in tiles of 64 x 64.
hipError_t launch_small(Form form, const Args& a, bool out_f32, hipStream_t stream);
hipError_t launch_small_fp8(const Args& a, hipStream_t stream);
// Forward products of few rows, of bf16 or (with scales) e4m3 matrices.
hipError_t launch_few_rows(const Args& a, bool fp8, hipStream_t stream);
size_t product_workspace_bytes(const moe_product_t& p, int rows);

hipError_t launch_quantize_rows(int rows, int features, int dtype, const void* x, uint8_t* q, float* scales, hipStream_t stream);
hipError_t launch_quantize_weights(const moe_product_t& p, const void* w, uint8_t* q, float* scales, uint8_t* q_t, float* scales_t,
                                   hipStream_t stream);

}  // namespace products
}  // namespace moe
