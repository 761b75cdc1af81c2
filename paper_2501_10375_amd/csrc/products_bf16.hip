// Launches of the grouped bf16 products, see products_bf16.h.
#include "products_bf16.h"

namespace moe {
namespace products {
namespace {

template <int FORM, bool OUT32>
hipError_t launch(const Args& a, void* workspace, hipStream_t stream) {
    float* scratch = static_cast<float*>(workspace);
    Told* told = reinterpret_cast<Told*>(static_cast<char*>(workspace) + kScratchBytes);
    const int grid = persistent_grid();
    product_gemm_kernel<FORM, OUT32><<<grid, 256, 0, stream>>>(a, scratch, told);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || !may_cut(static_cast<Form>(FORM), a, kStepC, grid)) return e;
    join_pieces_kernel<OUT32><<<kJoinWorkgroups, 256, 0, stream>>>(a.out, FORM == kForward ? a.n : a.k, a.accumulate, scratch, told);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_bf16(Form form, const Args& a, bool out_f32, void* workspace, hipStream_t stream) {
    switch (form) {
        case kForward: return launch<kForward, false>(a, workspace, stream);
        case kDgrad: return launch<kDgrad, false>(a, workspace, stream);
        default: return out_f32 ? launch<kWgrad, true>(a, workspace, stream) : launch<kWgrad, false>(a, workspace, stream);
    }
}

size_t product_workspace_bytes(const moe_product_t& p, int) { return p.dtype == MOE_F32 ? kScratchFloats * sizeof(float) : kWorkspaceBytes; }

}  // namespace products
}  // namespace moe
