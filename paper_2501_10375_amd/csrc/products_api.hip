// C ABI of the grouped products: argument validation on the host, then kernel launches on the caller's stream.  See
// include/moe_products.h for the contract of each call.
#include "products_internal.h"

using namespace moe;
using products::Args;

namespace {

constexpr int kMaxFeatures = 1 << 20, kMaxRows = 1 << 23;

bool bad_features(int f) { return f <= 0 || f > kMaxFeatures || f % 64 != 0; }

int check_product(const moe_product_t* p) {
    if (p == nullptr) return MOE_ERR_NULL;
    if (p->dtype != MOE_F32 && p->dtype != MOE_BF16) return MOE_ERR_DTYPE;
    if (bad_features(p->out_features) || bad_features(p->in_features)) return MOE_ERR_SHAPE;
    if ((int64_t)p->out_features * p->in_features >= (int64_t)1 << 31) return MOE_ERR_SHAPE;
    if (p->n_experts < 1 || p->n_experts > 64) return MOE_ERR_SHAPE;
    return MOE_OK;
}

bool bad_rows(int rows) { return rows < 0 || rows > kMaxRows; }

template <size_t N>
int check_pointers(const void* const (&ptrs)[N], bool required) {
    for (const void* p : ptrs)
        if (p == nullptr && required) return MOE_ERR_NULL;
    for (const void* p : ptrs)
        if ((reinterpret_cast<uintptr_t>(p) & 15u) != 0) return MOE_ERR_ALIGN;
    return MOE_OK;
}

// Everything that a product checks: `per_row` buffers may be null in a call without rows.
template <size_t N, size_t M>
int check_call(const moe_product_t* product, int rows, const void* const (&always)[N], const void* const (&per_row)[M],
               const int32_t* offsets, const void* workspace, size_t workspace_bytes) {
    if (int rc = check_product(product)) return rc;
    if (bad_rows(rows)) return MOE_ERR_SHAPE;
    if (offsets == nullptr && product->n_experts != 1) return MOE_ERR_NULL;
    if (workspace == nullptr) return MOE_ERR_NULL;
    if (int rc = check_pointers(always, true)) return rc;
    if (int rc = check_pointers(per_row, rows > 0)) return rc;
    const void* const others[] = {offsets, workspace};
    if (int rc = check_pointers(others, false)) return rc;
    return workspace_bytes < products::product_workspace_bytes(*product, rows) ? MOE_ERR_WORKSPACE : MOE_OK;
}

int status(hipError_t e) { return e == hipSuccess ? MOE_OK : MOE_ERR_DEVICE; }

products::Size size_of(const Args& a) { return {a.experts, a.rows, a.n, a.k}; }

int enqueue(products::Form form, const moe_product_t& p, int32_t rows, const void* q, const void* second, const int32_t* offsets,
            void* out, bool out_f32, int accumulate, void* workspace, void* hip_stream) {
    const Args a = {q, second, out, offsets, p.n_experts, rows, p.out_features, p.in_features, nullptr, nullptr, accumulate};
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    if (p.dtype == MOE_F32) return status(products::launch_f32(form, a, workspace, stream));
    switch (products::choose_way(form, size_of(a), false)) {
        case products::kFewRows: return status(products::launch_few_rows(a, false, stream));
        case products::kSmallTiles: return status(products::launch_small(form, a, out_f32, stream));
        default: return status(products::launch_bf16(form, a, out_f32, workspace, stream));
    }
}

}  // namespace

extern "C" {

int moe_product_workspace_bytes(const moe_product_t* product, int32_t max_rows, size_t* out_bytes) {
    if (out_bytes == nullptr) return MOE_ERR_NULL;
    if (int rc = check_product(product)) return rc;
    if (bad_rows(max_rows)) return MOE_ERR_SHAPE;
    *out_bytes = products::product_workspace_bytes(*product, max_rows);
    return MOE_OK;
}

int moe_grouped_product(const moe_product_t* product, int32_t rows, const void* x, const int32_t* offsets, const void* w,
                        void* y, void* workspace, size_t workspace_bytes, void* hip_stream) {
    const void* const always[] = {w};
    const void* const per_row[] = {x, y};
    if (int rc = check_call(product, rows, always, per_row, offsets, workspace, workspace_bytes)) return rc;
    if (rows == 0) return MOE_OK;
    return enqueue(products::kForward, *product, rows, x, w, offsets, y, false, 0, workspace, hip_stream);
}

int moe_grouped_product_dgrad(const moe_product_t* product, int32_t rows, const void* dy, const int32_t* offsets,
                              const void* w, void* dx, void* workspace, size_t workspace_bytes, void* hip_stream) {
    const void* const always[] = {w};
    const void* const per_row[] = {dy, dx};
    if (int rc = check_call(product, rows, always, per_row, offsets, workspace, workspace_bytes)) return rc;
    if (rows == 0) return MOE_OK;
    return enqueue(products::kDgrad, *product, rows, dy, w, offsets, dx, false, 0, workspace, hip_stream);
}

int moe_grouped_product_wgrad(const moe_product_t* product, int32_t rows, const void* dy, const void* x,
                              const int32_t* offsets, void* dw, int32_t dw_dtype, int32_t accumulate, void* workspace,
                              size_t workspace_bytes, void* hip_stream) {
    const void* const always[] = {dw};
    const void* const per_row[] = {dy, x};
    if (int rc = check_call(product, rows, always, per_row, offsets, workspace, workspace_bytes)) return rc;
    if (dw_dtype != MOE_F32 && (dw_dtype != product->dtype || accumulate != 0)) return MOE_ERR_DTYPE;
    if (rows == 0 && accumulate != 0) return MOE_OK;
    return enqueue(products::kWgrad, *product, rows, dy, x, offsets, dw, dw_dtype == MOE_F32, accumulate != 0, workspace, hip_stream);
}

int moe_quantize_rows_fp8(int32_t rows, int32_t features, int32_t dtype, const void* x, uint8_t* q, float* scales,
                          void* hip_stream) {
    if (dtype != MOE_F32 && dtype != MOE_BF16) return MOE_ERR_DTYPE;
    if (bad_rows(rows) || bad_features(features)) return MOE_ERR_SHAPE;
    const void* const ptrs[] = {x, q, scales};
    if (int rc = check_pointers(ptrs, rows > 0)) return rc;
    if (rows == 0) return MOE_OK;
    return status(products::launch_quantize_rows(rows, features, dtype, x, q, scales, static_cast<hipStream_t>(hip_stream)));
}

int moe_quantize_weights_fp8(const moe_product_t* product, const void* w, uint8_t* q, float* scales, uint8_t* q_t,
                             float* scales_t, void* hip_stream) {
    if (int rc = check_product(product)) return rc;
    const void* const ptrs[] = {w, q, scales};
    if (int rc = check_pointers(ptrs, true)) return rc;
    const void* const transposed[] = {q_t, scales_t};
    if (int rc = check_pointers(transposed, q_t != nullptr || scales_t != nullptr)) return rc;
    return status(products::launch_quantize_weights(*product, w, q, scales, q_t, scales_t, static_cast<hipStream_t>(hip_stream)));
}

int moe_grouped_product_fp8(const moe_product_t* product, int32_t rows, const uint8_t* xq, const float* x_scales,
                            const int32_t* offsets, const uint8_t* wq, const float* w_scales, void* y, void* workspace,
                            size_t workspace_bytes, void* hip_stream) {
    const void* const always[] = {wq, w_scales};
    const void* const per_row[] = {xq, x_scales, y};
    if (int rc = check_call(product, rows, always, per_row, offsets, workspace, workspace_bytes)) return rc;
    if (product->dtype != MOE_BF16) return MOE_ERR_DTYPE;
    if (rows == 0) return MOE_OK;
    const Args a = {xq, wq, y, offsets, product->n_experts, rows, product->out_features, product->in_features, x_scales, w_scales, 0};
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    switch (products::choose_way(products::kForward, size_of(a), true)) {
        case products::kFewRows: return status(products::launch_few_rows(a, true, stream));
        case products::kSmallTiles: return status(products::launch_small_fp8(a, stream));
        default: return status(products::launch_fp8(a, workspace, stream));
    }
}

}  // extern "C"
