/*
 * moe_products.h - products of rows grouped by expert, their gradients, and
 * their form in 8-bit floating point.
 *
 * moe_expert_ffn (moe.h) runs whole SwiGLU experts.  The calls here are the
 * products that experts are made of, for callers that put an expert of
 * another form together, train its weights, or hold them in 8 bits: the rows
 * of a matrix are sorted by expert, a table of offsets says where each
 * expert's rows begin, and every row is multiplied by its expert's matrix.
 *
 * The conventions of moe.h hold (device pointers, dense row-major, 16-byte
 * aligned, caller-owned buffers, calls that only enqueue kernels and may be
 * recorded into a HIP graph, status codes, validation before the first HIP
 * call, no floating-point atomics: two calls on the same inputs give bitwise
 * identical outputs), and:
 *   - offsets [E + 1], int32, on the device: rows offsets[e] ... offsets[e + 1] - 1
 *     belong to expert e.  The values ascend and lie in [0, rows]; any number of
 *     experts may have no rows.  Rows before offsets[0] and from offsets[E] on belong to
 *     nobody: they are not read, and the outputs' rows there are left as they were.
 *     The library does not read the table on the host.  Values outside [0, rows] are
 *     taken as the nearer end, so no call reads or writes outside its
 *     buffers; the results of a table that does not ascend are unspecified.
 *   - offsets == NULL, with n_experts == 1: all rows belong to the one expert (a
 *     plain product).
 *   - Limits: out_features and in_features are multiples of 64 up to 1048576,
 *     n_experts <= 64, rows <= 8388608, and one expert's matrix has less than 2^31
 *     elements.
 *   - rows == 0 is MOE_OK; the per-row buffers may then be NULL.
 *   - An output overlaps no other buffer of its call.
 *   - Sums are held in fp32 (one rounding to the output's type).  For fp32
 *     operands the products are fp32 products, not ones of shorter formats.
 *   - NaN and infinities go where the formulas take them; rows of other experts, rows of
 *     nobody and memory behind the buffers never reach a result.
 */
#ifndef MOE_PRODUCTS_H
#define MOE_PRODUCTS_H

#include "moe.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct {
    int32_t n_experts;    /* E                                             */
    int32_t out_features; /* N: rows of an expert's matrix                  */
    int32_t in_features;  /* K: columns of an expert's matrix               */
    int32_t dtype;        /* moe_dtype_t of the matrices that are not 8-bit */
} moe_product_t;

/*
 * Scratch bytes that the products below need for calls of at most `max_rows`
 * rows (one size for all of them).  It is what the largest calls of a dtype need, 66.9 MB for
 * MOE_BF16 and the 8-bit product, 33.6 MB for MOE_F32, whatever the features and rows: one workspace serves products of all
 * shapes of its dtype, one after another, and calls too small to use any of it ask for it too.
 * The conventions of moe.h for workspaces
 * hold: nothing in it needs initialising, two calls that overlap in time need
 * two of them.
 * Errors: MOE_ERR_NULL, MOE_ERR_SHAPE, MOE_ERR_DTYPE.
 */
int moe_product_workspace_bytes(const moe_product_t* product, int32_t max_rows, size_t* out_bytes);

/*
 * y[r, n] = sum_k x[r, k] * w[e, n, k], e the expert of row r.
 *   x [rows, K] in, w [E, N, K] in, y [rows, N] out, all of product->dtype
 */
int moe_grouped_product(const moe_product_t* product, int32_t rows, const void* x, const int32_t* offsets, const void* w,
                        void* y, void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * Gradient of moe_grouped_product with respect to its rows:
 *   dx[r, k] = sum_n dy[r, n] * w[e, n, k]
 *   dy [rows, N] in, w [E, N, K] in, dx [rows, K] out, all of product->dtype
 */
int moe_grouped_product_dgrad(const moe_product_t* product, int32_t rows, const void* dy, const int32_t* offsets,
                              const void* w, void* dx, void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * Gradient of moe_grouped_product with respect to the experts' matrices:
 *   dw[e, n, k] = sum over the rows r of expert e of dy[r, n] * x[r, k]
 * accumulate = 0 overwrites (an expert without rows gets zeros), 1 adds to the
 * existing values (gradients over several micro-batches).
 *   dy [rows, N], x [rows, K] in, product->dtype
 *   dw [E, N, K] out, dw_dtype: MOE_F32, or product->dtype without accumulate
 *   (sums over calls are held in fp32: MOE_ERR_DTYPE otherwise)
 */
int moe_grouped_product_wgrad(const moe_product_t* product, int32_t rows, const void* dy, const void* x,
                              const int32_t* offsets, void* dw, int32_t dw_dtype, int32_t accumulate, void* workspace,
                              size_t workspace_bytes, void* hip_stream);

/*
 * Block-scaled 8-bit floating point: a matrix is held as e4m3 numbers (OCP: 4 exponent bits, 3
 * mantissa bits, largest value 448, no infinities) and an fp32 scale for each
 * block; a value is number * scale.  Blocks are 128 consecutive
 * values of a row (activations), or tiles of 128 x 128 (weights); the last ones of
 * a dimension that 128 does not divide hold 64.
 *   scale  = max(largest absolute value of the block, 2^-60) / 448, rounded to nearest
 *   number = value / scale, rounded to fp32 and then to e4m3, both to nearest even; what becomes zero keeps
 *            the value's sign
 * A block with an infinity or a NaN becomes NaN altogether, its scale too.
 *
 * moe_quantize_rows_fp8:    x [rows, features] -> q [rows, features], scales [rows, ceil(features / 128)]
 * moe_quantize_weights_fp8: w [E, N, K] -> q [E, N, K], scales [E, ceil(N / 128), ceil(K / 128)] and, where
 *   q_t and scales_t are not NULL (both or neither), the same numbers transposed:
 *   q_t [E, K, N], scales_t [E, ceil(K / 128), ceil(N / 128)].  moe_grouped_product_fp8 with
 *   those, quantised rows of dy and a product of swapped features is the gradient with respect to the rows.
 *   dtype: moe_dtype_t of x; features: as in_features above; rows <= 8388608
 */
int moe_quantize_rows_fp8(int32_t rows, int32_t features, int32_t dtype, const void* x, uint8_t* q, float* scales,
                          void* hip_stream);
int moe_quantize_weights_fp8(const moe_product_t* product, const void* w, uint8_t* q, float* scales, uint8_t* q_t,
                             float* scales_t, void* hip_stream);

/*
 * moe_grouped_product on block-scaled operands:
 *   y[r, n] = sum over blocks b of x_scales[r, b] * w_scales[e, n / 128, b] * (sum over k in b of xq[r, k] * wq[e, n, k])
 *   xq [rows, K], x_scales [rows, ceil(K / 128)], wq [E, N, K], w_scales [E, ceil(N / 128), ceil(K / 128)] in;
 *   y [rows, N] out, bf16: product->dtype must be MOE_BF16
 * The sum inside a block is the matrix instruction's, which keeps fewer bits than fp32.  It adds eight products of consecutive k
 * at a time, and of each of them what lies below 2^(E - 13) is lost, E the largest sum of two exponents among the eight (-6 for
 * a subnormal number): at most 7 * 2^-13 of the block's sum of absolute products, 8 times that where the largest of the eight products has a
 * subnormal factor.  On normally distributed numbers it was at most 2e-5 of it (1.4e-6 on average), on random bit patterns 2e-4 (2e-5).
 * The sums of eight and the blocks are added in fp32.
 * The two scales of a block are multiplied first, in fp32: a product of scales beyond its range makes the block infinite, or NaN where its sum is
 * zero, and one below 2^-126 has fewer bits.  (Of quantised operands: where the product of their largest values in the block exceeds 2^145 or is
 * below 2^-108.)
 */
int moe_grouped_product_fp8(const moe_product_t* product, int32_t rows, const uint8_t* xq, const float* x_scales,
                            const int32_t* offsets, const uint8_t* wq, const float* w_scales, void* y, void* workspace,
                            size_t workspace_bytes, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* MOE_PRODUCTS_H */
