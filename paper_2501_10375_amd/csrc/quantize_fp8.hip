// Quantisation to e4m3 with a scale for each block of 128 values of a row or tile of 128 x 128.
//
// number = e4m3(fp32(value / scale)), scale = fp32(max(amax, 2^-60) / 448).  Both roundings are exact ones, so the quotient is a true
// fp32 division; with r = 1 / scale it is q0 = x r, then q0 + r (x - q0 scale) in two fused operations, which is the correctly rounded
// quotient for a correctly rounded r (Markstein).  2^-60 keeps the remainder of every value that does not become zero
// a normal number.  amax is a maximum of bit patterns without their sign: those of infinities and NaN are the
// largest, and a block that has one gets a NaN for its scale, which makes every quotient NaN.
#include "bf16_utils.h"
#include "products_internal.h"

namespace moe {
namespace products {
namespace {

typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) unsigned int u32x4;

constexpr int kThreads = 256, kBlock = 128;

struct Eight {
    float v[8];
    __device__ void load(const float* p) {
        const f32x4 a = *reinterpret_cast<const f32x4*>(p), b = *reinterpret_cast<const f32x4*>(p + 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = a[i], v[4 + i] = b[i];
    }
    __device__ void load(const uint16_t* p) {
        const u32x4 a = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(a[i] << 16);
            v[2 * i + 1] = __uint_as_float(a[i] & 0xffff0000u);
        }
    }
    __device__ uint32_t amax_bits() const {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(v[i]) & 0x7fffffffu);
        return m;
    }
    __device__ uint2 quantised(float scale, float r) const {
        float q[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float q0 = v[i] * r;
            q[i] = fmaf(-fmaf(q0, scale, -v[i]), r, q0);   // (turned twice, so that a remainder of zero is -0, which leaves q0 its sign where that is zero too)
        }
        int lo = __builtin_amdgcn_cvt_pk_fp8_f32(q[0], q[1], 0, false), hi = __builtin_amdgcn_cvt_pk_fp8_f32(q[4], q[5], 0, false);
        lo = __builtin_amdgcn_cvt_pk_fp8_f32(q[2], q[3], lo, true);
        hi = __builtin_amdgcn_cvt_pk_fp8_f32(q[6], q[7], hi, true);
        return make_uint2((uint32_t)lo, (uint32_t)hi);
    }
};

__device__ inline float scale_of(uint32_t amax_bits) {
    if (amax_bits >= 0x7f800000u) return __builtin_nanf("");
    return fmaxf(__uint_as_float(amax_bits), 0x1p-60f) / 448.f;
}

// Rows: 16 lanes take a block, eight values each; a wavefront has kInFlight * 4 blocks requested at a time.
constexpr int kInFlight = 4;

template <typename T>
__global__ __launch_bounds__(kThreads) void quantize_rows_kernel(const T* __restrict__ x, uint8_t* __restrict__ q, float* __restrict__ scales,
                                                                 long blocks, int features, int row_blocks) {
    const int at = threadIdx.x % 16 * 8;
    const long first = (long)blockIdx.x * (kThreads / 16 * kInFlight) + threadIdx.x / 16;
    Eight v[kInFlight];
    long from[kInFlight];   // element of the lane's first value, -1: none
#pragma unroll
    for (int i = 0; i < kInFlight; ++i) {
        const long b = first + i * (kThreads / 16);
        const long row = b / row_blocks;
        const int c = (int)(b - row * row_blocks) * kBlock + at;
        from[i] = b < blocks && c < features ? row * features + c : -1;
        if (from[i] >= 0) v[i].load(x + from[i]);
        else v[i] = Eight{};
    }
#pragma unroll
    for (int i = 0; i < kInFlight; ++i) {
        uint32_t m = v[i].amax_bits();
#pragma unroll
        for (int d = 8; d > 0; d >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, d, 64));
        const float scale = scale_of(m), r = 1.f / scale;
        if (from[i] < 0) continue;
        *reinterpret_cast<uint2*>(q + from[i]) = v[i].quantised(scale, r);
        if (at == 0) scales[first + i * (kThreads / 16)] = scale;
    }
}

// Weights: a workgroup takes a tile.  A thread holds eight columns of eight consecutive rows; the transposed numbers go through LDS, so that
// both forms are written in whole lines.
template <typename T>
__global__ __launch_bounds__(kThreads) void quantize_weights_kernel(const T* __restrict__ w, uint8_t* __restrict__ q, float* __restrict__ scales,
                                                                    uint8_t* __restrict__ q_t, float* __restrict__ scales_t, int n, int k) {
    __shared__ uint32_t waves_max[kThreads / 64];
    __shared__ __attribute__((aligned(16))) unsigned char turned[kBlock * (kBlock + 16)];   // [column][row]
    const int nb = (n + kBlock - 1) / kBlock, kb = (k + kBlock - 1) / kBlock;
    const int bk = blockIdx.x % kb, bn = blockIdx.x / kb % nb, e = blockIdx.x / kb / nb;
    const int c = threadIdx.x % 16 * 8, r0 = threadIdx.x / 16 * 8;
    const int height = min(kBlock, n - bn * kBlock), width = min(kBlock, k - bk * kBlock);
    const size_t origin = ((size_t)e * n + (size_t)bn * kBlock) * k + (size_t)bk * kBlock;
    const bool inside = c < width && r0 < height;   // (both are multiples of 8, like the thread's square)
    Eight v[8];
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (inside) v[i].load(w + origin + (size_t)(r0 + i) * k + c);
        else v[i] = Eight{};
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, v[i].amax_bits());
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, d, 64));
    if (threadIdx.x % 64 == 0) waves_max[threadIdx.x / 64] = m;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kThreads / 64; ++i) m = max(m, waves_max[i]);
    const float scale = scale_of(m), r = 1.f / scale;
    uint2 out[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        out[i] = v[i].quantised(scale, r);
        if (inside) *reinterpret_cast<uint2*>(q + origin + (size_t)(r0 + i) * k + c) = out[i];
    }
    if (threadIdx.x == 0) {
        scales[((size_t)e * nb + bn) * kb + bk] = scale;
        if (scales_t != nullptr) scales_t[((size_t)e * kb + bk) * nb + bn] = scale;
    }
    if (q_t == nullptr) return;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        uint64_t column = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) column |= (uint64_t)(((j < 4 ? out[i].x : out[i].y) >> (j % 4 * 8)) & 0xffu) << (i * 8);
        *reinterpret_cast<uint64_t*>(turned + (c + j) * (kBlock + 16) + r0) = column;
    }
    __syncthreads();
    const size_t origin_t = ((size_t)e * k + (size_t)bk * kBlock) * n + (size_t)bn * kBlock;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int row = i * 32 + threadIdx.x / 8, col = threadIdx.x % 8 * 16;
        if (row < width && col < height)
            *reinterpret_cast<u32x4*>(q_t + origin_t + (size_t)row * n + col) = *reinterpret_cast<const u32x4*>(turned + row * (kBlock + 16) + col);
    }
}

}  // namespace

hipError_t launch_quantize_rows(int rows, int features, int dtype, const void* x, uint8_t* q, float* scales, hipStream_t stream) {
    const int row_blocks = (features + kBlock - 1) / kBlock;
    const long blocks = (long)rows * row_blocks;
    constexpr long per_group = kThreads / 16 * kInFlight;
    const dim3 grid((unsigned)((blocks + per_group - 1) / per_group));
    if (dtype == MOE_F32)
        quantize_rows_kernel<<<grid, kThreads, 0, stream>>>(static_cast<const float*>(x), q, scales, blocks, features, row_blocks);
    else
        quantize_rows_kernel<<<grid, kThreads, 0, stream>>>(static_cast<const uint16_t*>(x), q, scales, blocks, features, row_blocks);
    return hipGetLastError();
}

hipError_t launch_quantize_weights(const moe_product_t& p, const void* w, uint8_t* q, float* scales, uint8_t* q_t, float* scales_t,
                                   hipStream_t stream) {
    const long nb = (p.out_features + kBlock - 1) / kBlock, kb = (p.in_features + kBlock - 1) / kBlock;
    const dim3 grid((unsigned)(p.n_experts * nb * kb));
    if (p.dtype == MOE_F32)
        quantize_weights_kernel<<<grid, kThreads, 0, stream>>>(static_cast<const float*>(w), q, scales, q_t, scales_t, p.out_features, p.in_features);
    else
        quantize_weights_kernel<<<grid, kThreads, 0, stream>>>(static_cast<const uint16_t*>(w), q, scales, q_t, scales_t, p.out_features, p.in_features);
    return hipGetLastError();
}

}  // namespace products
}  // namespace moe
