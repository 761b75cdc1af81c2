// Grouped products on the fp32 matrix instructions: the forward product and both gradients of one tile kernel.
//
// A workgroup computes a square tile of the output, its four wavefronts a quarter each.  Every K step of 16 goes through LDS as
// [c][row] for both operands, whichever way they lie in memory: an operand whose contraction is contiguous is written transposed,
// one whose rows are (the weights of dgrad, both operands of wgrad) as it is.  v_mfma_f32_16x16x4_f32 takes one number a lane,
// row lane % 16 and c lane / 16, so a fragment is one ds_read_b32 without bank conflicts (a row of the LDS is the tile + 16 floats,
// 16 banks further than the one before).  The features are the instruction's first operand, so that a lane ends
// up with four consecutive ones of a row.
#include "bf16_utils.h"
#include "products_internal.h"

namespace moe {
namespace products {
namespace {

typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(2))) float f32x2;

constexpr int kThreads = 256, kBK = 16;

__device__ inline f32x4 load4(const float* p) { return *reinterpret_cast<const f32x4*>(p); }
__device__ inline f32x4 load4(const uint16_t* p) {
    const uint2 v = *reinterpret_cast<const uint2*>(p);
    return f32x4{__uint_as_float(v.x << 16), __uint_as_float(v.x & 0xffff0000u), __uint_as_float(v.y << 16), __uint_as_float(v.y & 0xffff0000u)};
}
__device__ inline f32x4 load4(const uint8_t* p) {
    const int v = *reinterpret_cast<const int*>(p);
    const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8(v, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(v, true);
    return f32x4{a[0], a[1], b[0], b[1]};
}
__device__ inline void store4(float* p, f32x4 v) { *reinterpret_cast<f32x4*>(p) = v; }
__device__ inline void store4(uint16_t* p, f32x4 v) {
    *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
}

// One operand of a tile: `base` is its element (row 0, c 0).  ROWS: the contraction is contiguous, consecutive rows are `ld` apart; else
// rows are contiguous and consecutive c are `ld` apart.  Rows from `limit` on don't exist, nor do c from `depth` on.
template <typename T, bool ROWS, int TILE>
struct Operand {
    static constexpr int kQuads = TILE * kBK / 4 / kThreads;
    const T* base;
    size_t ld;
    int limit, depth;
    const float* scales;   // per row of the tile (ROWS), or a single one; null: none
    size_t scale_ld;
    f32x4 v[kQuads];

    __device__ void load(int c0) {
#pragma unroll
        for (int i = 0; i < kQuads; ++i) {
            const int t = threadIdx.x + i * kThreads;
            const int row = ROWS ? t / 4 : t % (TILE / 4) * 4, c = c0 + (ROWS ? t % 4 * 4 : t / (TILE / 4));
            v[i] = f32x4{0.f, 0.f, 0.f, 0.f};
            if (row < limit && c < depth) {
                v[i] = load4(base + (ROWS ? (size_t)row * ld + c : (size_t)c * ld + row));
                if constexpr (sizeof(T) == 1) v[i] *= scales[row * scale_ld + c / 128];
            }
        }
    }
    __device__ void stage(float* lds) const {
#pragma unroll
        for (int i = 0; i < kQuads; ++i) {
            const int t = threadIdx.x + i * kThreads;
            if constexpr (ROWS) {
#pragma unroll
                for (int j = 0; j < 4; ++j) lds[(t % 4 * 4 + j) * (TILE + 16) + t / 4] = v[i][j];
            } else {
                *reinterpret_cast<f32x4*>(lds + t / (TILE / 4) * (TILE + 16) + t % (TILE / 4) * 4) = v[i];
            }
        }
    }
};

template <typename T, typename O, int FORM, int TILE>
__global__ __launch_bounds__(kThreads, 2) void product_kernel(Args a) {
    constexpr int kF = TILE / 32;   // fragments of each operand a wavefront
    __shared__ __attribute__((aligned(16))) float lds[2][2][kBK * (TILE + 16)];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int features = FORM == kForward ? a.n : a.k;
    const int f_tiles = (features + TILE - 1) / TILE;
    const int f0 = blockIdx.x % f_tiles * TILE;
    const int m = blockIdx.x / f_tiles;
    int e, row0, rows, depth;
    Operand<T, FORM == kForward, TILE> p;
    Operand<T, FORM != kWgrad, TILE> q;
    O* out;
    if constexpr (FORM == kWgrad) {
        const int n_tiles = (a.n + TILE - 1) / TILE;
        e = m / n_tiles;
        const int n0 = m % n_tiles * TILE;
        int first, end;
        expert_rows(a, lane, first, end);
        first = __builtin_amdgcn_readlane(first, e);
        depth = __builtin_amdgcn_readlane(end, e) - first;
        rows = min(TILE, a.n - n0);
        q.base = static_cast<const T*>(a.q) + (size_t)first * a.n + n0;
        q.ld = a.n;
        p.base = static_cast<const T*>(a.p) + (size_t)first * a.k + f0;
        p.ld = a.k;
        out = static_cast<O*>(a.out) + ((size_t)e * a.n + n0) * a.k + f0;
    } else {
        if (!find_row_tile(a, m, TILE, e, row0, rows)) return;
        depth = FORM == kForward ? a.k : a.n;
        q.base = static_cast<const T*>(a.q) + (size_t)row0 * depth;
        q.ld = depth;
        p.base = static_cast<const T*>(a.p) + (size_t)e * a.n * a.k + (FORM == kForward ? (size_t)f0 * a.k : f0);
        p.ld = a.k;
        out = static_cast<O*>(a.out) + (size_t)row0 * features + f0;
        if constexpr (sizeof(T) == 1) {
            const int kb = (a.k + 127) / 128, nb = (a.n + 127) / 128;
            q.scales = a.q_scales + (size_t)row0 * kb;
            q.scale_ld = kb;
            p.scales = a.p_scales + ((size_t)e * nb + f0 / 128) * kb;
            p.scale_ld = 0;
        }
    }
    q.limit = rows;
    p.limit = min(TILE, features - f0);
    q.depth = p.depth = depth;

    const int wf = wave % 2 * (TILE / 2), wr = wave / 2 * (TILE / 2);   // this wavefront's quarter
    const int at = lane / 16 * (TILE + 16) + lane % 16;
    f32x4 acc[kF][kF];   // [feature fragment][row fragment]
#pragma unroll
    for (int i = 0; i < kF; ++i)
#pragma unroll
        for (int j = 0; j < kF; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    const int steps = (depth + kBK - 1) / kBK;
    if (steps > 0) {
        p.load(0);
        q.load(0);
    }
    for (int s = 0; s < steps; ++s) {
        float *lp = lds[s & 1][0], *lq = lds[s & 1][1];
        p.stage(lp);
        q.stage(lq);
        __syncthreads();   // (the other pair of stages is written after the next one, which everybody reaches behind its reads)
        if (s + 1 < steps) {
            p.load((s + 1) * kBK);
            q.load((s + 1) * kBK);
        }
#pragma unroll
        for (int c = 0; c < kBK; c += 4) {
            float fp[kF], fq[kF];
#pragma unroll
            for (int i = 0; i < kF; ++i) {
                fp[i] = lp[c * (TILE + 16) + at + wf + i * 16];
                fq[i] = lq[c * (TILE + 16) + at + wr + i * 16];
            }
#pragma unroll
            for (int i = 0; i < kF; ++i)
#pragma unroll
                for (int j = 0; j < kF; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(fp[i], fq[j], acc[i][j], 0, 0, 0);
        }
    }
#pragma unroll
    for (int j = 0; j < kF; ++j) {
        const int row = wr + j * 16 + lane % 16;
        if (row >= rows) continue;
#pragma unroll
        for (int i = 0; i < kF; ++i) {
            const int f = wf + i * 16 + lane / 16 * 4;
            if (f >= p.limit) continue;
            O* to = out + (size_t)row * features + f;
            f32x4 v = acc[i][j];
            if constexpr (FORM == kWgrad && sizeof(O) == 4)
                if (a.accumulate) v += load4(to);
            store4(to, v);
        }
    }
}

template <typename T, typename O, int FORM, int TILE>
hipError_t launch(const Args& a, hipStream_t stream) {
    const long f_tiles = ((FORM == kForward ? a.n : a.k) + TILE - 1) / TILE;
    const long m_tiles = FORM == kWgrad ? (long)a.experts * ((a.n + TILE - 1) / TILE) : most_row_tiles(a.rows, a.experts, TILE);
    product_kernel<T, O, FORM, TILE><<<dim3((unsigned)(f_tiles * m_tiles)), dim3(kThreads), 0, stream>>>(a);
    return hipGetLastError();
}

template <typename T, typename O>
hipError_t launch_form(Form form, const Args& a, hipStream_t stream) {
    switch (form) {
        case kForward: return launch<T, O, kForward, 64>(a, stream);
        case kDgrad: return launch<T, O, kDgrad, 64>(a, stream);
        default: return launch<T, O, kWgrad, 64>(a, stream);
    }
}

}  // namespace

hipError_t launch_f32(Form form, const Args& a, hipStream_t stream) { return launch_form<float, float>(form, a, stream); }

}  // namespace products
}  // namespace moe
