// The gated feed-forward block's products for every type and size the entry points take: v_mfma_f32_16x16x4_f32 on fp32 values (bf16 operands are widened as
// their tiles go to LDS).
//
// Forward: one tile of x against one of each weight matrix, two accumulators; the activation and the product with U happen in registers.  dx: one accumulator
// over both pairs of operands.  64 x 64 outputs to a work-group of 4 wavefronts stacked along the rows, K tiles of 32 through registers into LDS, the next one
// requested while one is multiplied.  Operands are swapped (the accumulator is the transposed block), so that a lane holds 4 consecutive columns of its row.
// Bound by the fp32 matrix rate where rows are many (7 684 x 256 x 1024 forward 84 us: 96 TFLOP/s of 131 that a large product reaches); bf16 comes here with force_generic only.
// Contraction step (u, j) of a tile uses k = 16 u + 4 g + j for both operands: fragments are float4 reads along k.
#include "gated_mlp.hpp"
#include "gemm_epilogue.hpp"
#include <type_traits>

namespace {

constexpr int GK = 32, GLD = GK + 4, GTILE = 64 * GLD;

__device__ __forceinline__ f32x4_t mfma4(float a, float b, f32x4_t c) { return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0); }

// 64 rows x 32 k of a row-major operand, 8 values of a row to a thread
template <class T> struct Rows64 {
    float v[8];
    __device__ __forceinline__ void load(const T* src, int r0, int rows, int k0, int K) {
        const int r = r0 + (threadIdx.x >> 2), k = k0 + (threadIdx.x & 3) * 8;
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = 0.f;
        if (r < rows && k < K) Vec8<T>::load(src + (size_t)r * K + k, v);          // (K is a multiple of 8)
    }
    __device__ __forceinline__ void store(float* tile) const {
        Vec8<float>::store(tile + (threadIdx.x >> 2) * GLD + (threadIdx.x & 3) * 8, v);
    }
};

template <class T> __device__ __forceinline__ void put4(T* p, const f32x4_t& v) {
    typedef T T4 __attribute__((ext_vector_type(4)));
    T4 x;
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = from_f32<T>(v[e]);
    *reinterpret_cast<T4*>(p) = x;
}
template <class T> __device__ __forceinline__ f32x4_t get4(const T* p) {
    typedef T T4 __attribute__((ext_vector_type(4)));
    const T4 x = *reinterpret_cast<const T4*>(p);
    return f32x4_t{to_f32(x[0]), to_f32(x[1]), to_f32(x[2]), to_f32(x[3])};
}

// ACT: an activation, or -1: dx
template <class T, int ACT> __global__ __launch_bounds__(256, 2) void glu_general_kernel(GluArgs a, int tiles_m, int tiles_n) {
    constexpr bool FWD = ACT >= 0;
    constexpr int NB = FWD ? 2 : 1;
    __shared__ __attribute__((aligned(16))) float lds[(1 + NB) * GTILE];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15, g = lane >> 4;
    const int logical = xcd_contiguous(blockIdx.x, gridDim.x);
    const int m0 = logical / tiles_n * 64, n0 = logical % tiles_n * 64;
    const int K = FWD ? a.d : a.ff, N = FWD ? a.ff : a.d, steps = (K + GK - 1) / GK, all = FWD ? steps : 2 * steps;
    f32x4_t acc[NB][4];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[b][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    Rows64<T> ta, tb[NB];
    auto fetch = [&](int step) {
        const bool second = !FWD && step >= steps;
        const int k0 = (second ? step - steps : step) * GK;
        ta.load((const T*)(FWD ? a.x : second ? a.du : a.dg), m0, a.rows, k0, K);
        tb[0].load((const T*)(second ? a.wu : a.wg), n0, N, k0, K);
        if constexpr (FWD) tb[NB - 1].load((const T*)a.wu, n0, N, k0, K);
    };
    fetch(0);
    for (int step = 0; step < all; ++step) {
        __syncthreads();
        ta.store(lds);
#pragma unroll
        for (int b = 0; b < NB; ++b) tb[b].store(lds + (1 + b) * GTILE);
        __syncthreads();
        if (step + 1 < all) fetch(step + 1);
#pragma unroll
        for (int u = 0; u < GK / 16; ++u) {
            const float4 x = *reinterpret_cast<const float4*>(lds + (wave * 16 + col) * GLD + 16 * u + 4 * g);
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float4 w = *reinterpret_cast<const float4*>(lds + (1 + b) * GTILE + (j * 16 + col) * GLD + 16 * u + 4 * g);
                    acc[b][j] = mfma4(w.x, x.x, acc[b][j]);
                    acc[b][j] = mfma4(w.y, x.y, acc[b][j]);
                    acc[b][j] = mfma4(w.z, x.z, acc[b][j]);
                    acc[b][j] = mfma4(w.w, x.w, acc[b][j]);
                }
        }
    }
    const int m = m0 + wave * 16 + col;
    if (m >= a.rows) return;
    const bool valid = !a.row_valid || a.row_valid[m] >= 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int n = n0 + 16 * j + 4 * g;
        if (n >= N) continue;
        const size_t at = (size_t)m * N + n;
        f32x4_t v = acc[0][j];
        if constexpr (FWD) {
            f32x4_t u = acc[NB - 1][j], h;
            if (a.bg) v += get4((const T*)a.bg + n);
            if (a.bu) u += get4((const T*)a.bu + n);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                v[e] = valid ? v[e] : 0.f;
                u[e] = valid ? u[e] : 0.f;
                h[e] = valid ? glu_act<ACT>(v[e]) * u[e] : 0.f;
            }
            put4((T*)a.h + at, h);
            if (a.g) {
                put4((T*)a.g + at, v);
                put4((T*)a.u + at, u);
            }
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = valid ? v[e] : 0.f;
            put4((T*)a.dx + at, v);
        }
    }
}

template <class T, int ACT> ds_status launch(const GluArgs& a, hipStream_t st) {
    const int N = ACT >= 0 ? a.ff : a.d, tiles_m = (a.rows + 63) / 64, tiles_n = (N + 63) / 64;
    hipLaunchKernelGGL((glu_general_kernel<T, ACT>), dim3((unsigned)tiles_m * tiles_n), dim3(256), 0, st, a, tiles_m, tiles_n);
    DS_LAUNCH_CHECK();
    return DS_OK;
}

}  // namespace

ds_status glu_fwd_general(const GluArgs& a, hipStream_t st) {
    return glu_by_act(a.act, [&](auto act) { return a.dtype == DS_DTYPE_BF16 ? launch<bf16_t, decltype(act)::value>(a, st) : launch<float, decltype(act)::value>(a, st); });
}
ds_status glu_dx_general(const GluArgs& a, hipStream_t st) { return a.dtype == DS_DTYPE_BF16 ? launch<bf16_t, -1>(a, st) : launch<float, -1>(a, st); }
