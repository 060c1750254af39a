// Arguments shared by the kernels of the gated feed-forward block.
//
// Forward, weights [d_ff][d]:   G = x Wg^T + bg,  U = x Wu^T + bu,  H = act(G) U.
// Backward, weights [d][d_ff]:  dG = dH U act'(G),  dU = dH act(G),  dx = dG Wg^T + dU Wu^T: one contraction over 2 d_ff.
// Weight gradients:             dWg = x^T dG,  dWu = x^T dU  ([d][d_ff]), dbg and dbu the column sums of dG and dU.
#pragma once
#include "common.hpp"
#include <type_traits>

struct GluArgs {
    int32_t dtype, act, rows, d, ff;
    const void *x, *wg, *wu, *bg, *bu;
    const int32_t* row_valid;                           // NULL, or [rows]: a negative entry makes a row of zeros
    void *h, *g, *u;                                    // g, u: both or neither
    const void *dg, *du;                                // backward: the operands of dx
    void* dx;
    int32_t splits;                                     // dx: pieces of the contraction, and where their sums go
    float* part;
};

// The activation of z and its derivative.  DS_ACT_RELU's at 0 is 0.
template <int ACT> __device__ __forceinline__ void glu_act(float z, float& f, float& df) {
    if constexpr (ACT == DS_ACT_GELU) {
        gelu_and_grad_f(z > 30.f ? 30.f : z < -30.f ? -30.f : z, f, df);       // (beyond, the logistic term is 1 or 0, and z * z may overflow; NaN stays)
        f = z > 30.f ? z : f;
    } else if constexpr (ACT == DS_ACT_SILU) {
        const float s = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.4426950408889634f * z));
        f = z * s;
        df = s * __builtin_fmaf(z, 1.0f - s, 1.0f);
    } else {
        f = z < 0.f ? 0.f : z;                          // (NaN stays)
        df = z > 0.f ? 1.f : z <= 0.f ? 0.f : z;
    }
}
template <int ACT> __device__ __forceinline__ float glu_act(float z) {
    if constexpr (ACT == DS_ACT_GELU) return gelu_f(z);
    float f, df;
    glu_act<ACT>(z, f, df);
    return f;
}
template <class F> ds_status glu_by_act(int act, F&& f) {
    if (act == DS_ACT_GELU) return f(std::integral_constant<int, DS_ACT_GELU>{});
    if (act == DS_ACT_SILU) return f(std::integral_constant<int, DS_ACT_SILU>{});
    return f(std::integral_constant<int, DS_ACT_RELU>{});
}

ds_status glu_fwd_general(const GluArgs& a, hipStream_t st);
ds_status glu_dx_general(const GluArgs& a, hipStream_t st);
// bf16 on the matrix cores (gated_mlp_mfma.hip), any size: 128 x 128 tiles; few rows; weight gradients with 2 splits [d][d_ff] floats of workspace if splits > 1
ds_status glu_fwd_tile(const GluArgs& a, hipStream_t st);
ds_status glu_dx_tile(const GluArgs& a, int splits, float* workspace, hipStream_t st);      // splits > 1: as many [rows][d] floats of workspace
constexpr int kGluFewRows = 64;
ds_status glu_fwd_few(const GluArgs& a, hipStream_t st);
struct GluWgrad {
    int32_t rows, d, ff, accumulate, splits;
    const void *x, *dy[2];
    float *dw[2], *workspace;
};
ds_status glu_wgrad_tile(const GluWgrad& a, hipStream_t st);
// fp32 as eight bf16 products of its parts (gemm_f32.hip); dx of few rows as two products
bool glu_f32_supported(const GluArgs& a);
ds_status glu_fwd_f32(const GluArgs& a, hipStream_t st);
ds_status glu_dx_f32(const GluArgs& a, float* ws, size_t ws_floats, hipStream_t st);
int glu_dx_f32_columns(const GluArgs& a);              // columns of a tile of dx; 0: two products instead
// the same with 256 x 256 tiles (gemm.hip): d and d_ff multiples of 64, dx: d of 256; and the estimate of their time in microseconds, of `columns` (a multiple of 256)
// weight rows and a contraction over K
ds_status glu_fwd_big(const GluArgs& a, float* ws, size_t ws_floats, hipStream_t st);
ds_status glu_dx_big(const GluArgs& a, float* ws, size_t ws_floats, hipStream_t st);
double glu_big_cost(int M, int columns, int K, size_t ws_floats);
// how such a product divides its tiles: whole ones, those whose contraction is cut up, pieces of it, whether work-groups are persistent
void glu_big_division(const GluArgs& a, bool dx, size_t ws_floats, int32_t* out);
