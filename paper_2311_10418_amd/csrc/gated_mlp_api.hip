// C-ABI entry points and dispatch of the gated feed-forward block.
#include "gated_mlp.hpp"
#include "gemm.hpp"
#include <algorithm>
#include <initializer_list>
#include <type_traits>

namespace {

// dG and dU, 8 elements to a thread.  They are outputs, which the weight gradients take, and dx is made of them as they are stored: in bf16 the matrix instructions would round them as they
// are multiplied all the same (error of dx against 64 bits, relative, 0.0023; rounded once from fp32 it would be 0.0017).  dg may be g, du may be u.  Bound by memory: three tensors read, two written
// (65 629 x 2816 in bf16: 309 us, 6.0 TB/s).
template <class T, int ACT>
__global__ __launch_bounds__(256) void glu_grad_kernel(long long n8, int ff8, const T* __restrict__ dh, const T* g, const T* u, const int32_t* __restrict__ row_valid, T* dg, T* du) {
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < n8; i += (long long)gridDim.x * 256) {
        float zg[8], zu[8], z[8], a[8], b[8];
        const bool valid = !row_valid || row_valid[(uint32_t)(i / ff8)] >= 0;
        Vec8<T>::load(dh + i * 8, z);
        Vec8<T>::load(g + i * 8, zg);
        Vec8<T>::load(u + i * 8, zu);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            float f, df;
            glu_act<ACT>(zg[j], f, df);
            a[j] = valid ? z[j] * zu[j] * df : 0.f;
            b[j] = valid ? z[j] * f : 0.f;
        }
        Vec8<T>::store(dg + i * 8, a);
        Vec8<T>::store(du + i * 8, b);
    }
}

template <class T> ds_status grad_launch(const GluArgs& a, const void* dh, const void* g, const void* u, void* dg, void* du, hipStream_t st) {
    return glu_by_act(a.act, [&](auto act) -> ds_status {
        const long long n8 = (long long)a.rows * a.ff / 8;
        const unsigned blocks = (unsigned)std::min<long long>((n8 + 255) / 256, 1 << 16);
        hipLaunchKernelGGL((glu_grad_kernel<T, decltype(act)::value>), dim3(blocks), dim3(256), 0, st, n8, a.ff / 8, (const T*)dh, (const T*)g, (const T*)u, a.row_valid, (T*)dg, (T*)du);
        DS_LAUNCH_CHECK();
        return DS_OK;
    });
}

constexpr int64_t kSumFloats = 128;                    // for each column: room for the biases' gradients
constexpr int kWide = 1 << 16, kRows = 0x7fffffff - (1 << 16);

ds_status check(int32_t dtype, int32_t rows, int32_t d, int32_t ff, std::initializer_list<const void*> needed, std::initializer_list<const void*> others, const float* workspace,
                int64_t workspace_floats) {
    if (dtype != DS_DTYPE_F32 && dtype != DS_DTYPE_BF16) return DS_EINVAL;
    if (rows < 0 || rows > kRows || d <= 0 || d % 8 || d > kWide || ff <= 0 || ff % 8 || ff > kWide) return DS_EINVAL;
    if (((int64_t)rows + 63) / 64 * ((std::max(d, ff) + 63) / 64) > 0x7fffffff / 256) return DS_EINVAL;       // (work-items of a launch)
    for (const void* p : needed)
        if ((!p && rows > 0) || ((uintptr_t)p & 15)) return DS_EINVAL;           // (a tensor without rows has no address)
    for (const void* p : others)
        if ((uintptr_t)p & 15) return DS_EINVAL;
    if (workspace_floats < 0 || (workspace_floats > 0 && (!workspace || ((uintptr_t)workspace & 15)))) return DS_EINVAL;
    return DS_OK;
}
// Estimated microseconds of the 128 x 128 tiles: two work-groups to a compute unit, which share it; per K tile 0.93 for two, 0.55 for one alone.  Measured (warm, d x d_ff,
// rows: estimate / measured), forward: 1024 x 2816, 512 14 / 14, 957 20 / 18, 1500 30 / 29, 4096 52 / 49, 8192 94 / 88; 2048 x 5504, 700 53 / 50, 8192 343 / 339; 256 x 1024,
// 8192 14 / 16.
double tile_cost(int64_t groups, int steps) {
    const int64_t full = groups / 512, rest = groups % 512;
    return 4 + full * (0.93 * steps + 1.2) + (rest == 0 ? 0 : rest <= 256 ? 0.55 * steps + 1.2 : 0.9 * steps + 1.2);
}
// How a product goes: 256 x 256 tiles, or 128 x 128 with the contraction of dx in `splits` pieces.  Both sides by their estimates (that of the large tiles: gemm.hip);
// measured, large / small: forward 1024 x 2816, 957 rows 33 / 18 us, 4096 61 / 49, 16 384 180 / 187, 40 000 408 / 459; 2048 x 5504, 512 44 / 31, 957 47 / 51, 8192 288 / 339.
struct GluChoice { bool big; int splits; };
GluChoice choose(const GluArgs& a, bool dx, size_t ws_floats) {
    GluChoice c = {false, 1};
    const int64_t groups = (int64_t)((a.rows + 127) / 128) * (dx ? (a.d + 127) / 128 : (a.ff + 63) / 64);
    const int steps = dx ? 2 * ((a.ff + 63) / 64) : (a.d + 63) / 64;
    double cost = tile_cost(groups, steps);
    if (dx)
        for (int s = 2; s <= 16 && groups * s <= 512 && steps / s >= 4 && (size_t)s * a.rows * a.d <= ws_floats; ++s) {
            const double split = tile_cost(groups * s, (steps + s - 1) / s) + 4 + 1e-6 * s * a.rows * a.d;
            if (split < 0.95 * cost) cost = split, c.splits = s;
        }
    if (a.d % 64 || a.ff % 64 || (dx && a.d % 256)) return c;
    const int columns = dx ? a.d : (a.ff + 127) / 128 * 256, K = dx ? 2 * a.ff : a.d;
    c.big = glu_big_cost(a.rows, columns, K, ws_floats) < cost;
    return c;
}
// fp32: bf16 parts where the contraction is long enough to pay for their prologue.  us, fp32 products / bf16 parts: forward d = 128, 4 096 rows 15 / 14, 957 rows 9 / 11; 192 x 768, 2 048 rows
// 20 / 17; 256 x 1024, 7 684 rows 84 / 71, 128 rows 15 / 13; 1024 x 2816, 957 rows 118 / 94, 7 684 rows 778 / 628; backward 128 x 512, 957 rows 35 / 26; 256 x 1024, 957 rows 65 / 40;
// 1024 x 2816, 128 rows 155 / 46, 7 684 rows 867 / 737.
bool split_f32(const GluArgs& a, bool dx) { return (dx || a.d >= 192) && glu_f32_supported(a); }
// Shares of the rows of the weight gradients' 128 x 128 tiles, by an estimate: two work-groups to a compute unit 1.05 us per 64 rows, one alone 0.7, and the launch that adds shares up.
// Measured, us, with 1 / 2 / 3 / 4 shares (chosen: *): d x d_ff x rows 1856 x 960 x 1418 *23 / 28 / 35 / 41; 832 x 384 x 784 *11 / 12 / 13 / 14; 1000 x 1000 x 2000 26 / *23 / 24 / 25, 20 000 215 / 125 / 113 /
// *93; 512 x 4416 x 49 573 643 / 694 / *522, 5 000 *65 / 72 / 66; 128 x 192 x 65 536 591 / 301 / 204 / 152, with 32 / 64 /
// 128 31 / *27 / 31.
int wgrad_splits(int rows, int d, int ff, int64_t ws_floats) {
    const int64_t tiles = (int64_t)((d + 127) / 128) * ((ff + 127) / 128) * 2, outputs = 2 * (int64_t)d * ff, steps = ((int64_t)rows + 63) / 64;
    int best = 1;
    double least = 0;
    for (int s = 1; s <= 128 && s <= steps && (s == 1 || s * outputs <= ws_floats); ++s) {
        const int64_t full = tiles * s / 512, rest = tiles * s % 512;
        const double rounds = 1.05 * full + (rest == 0 ? 0 : rest <= 256 ? 0.7 : 0.7 + 0.35 * (rest - 256) / 256);
        const double cost = rounds * ((steps + s - 1) / s) + (s > 1 ? 4 + 0.03 * s + 1e-6 * (s + 1) * outputs : 0);
        if (s == 1 || cost < least) least = cost, best = s;
    }
    return best;
}
bool known_act(int32_t act) { return act == DS_ACT_GELU || act == DS_ACT_SILU || act == DS_ACT_RELU; }

}  // namespace

extern "C" int64_t ds_gated_mlp_workspace_floats(int32_t rows, int32_t d, int32_t d_ff) {
    if (rows <= 0 || d <= 0 || d_ff <= 0) return 0;
    return std::max((int64_t)1 << 24, kSumFloats * d_ff);
}

// For tests: what `choose` says of a bf16 call with more than kGluFewRows rows: 256 x 256 tiles, pieces of the contraction; dx = 2: shares of the weight gradients' tiles.  Not part of
// the C ABI's header.
extern "C" void ds_gated_mlp_choice(int32_t rows, int32_t d, int32_t d_ff, int32_t dx, int64_t workspace_floats, int32_t* out) {
    GluArgs a = {};
    a.rows = rows; a.d = d; a.ff = d_ff;
    const GluChoice c = dx == 2 ? GluChoice{false, wgrad_splits(rows, d, d_ff, workspace_floats)} : choose(a, dx != 0, (size_t)workspace_floats);
    out[0] = c.big;
    out[1] = c.splits;
}

// For tests: `choose`'s first member, then (of the 256 x 256 tiles, taken or not) glu_big_division.  Not part of the C ABI's header.
extern "C" void ds_gated_mlp_division(int32_t rows, int32_t d, int32_t d_ff, int32_t dx, int64_t workspace_floats, int32_t* out) {
    GluArgs a = {};
    a.rows = rows; a.d = d; a.ff = d_ff;
    out[0] = choose(a, dx != 0, (size_t)workspace_floats).big;
    glu_big_division(a, dx != 0, (size_t)workspace_floats, out + 1);
}

// For tests: columns of a tile of dx in fp32, 0: two products, -1: fp32 matrix instructions.  Not part of the C ABI's header.
extern "C" int32_t ds_gated_mlp_f32_columns(int32_t rows, int32_t d, int32_t d_ff) {
    GluArgs a = {};
    a.dtype = DS_DTYPE_F32; a.rows = rows; a.d = d; a.ff = d_ff;
    return split_f32(a, true) ? glu_dx_f32_columns(a) : -1;
}

extern "C" ds_status ds_gated_mlp_fwd(int32_t dtype, int32_t act, int32_t rows, int32_t d, int32_t d_ff, const void* x, const void* wg, const void* wu, const void* bg,
                                      const void* bu, const int32_t* row_valid, void* h, void* g, void* u, float* workspace, int64_t workspace_floats,
                                      int32_t force_generic, void* hip_stream) {
    const ds_status r = check(dtype, rows, d, d_ff, {x, wg, wu, h}, {bg, bu, g, u}, workspace, workspace_floats);
    if (r != DS_OK) return r;
    if (!known_act(act) || !g != !u) return DS_EINVAL;
    if (rows == 0) return DS_OK;
    GluArgs a = {};
    a.dtype = dtype; a.act = act; a.rows = rows; a.d = d; a.ff = d_ff;
    a.x = x; a.wg = wg; a.wu = wu; a.bg = bg; a.bu = bu; a.row_valid = row_valid; a.h = h; a.g = g; a.u = u;
    if (force_generic) return glu_fwd_general(a, (hipStream_t)hip_stream);
    if (rows <= kGluFewRows) return glu_fwd_few(a, (hipStream_t)hip_stream);
    if (dtype == DS_DTYPE_F32) return split_f32(a, false) ? glu_fwd_f32(a, (hipStream_t)hip_stream) : glu_fwd_general(a, (hipStream_t)hip_stream);
    const size_t floats = workspace_floats > 0 ? (size_t)workspace_floats : 0;
    if (choose(a, false, floats).big) return glu_fwd_big(a, workspace, floats, (hipStream_t)hip_stream);
    return glu_fwd_tile(a, (hipStream_t)hip_stream);
}

extern "C" ds_status ds_gated_mlp_bwd(int32_t dtype, int32_t act, int32_t rows, int32_t d, int32_t d_ff, const void* dh, const void* g, const void* u, const void* wg,
                                      const void* wu, const int32_t* row_valid, void* dg, void* du, void* dx, float* workspace, int64_t workspace_floats,
                                      int32_t force_generic, void* hip_stream) {
    ds_status r = check(dtype, rows, d, d_ff, {dh, g, u, wg, wu, dg, du, dx}, {}, workspace, workspace_floats);
    if (r != DS_OK) return r;
    if (!known_act(act)) return DS_EINVAL;
    if (rows == 0) return DS_OK;
    hipStream_t st = (hipStream_t)hip_stream;
    GluArgs a = {};
    a.dtype = dtype; a.act = act; a.rows = rows; a.d = d; a.ff = d_ff;
    a.wg = wg; a.wu = wu; a.row_valid = row_valid; a.dg = dg; a.du = du; a.dx = dx;
    r = dtype == DS_DTYPE_BF16 ? grad_launch<bf16_t>(a, dh, g, u, dg, du, st) : grad_launch<float>(a, dh, g, u, dg, du, st);
    if (r != DS_OK) return r;
    const size_t floats = workspace_floats > 0 ? (size_t)workspace_floats : 0;
    if (force_generic || (dtype == DS_DTYPE_F32 && !split_f32(a, true))) return glu_dx_general(a, st);
    if (dtype == DS_DTYPE_F32) return glu_dx_f32(a, floats ? workspace : nullptr, floats, st);
    const GluChoice c = choose(a, true, floats);
    return c.big ? glu_dx_big(a, workspace, floats, st) : glu_dx_tile(a, c.splits, workspace, st);
}

extern "C" ds_status ds_gated_mlp_wgrad(int32_t dtype, int32_t rows, int32_t d, int32_t d_ff, const void* x, const void* dg, const void* du, float* dwg, float* dwu, float* dbg,
                                        float* dbu, int32_t accumulate, float* workspace, int64_t workspace_floats, int32_t force_generic, void* hip_stream) {
    ds_status r = check(dtype, rows, d, d_ff, {x, dg, du, dwg, dwu}, {dbg, dbu}, workspace, workspace_floats);
    if (r != DS_OK) return r;
    if (rows == 0 || (accumulate != 0 && accumulate != 1) || !dbg != !dbu) return DS_EINVAL;
    if (dbg && workspace_floats < kSumFloats * d_ff) return DS_EINVAL;
    hipStream_t st = (hipStream_t)hip_stream;
    TnGroup group;
    group.n = 2; group.K = rows; group.accumulate = accumulate; group.f32 = dtype == DS_DTYPE_F32;
    group.p[0] = TnProblem{x, dg, dwg, d, d_ff};
    group.p[1] = TnProblem{x, du, dwu, d, d_ff};
    for (int i = 0; i < TnGroup::kSlabs; ++i) {
        group.slab[i] = workspace;
        group.slab_end[i] = (int32_t)std::min<int64_t>(workspace_floats >> group.block_log2(), INT32_MAX);
    }
    TnPick pick{-1, 1};
    if (!force_generic && tn_group_takes(group.p[0], rows, group.f32)) pick = pick_tn_group(group);
    if (pick.kind >= 0) {
        r = launch_tn_group(pick, group, st);
        if (r != DS_OK) return r;
    } else if (dtype == DS_DTYPE_BF16 && !force_generic && !tn_group_takes(group.p[0], rows, false)) {
        // sizes that the products' own kernels do not take
        GluWgrad w = {rows, d, d_ff, accumulate, 1, x, {dg, du}, {dwg, dwu}, workspace};
        w.splits = wgrad_splits(rows, d, d_ff, workspace_floats);
        r = glu_wgrad_tile(w, st);
        if (r != DS_OK) return r;
    } else {
        for (int i = 0; i < 2; ++i) {
            GemmEpi p{};
            p.accumulate = accumulate;
            r = launch_gemm(dtype, 1, 0, d, d_ff, rows, x, i ? du : dg, i ? dwu : dwg, DS_EPI_ACC32, p, force_generic != 0, workspace_floats > 0 ? workspace : nullptr,
                            (size_t)workspace_floats, st);
            if (r != DS_OK) return r;
        }
    }
    if (!dbg) return DS_OK;
    SumGroup sums;                                      // (behind the products in the stream: the workspace is free again)
    sums.n = 2; sums.accumulate = accumulate;
    sums.it[0] = SumItem{dg, dbg, rows, d_ff, d_ff, 1};
    sums.it[1] = SumItem{du, dbu, rows, d_ff, d_ff, 1};
    int launched = 0;
    return launch_sum_group(dtype, sums, workspace, (size_t)workspace_floats, st, &launched);
}
