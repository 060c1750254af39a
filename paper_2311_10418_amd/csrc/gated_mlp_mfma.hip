// The gated feed-forward block's products in bf16 on the matrix cores (v_mfma_f32_16x16x32_bf16), for every size: what has the 256 x 256 kernel's sizes and
// enough rows goes there (gemm.hip), the rest comes here.
//
// Tiles (glu_tile_kernel, glu_wgrad_kernel): 128 x 128, K tiles of 64, four wavefronts in a 2 x 2 arrangement with 64 x 64 outputs each, two work-groups to a
// compute unit.  Operands go global -> LDS directly through raw buffers: what lies behind the last row or, in a ragged last K tile, behind the end of a row (a
// lane offset beyond every length) arrives as zeros.  Two stages, the next K tile in flight while one is multiplied.  LDS rows are swizzled by 16-byte chunks
// (weight gradients: by 32 bytes) as in gemm.hip, by choosing which global chunk a lane fetches.
//
// Forward, the two weight matrices share a tile: of the 64 weight rows that a wavefront multiplies 32 are Wg's and 32 Wu's for the same 32 columns of H, so that
// both pre-activations of an output are in the same lane and register position, and the activation is one pass over registers.  dx: the K loop runs through
// (dG, Wg) and then through (dU, Wu) into the same accumulators.
//
// Bound by the latency of a K tile's transfers and reads, which two work-groups to a compute unit hide in part: 957 rows, 1024 x 2816, forward 18.5 us (597 TFLOP/s), where the grid
// is 352 work-groups for 512 places; 4 096 rows 49 us (960 TFLOP/s).
#include "gated_mlp.hpp"
#include "gemm_epilogue.hpp"
#include <algorithm>
#include <type_traits>

namespace {

constexpr int TK = 64, TILE = 128 * TK * 2, STAGE = 2 * TILE;      // bytes of an operand's K tile, of both
constexpr uint32_t kBeyond = 0x80000000u;

__device__ __forceinline__ f32x4_t mfma(const bf16x8_t& a, const bf16x8_t& b, const f32x4_t& c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4_t zero4() { return f32x4_t{0.f, 0.f, 0.f, 0.f}; }
__device__ __forceinline__ void put4(bf16_t* p, const f32x4_t& v) {
    bf16x4_t x;
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = (bf16_t)v[e];
    *reinterpret_cast<bf16x4_t*>(p) = x;
}
__device__ __forceinline__ f32x4_t get4(const bf16_t* p) {
    const bf16x4_t x = *reinterpret_cast<const bf16x4_t*>(p);
    return f32x4_t{(float)x[0], (float)x[1], (float)x[2], (float)x[3]};
}
// this wavefront's transfers have landed, then everybody's; the stage read in the previous step is free
__device__ __forceinline__ void wait_and_sync() {
    __builtin_amdgcn_s_waitcnt(0x0070);             // vmcnt(0) lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
}

// 32 rows (row-major, ld elements) x 64 k of a wavefront's part of an operand: four transfers of 8 rows
struct RowLoader {
    const char* base;                               // first row, k = 0
    uint32_t bytes;                                 // of the rows that exist, from there
    uint32_t off[4], beyond[2];
    __device__ __forceinline__ void setup(const void* src, long long ld, int r0, int rows, int K, int lane) {
        base = reinterpret_cast<const char*>(src) + (long long)r0 * ld * 2;
        const int left = min(max(rows - r0, 0), 32);
        bytes = left ? (uint32_t)((left - 1) * (uint32_t)ld + K) * 2u : 0u;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int row = i * 8 + (lane >> 3), chunk = (lane & 7) ^ ((row >> 1) & 7);
            off[i] = dma_lane_offset<4>((uint32_t)row * (uint32_t)ld * 2u + chunk * 16, i);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) beyond[i] = ((lane & 7) ^ ((i * 4 + (lane >> 4)) & 7)) * 8 >= (K & (TK - 1)) ? kBeyond : 0u;
    }
    // k0: a multiple of 64 below K
    __device__ __forceinline__ void issue(uint32_t lds, int k0, int K) const {
        const uint32_t skip = (uint32_t)k0 * 2u;
        const i32x4_t buf = make_raw_buffer(base + skip - 3 * 1024, bytes ? bytes - skip + 3 * 1024u : 0u);
        if (k0 + TK <= K) {
            lds_dma16_buffer_group<4>(buf, off, lds);
        } else {
            uint32_t o[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) o[i] = off[i] + beyond[i & 1];
            lds_dma16_buffer_group<4>(buf, o, lds);
        }
    }
};

// ACT: an activation, or -1: dx
template <int ACT> __global__ __launch_bounds__(256, 2) void glu_tile_kernel(GluArgs a, int tiles_m, int tiles_n) {
    constexpr bool FWD = ACT >= 0;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave >> 1, wn = wave & 1;
    const int fr = lane & 15, fg = lane >> 4;
    // groups of 8 tile rows, column by column inside a group
    const int logical = xcd_contiguous(blockIdx.x, gridDim.x), group = logical / (8 * tiles_n), in = logical - group * 8 * tiles_n, deep = min(8, tiles_m - 8 * group);
    const int m0 = __builtin_amdgcn_readfirstlane((8 * group + in % deep) * 128), n0 = __builtin_amdgcn_readfirstlane(in / deep * (FWD ? 64 : 128));
    const int K = FWD ? a.d : a.ff, N = FWD ? a.ff : a.d, steps = (K + TK - 1) / TK, all = FWD ? steps : 2 * steps;
    // dx: this work-group's piece of the contraction
    const int per = FWD ? all : (all + a.splits - 1) / a.splits, begin = FWD ? 0 : min((int)blockIdx.y * per, all), end = FWD ? all : min(begin + per, all);
    const uint32_t lds0 = lds_address(smem);
    RowLoader la[FWD ? 1 : 2], lb[FWD ? 1 : 2];
    if constexpr (FWD) {
        la[0].setup(a.x, K, m0 + wave * 32, a.rows, K, lane);
        lb[0].setup(wave & 1 ? a.wu : a.wg, K, n0 + (wave >> 1) * 32, N, K, lane);
    } else {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            la[i].setup(i ? a.du : a.dg, K, m0 + wave * 32, a.rows, K, lane);
            lb[i].setup(i ? a.wu : a.wg, K, n0 + wave * 32, N, K, lane);
        }
    }
    auto issue = [&](int step) {
        const uint32_t to = lds0 + (step & 1) * STAGE + wave * 4096;
        if (FWD || step < steps) {
            la[0].issue(to, step * TK, K);
            lb[0].issue(to + TILE, step * TK, K);
        } else {
            la[FWD ? 0 : 1].issue(to, (step - steps) * TK, K);
            lb[FWD ? 0 : 1].issue(to + TILE, (step - steps) * TK, K);
        }
    };
    f32x4_t acc[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = zero4();
    const int at[2] = {fr * 128 + ((fg ^ ((fr >> 1) & 7)) << 4), fr * 128 + (((4 + fg) ^ ((fr >> 1) & 7)) << 4)};
    if (begin < end) issue(begin);
    for (int step = begin; step < end; ++step) {
        wait_and_sync();
        if (step + 1 < end) issue(step + 1);
        const char *ta = smem + (step & 1) * STAGE + wm * 8192, *tb = smem + (step & 1) * STAGE + TILE + wn * 8192;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            bf16x8_t fa[4], fb[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                fb[i] = *reinterpret_cast<const bf16x8_t*>(tb + i * 2048 + at[s]);
                fa[i] = *reinterpret_cast<const bf16x8_t*>(ta + i * 2048 + at[s]);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = mfma(fb[j], fa[i], acc[i][j]);       // the transposed block: 4 consecutive columns to a lane
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int m = m0 + wm * 64 + i * 16 + fr;
        if (m >= a.rows) continue;
        const bool valid = !a.row_valid || a.row_valid[m] >= 0;
#pragma unroll
        for (int j = 0; j < (FWD ? 2 : 4); ++j) {
            const int n = n0 + wn * (FWD ? 32 : 64) + j * 16 + fg * 4;
            if (n >= N) continue;
            const size_t to = (size_t)m * N + n;
            f32x4_t v = acc[i][j];
            if constexpr (FWD) {
                f32x4_t u = acc[i][j + 2], h;
                if (a.bg) v += get4((const bf16_t*)a.bg + n);
                if (a.bu) u += get4((const bf16_t*)a.bu + n);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    v[e] = valid ? v[e] : 0.f;
                    u[e] = valid ? u[e] : 0.f;
                    h[e] = valid ? glu_act<ACT>(v[e]) * u[e] : 0.f;
                }
                put4((bf16_t*)a.h + to, h);
                if (a.g) {
                    put4((bf16_t*)a.g + to, v);
                    put4((bf16_t*)a.u + to, u);
                }
            } else if (a.splits > 1) {
                *reinterpret_cast<f32x4_t*>(a.part + (size_t)blockIdx.y * a.rows * a.d + to) = v;
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = valid ? v[e] : 0.f;
                put4((bf16_t*)a.dx + to, v);
            }
        }
    }
}

// ---------------------------------------------------------------- weight gradients: dW[d][ff] = x^T dY, blockIdx.z 0: dG, 1: dU; blockIdx.y: a share of the rows
// 64 rows x 128 columns of a row-major operand, rows past the end as zeros (columns past the end are whatever follows: their products are not stored)
struct ColumnLoader {
    const char* base;
    long long ld2;
    uint32_t off[4];
    int cols_left2;                                 // bytes of a row from the tile's first column on
    __device__ __forceinline__ void setup(const void* src, int ld, int c0, int wave, int lane) {
        base = reinterpret_cast<const char*>(src) + (long long)c0 * 2;
        ld2 = (long long)ld * 2;
        cols_left2 = (ld - c0) * 2;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int row = (wave * 4 + i) * 4 + (lane >> 4), pos = lane & 15, chunk = (((pos >> 1) ^ (row & 7)) << 1) | (pos & 1);
            off[i] = dma_lane_offset<4>((uint32_t)row * (uint32_t)ld2 + chunk * 16, i);
        }
    }
    // rows k0 .. k0 + 63 of those below k_end (k0 < k_end)
    __device__ __forceinline__ void issue(uint32_t lds, int k0, int k_end) const {
        const uint32_t bytes = (uint32_t)(min(TK, k_end - k0) - 1) * (uint32_t)ld2 + (uint32_t)cols_left2;
        lds_dma16_buffer_group<4>(make_raw_buffer(base + (long long)k0 * ld2 - 3 * 1024, bytes + 3 * 1024u), off, lds);
    }
};

__global__ __launch_bounds__(256, 2) void glu_wgrad_kernel(GluWgrad a, int tiles_m, int tiles_n) {
    extern __shared__ __attribute__((aligned(16))) char smem[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave >> 1, wn = wave & 1;
    const int fr = lane & 15, fg = lane >> 4;
    const int logical = xcd_contiguous(blockIdx.x, gridDim.x), which = blockIdx.z, split = blockIdx.y;
    const int m0 = __builtin_amdgcn_readfirstlane(logical % tiles_m * 128), n0 = __builtin_amdgcn_readfirstlane(logical / tiles_m * 128);
    const int steps = (a.rows + TK - 1) / TK, per = (steps + a.splits - 1) / a.splits;
    const int k_begin = min(split * per * TK, a.rows), k_end = min(k_begin + per * TK, a.rows);
    const uint32_t lds0 = lds_address(smem);
    ColumnLoader la, lb;
    la.setup(a.x, a.d, m0, wave, lane);
    lb.setup(a.dy[which], a.ff, n0, wave, lane);
    auto issue = [&](int k0, int turn) {
        const uint32_t to = lds0 + turn * STAGE + wave * 4096;
        la.issue(to, k0, k_end);
        lb.issue(to + TILE, k0, k_end);
    };
    f32x4_t acc[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = zero4();
    // a fragment (16 columns x 32 rows) is two transpose reads of 16 rows x 32 bytes: lane (i = lane % 16, g = lane / 16) addresses row 4 g + i / 4 and receives
    // column i at rows 4 g .. 4 g + 3
    typedef short s16x4_t __attribute__((ext_vector_type(4)));
    typedef short s16x8_t __attribute__((ext_vector_type(8)));
    typedef __attribute__((address_space(3))) s16x4_t* lds4_t;
    const int tr_row = 4 * fg + (fr >> 2), tr_lane = tr_row * 256 + (lane & 3) * 8;
    auto fragment = [&](const char* tile, int unit, int s) {
        const char* q = tile + tr_lane + ((unit ^ (tr_row & 7)) << 5) + s * (32 * 256);
        const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4_t)q), hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4_t)(q + 16 * 256));
        const s16x8_t v = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        return __builtin_bit_cast(bf16x8_t, v);
    };
    if (k_begin < k_end) issue(k_begin, 0);
    int turn = 0;
    for (int k0 = k_begin; k0 < k_end; k0 += TK, turn ^= 1) {
        wait_and_sync();
        if (k0 + TK < k_end) issue(k0 + TK, turn ^ 1);
        const char *ta = smem + turn * STAGE, *tb = ta + TILE;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            bf16x8_t fa[4], fb[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                fb[i] = fragment(tb, wn * 4 + i, s);
                fa[i] = fragment(ta, wm * 4 + i, s);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = mfma(fb[j], fa[i], acc[i][j]);
        }
    }
    float* out = a.splits > 1 ? a.workspace + (size_t)(which * a.splits + split) * a.d * a.ff : a.dw[which];
    const bool add = a.splits == 1 && a.accumulate;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int m = m0 + wm * 64 + i * 16 + fr;
        if (m >= a.d) continue;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int n = n0 + wn * 64 + j * 16 + fg * 4;
            if (n >= a.ff) continue;
            f32x4_t* to = reinterpret_cast<f32x4_t*>(out + (size_t)m * a.ff + n);
            *to = add ? *to + acc[i][j] : acc[i][j];
        }
    }
}

// the shares' sums, in their order; four values to a thread, eight loads in flight
__global__ __launch_bounds__(256) void glu_wgrad_finish_kernel(GluWgrad a, long long n4) {
    const f32x4_t* from = reinterpret_cast<const f32x4_t*>(a.workspace) + (size_t)blockIdx.y * a.splits * n4;
    f32x4_t* to = reinterpret_cast<f32x4_t*>(a.dw[blockIdx.y]);
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < n4; i += (long long)gridDim.x * 256) {
        f32x4_t sum = from[i];
        int s = 1;
        for (; s + 8 <= a.splits; s += 8) {
            f32x4_t v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = from[(size_t)(s + j) * n4 + i];
#pragma unroll
            for (int j = 0; j < 8; ++j) sum += v[j];
        }
        for (; s < a.splits; ++s) sum += from[(size_t)s * n4 + i];
        to[i] = a.accumulate ? to[i] + sum : sum;
    }
}

// ---------------------------------------------------------------- few rows
// The weights are what is read, once: a work-group takes 8 columns of H, its four wavefronts a quarter of K each, operands straight from memory into fragments.
// The 16 weight rows of a block are 8 of Wg and the same 8 of Wu; the wavefronts' sums and the two halves meet in LDS.  RB blocks of 16 rows of x.
// Bound by memory: 16 rows, 1024 x 2816, bf16, weights of 11.5 MB in 6.2 us (1.9 TB/s; about 4 of them are the start, first trip and end of any kernel).
// A lane's piece of a row is 16 bytes: bf16 one instruction of 16x16x32 for 4 lanes' pieces, fp32 four of 16x16x4.
template <class T> struct FewPiece;
template <> struct FewPiece<bf16_t> {
    typedef bf16x8_t type;
    static __device__ __forceinline__ f32x4_t product(const type& w, const type& x, const f32x4_t& c) { return mfma(w, x, c); }
};
template <> struct FewPiece<float> {
    typedef f32x4_t type;
    static __device__ __forceinline__ f32x4_t product(const type& w, const type& x, f32x4_t c) {
#pragma unroll
        for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(w[e], x[e], c, 0, 0, 0);
        return c;
    }
};
template <class T, int ACT, int RB> __global__ __launch_bounds__(256) void glu_few_kernel(GluArgs a) {
    typedef FewPiece<T> P;
    typedef typename P::type piece_t;
    constexpr int AHEAD = RB == 1 ? 8 : 4, N = 16 / sizeof(T), DEPTH = 4 * N;
    __shared__ __attribute__((aligned(16))) float part[4][RB * 16][16];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), fr = lane & 15, fg = lane >> 4, n0 = blockIdx.x * 8, K = a.d;
    const int steps = (K + DEPTH - 1) / DEPTH, per = (steps + 3) / 4, s_end = min(steps, (wave + 1) * per);
    const T* w = (const T*)(fr < 8 ? a.wg : a.wu) + (size_t)(n0 + (fr & 7)) * K;
    const T* x[RB];
#pragma unroll
    for (int b = 0; b < RB; ++b) x[b] = (const T*)a.x + (size_t)min(b * 16 + fr, a.rows - 1) * K;
    const piece_t none = {};
    f32x4_t acc[RB];
#pragma unroll
    for (int b = 0; b < RB; ++b) acc[b] = zero4();
    for (int s0 = wave * per; s0 < s_end; s0 += AHEAD) {
        piece_t fw[AHEAD], fx[AHEAD][RB];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const int k = (s0 + i) * DEPTH + fg * N;
            const bool in = s0 + i < s_end && k < K;       // (K is a multiple of 8)
            fw[i] = in ? *reinterpret_cast<const piece_t*>(w + k) : none;
#pragma unroll
            for (int b = 0; b < RB; ++b) fx[i][b] = in ? *reinterpret_cast<const piece_t*>(x[b] + k) : none;
        }
#pragma unroll
        for (int i = 0; i < AHEAD; ++i)
#pragma unroll
            for (int b = 0; b < RB; ++b) acc[b] = P::product(fw[i], fx[i][b], acc[b]);
    }
#pragma unroll
    for (int b = 0; b < RB; ++b) *reinterpret_cast<f32x4_t*>(&part[wave][b * 16 + fr][4 * fg]) = acc[b];
    __syncthreads();
    for (int o = threadIdx.x; o < RB * 16 * 8; o += 256) {
        const int m = o >> 3, c = o & 7, n = n0 + c;
        if (m >= a.rows) break;
        float g = (part[0][m][c] + part[1][m][c]) + (part[2][m][c] + part[3][m][c]);
        float u = (part[0][m][c + 8] + part[1][m][c + 8]) + (part[2][m][c + 8] + part[3][m][c + 8]);
        if (a.bg) g += to_f32(((const T*)a.bg)[n]);
        if (a.bu) u += to_f32(((const T*)a.bu)[n]);
        const bool valid = !a.row_valid || a.row_valid[m] >= 0;
        const size_t to = (size_t)m * a.ff + n;
        ((T*)a.h)[to] = from_f32<T>(valid ? glu_act<ACT>(g) * u : 0.f);
        if (a.g) {
            ((T*)a.g)[to] = from_f32<T>(valid ? g : 0.f);
            ((T*)a.u)[to] = from_f32<T>(valid ? u : 0.f);
        }
    }
}

template <int ACT> ds_status tile_launch(const GluArgs& a, hipStream_t st) {
    static std::atomic<uint64_t> allowed{0};
    auto kern = glu_tile_kernel<ACT>;
    const ds_status r = allow_dynamic_lds(kern, 2 * STAGE, allowed);
    if (r != DS_OK) return r;
    const int tiles_m = (a.rows + 127) / 128, tiles_n = ACT >= 0 ? (a.ff + 63) / 64 : (a.d + 127) / 128;
    hipLaunchKernelGGL(kern, dim3((unsigned)tiles_m * tiles_n, ACT >= 0 ? 1 : a.splits), dim3(256), 2 * STAGE, st, a, tiles_m, tiles_n);
    DS_LAUNCH_CHECK();
    return DS_OK;
}

}  // namespace

ds_status glu_fwd_tile(const GluArgs& a, hipStream_t st) {
    return glu_by_act(a.act, [&](auto act) { return tile_launch<decltype(act)::value>(a, st); });
}
ds_status glu_dx_tile(const GluArgs& a0, int splits, float* workspace, hipStream_t st) {
    GluArgs a = a0;
    a.splits = splits;
    a.part = workspace;
    const ds_status r = tile_launch<-1>(a, st);
    if (r != DS_OK || splits == 1) return r;
    GemmEpi p{};                                        // (rows that do not count are zeros in dG and dU, and so in dx)
    return launch_splitk_finish<bf16_t, DS_EPI_NONE>(a.rows, a.d, splits, workspace, a.dx, p, st);
}

template <class T> static ds_status few_launch(const GluArgs& a, hipStream_t st) {
    return glu_by_act(a.act, [&](auto act) -> ds_status {
        constexpr int ACT = decltype(act)::value;
        auto kern = a.rows <= 16 ? glu_few_kernel<T, ACT, 1> : a.rows <= 32 ? glu_few_kernel<T, ACT, 2> : glu_few_kernel<T, ACT, 4>;
        hipLaunchKernelGGL(kern, dim3(a.ff / 8), dim3(256), 0, st, a);
        DS_LAUNCH_CHECK();
        return DS_OK;
    });
}

ds_status glu_fwd_few(const GluArgs& a, hipStream_t st) { return a.dtype == DS_DTYPE_BF16 ? few_launch<bf16_t>(a, st) : few_launch<float>(a, st); }

ds_status glu_wgrad_tile(const GluWgrad& a, hipStream_t st) {
    static std::atomic<uint64_t> allowed{0};
    const ds_status r = allow_dynamic_lds(glu_wgrad_kernel, 2 * STAGE, allowed);
    if (r != DS_OK) return r;
    const int tiles_m = (a.d + 127) / 128, tiles_n = (a.ff + 127) / 128;
    hipLaunchKernelGGL(glu_wgrad_kernel, dim3((unsigned)tiles_m * tiles_n, a.splits, 2), dim3(256), 2 * STAGE, st, a, tiles_m, tiles_n);
    DS_LAUNCH_CHECK();
    if (a.splits == 1) return DS_OK;
    const long long n4 = (long long)a.d * a.ff / 4;
    hipLaunchKernelGGL(glu_wgrad_finish_kernel, dim3((unsigned)std::min<long long>((n4 + 255) / 256, 2048), 2), dim3(256), 0, st, a, n4);
    DS_LAUNCH_CHECK();
    return DS_OK;
}
