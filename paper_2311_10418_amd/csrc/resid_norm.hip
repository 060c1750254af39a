// The joint between two blocks, one pass over the rows: with N a LayerNorm or RMSNorm over the columns,
//     z = N_post(h)  (or h),   y = a_r x + a_b gate . z  (stored),   u = N_pre(y as stored)
// forward, and its gradient.  Bound by memory: forward two tensors are read and two written, backward four and two (a gate per
// token adds one to each side); what lies between stays in registers.
//
// A row belongs to NW wavefronts, 8 consecutive columns per lane (one 16-byte access per bf16 tensor); a work-group walks rows
// with the next row's loads in flight, and keeps the gains, the biases and (backward) the column sums of its rows in registers.
//
// Forward statistics: every wavefront takes the mean and the squared distances from it of its own columns (two passes over
// registers), and what the wavefronts have is joined through LDS, one barrier per norm: with n_w columns, mean m_w and squares
// q_w,  m = sum n_w m_w / d  and  q = sum q_w + n_w (m_w - m)^2, which cancels nothing.
// All sums, statistics and gradients of parameters are fp32; tensors are rounded once, as they are stored.
#include "common.hpp"

namespace {

constexpr int kMaxCols = 8192;
constexpr int kMaxRows = 0x7fffffff - (1 << 16);        // a turn further is still an int

struct NormVectors {                                    // gains, biases, column gate of the columns of a lane
    float post_g[8], post_b[8], pre_g[8], pre_b[8], gate[8];
};

struct ResidNormArgs {
    int32_t rows, d, gate_kind;
    float resid_scale, branch_scale;
    const int32_t* row_valid;
    const void *x, *h, *post_g, *post_b, *gate, *pre_g, *pre_b, *dy, *du;
    void *y, *u, *dx, *dh, *dgate;
    float* stats;                                       // [4][rows]: mean and rstd of h, mean and rstd of y
    float* partial;                                     // backward: [work-groups][4][d]
};

template <class T> struct Raw8;                         // 8 elements as loaded
template <> struct Raw8<bf16_t> {
    bf16x8_t v;
    __device__ __forceinline__ void load(const bf16_t* p) { v = *reinterpret_cast<const bf16x8_t*>(p); }
    __device__ __forceinline__ float at(int j) const { return (float)v[j]; }
};
template <> struct Raw8<float> {
    float4 a, b;
    __device__ __forceinline__ void load(const float* p) { a = *reinterpret_cast<const float4*>(p); b = *reinterpret_cast<const float4*>(p + 4); }
    __device__ __forceinline__ float at(int j) const { return j == 0 ? a.x : j == 1 ? a.y : j == 2 ? a.z : j == 3 ? a.w : j == 4 ? b.x : j == 5 ? b.y : j == 6 ? b.z : b.w; }
};

template <class T> __device__ __forceinline__ void load_vector(const void* p, int col, bool in, float fill, float (&v)[8]) {
    if (p && in) Vec8<T>::load((const T*)p + col, v);
    else
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = fill;
}

template <int NW> constexpr int rows_at_once() { return NW >= 4 ? 1 : 4 / NW; }

// mean and rstd of the rows of a work-group; v: this lane's columns, n_w: columns of its wavefront, red: LDS of this use
template <bool RMS, int NW>
__device__ __forceinline__ void row_moments(const float (&v)[8], bool in, int n_w, int d, float2 (*red)[NW], int slot, int part, int lane, float& mean, float& rstd) {
    float s = 0.f, q = 0.f, m = 0.f;
    if (!RMS) {
#pragma unroll
        for (int j = 0; j < 8; ++j) s += v[j];
        s = wave_sum(in ? s : 0.f);
        m = n_w > 0 ? s / (float)n_w : 0.f;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) q += (v[j] - m) * (v[j] - m);
    q = wave_sum(in ? q : 0.f);
    mean = m;
    if constexpr (NW > 1) {
        if (lane == 0) red[slot][part] = make_float2(m, q);
        __syncthreads();
        float all = 0.f, qs = 0.f;
        if (!RMS) {
#pragma unroll
            for (int w = 0; w < NW; ++w) all += (float)min(512, max(0, d - 512 * w)) * red[slot][w].x;
            all /= (float)d;
        }
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            const float2 r = red[slot][w];
            qs += r.y;
            if (!RMS) qs += (float)min(512, max(0, d - 512 * w)) * (r.x - all) * (r.x - all);
        }
        mean = all;
        q = qs;
    }
    rstd = 1.0f / sqrtf(q / (float)d + (RMS ? kRmsEps : kLnEps));
}

// ------------------------------------------------------------------ forward
template <class T, bool RMS, int NW>
__global__ __launch_bounds__(NW > 4 ? 64 * NW : 256) void resid_norm_fwd_kernel(ResidNormArgs a) {
    constexpr int RA = rows_at_once<NW>();
    __shared__ float2 red[2][2][RA][NW];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int slot = wave / NW, part = wave % NW;
    const int d = a.d, col = part * 512 + lane * 8;
    const bool in = col < d;
    const int n_w = min(512, max(0, d - 512 * part));
    const bool post = a.post_g != nullptr, pre = a.pre_g != nullptr;
    NormVectors w;
    load_vector<T>(a.post_g, col, in, 1.f, w.post_g);
    load_vector<T>(a.post_b, col, in, 0.f, w.post_b);
    load_vector<T>(a.pre_g, col, in, 1.f, w.pre_g);
    load_vector<T>(a.pre_b, col, in, 0.f, w.pre_b);
    load_vector<T>(a.gate_kind == DS_GATE_COL ? a.gate : nullptr, col, in, 1.f, w.gate);
    const bool row_gate = a.gate_kind == DS_GATE_ROW;
    Raw8<T> nx, nh, ng;
    int nvalid = 0;
    auto fetch = [&](int row) {
        if (row >= a.rows) return;
        nvalid = a.row_valid ? a.row_valid[row] : 0;
        if (!in) return;
        const size_t at = (size_t)row * d + col;
        nx.load((const T*)a.x + at);
        nh.load((const T*)a.h + at);
        if (row_gate) ng.load((const T*)a.gate + at);
    };
    const int step = gridDim.x * RA;
    fetch(blockIdx.x * RA + slot);
    int par = 0;
    for (int r0 = blockIdx.x * RA; r0 < a.rows; r0 += step, par ^= 1) {      // every wavefront: the same number of turns
        const int row = r0 + slot;
        const bool exists = row < a.rows, valid = nvalid >= 0;
        float z[8], x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            z[j] = in && exists && valid ? nh.at(j) : 0.f;
            x[j] = in && exists && valid ? nx.at(j) : 0.f;
        }
        float gate[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) gate[j] = row_gate && in && exists ? ng.at(j) : w.gate[j];
        fetch(row + step);
        float hm = 0.f, hr = 0.f, ym = 0.f, yr = 0.f;
        if (post) {
            row_moments<RMS, NW>(z, in, n_w, d, red[par][0], slot, part, lane, hm, hr);
#pragma unroll
            for (int j = 0; j < 8; ++j) z[j] = (z[j] - hm) * hr * w.post_g[j] + w.post_b[j];
        }
        float y[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float v = a.resid_scale * x[j] + a.branch_scale * gate[j] * z[j];
            y[j] = valid ? to_f32(from_f32<T>(v)) : 0.f;                      // the stream as it is stored: u is its norm
        }
        const size_t at = (size_t)row * d + col;
        if (in && exists) Vec8<T>::store((T*)a.y + at, y);
        if (pre) {
            row_moments<RMS, NW>(y, in, n_w, d, red[par][1], slot, part, lane, ym, yr);
            float u[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) u[j] = valid ? (y[j] - ym) * yr * w.pre_g[j] + w.pre_b[j] : 0.f;
            if (in && exists) Vec8<T>::store((T*)a.u + at, u);
        }
        if (lane == 0 && part == 0 && exists) {
            a.stats[row] = hm;
            a.stats[(size_t)a.rows + row] = hr;
            a.stats[2 * (size_t)a.rows + row] = ym;
            a.stats[3 * (size_t)a.rows + row] = yr;
        }
    }
}

// ------------------------------------------------------------------ backward
// sums of two values over the columns of a row
template <int NW>
__device__ __forceinline__ void row_sums(float& p, float& q, bool two, float2 (*red)[NW], int slot, int part, int lane) {
    if (two) p = wave_sum(p);
    q = wave_sum(q);
    if constexpr (NW > 1) {
        if (lane == 0) red[slot][part] = make_float2(p, q);
        __syncthreads();
        p = q = 0.f;
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            p += red[slot][w].x;
            q += red[slot][w].y;
        }
    }
}

// With dt = dy + N_pre'(du . pre_g) the gradient of y:  dx = a_r dt,  t = a_b dt,  q = gate . t,  dh = N_post'(q . post_g),  where
// N'(c) = rstd (c - mean(c) - hat mean(c hat))  (RMSNorm: no mean(c)).
// Column sums over the rows of a work-group: 0: sum s . hhat, 1: sum s, 2: sum du . yhat, 3: sum du, with s = q under a gate per
// token and s = t otherwise (without N_post hhat stands for h); the gains' and the column gate's gradients are products of the
// first two with vectors, taken once in the end: dpost_g = gate S0, dpost_b = gate S1, dgate = post_g S0 + post_b S1.
template <class T, bool RMS, int NW>
__global__ __launch_bounds__(NW > 4 ? 64 * NW : 256) void resid_norm_bwd_kernel(ResidNormArgs a) {
    constexpr int RA = rows_at_once<NW>();
    __shared__ float2 red[2][2][RA][NW];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int slot = wave / NW, part = wave % NW;
    const int d = a.d, col = part * 512 + lane * 8;
    const bool in = col < d;
    const bool post = a.post_g != nullptr, pre = a.pre_g != nullptr, row_gate = a.gate_kind == DS_GATE_ROW;
    const bool need_h = post || a.gate_kind != DS_GATE_NONE;
    const float inv_d = 1.0f / (float)d;
    float post_g[8], post_b[8], pre_g[8], cgate[8];
    load_vector<T>(a.post_g, col, in, 1.f, post_g);
    load_vector<T>(row_gate ? a.post_b : nullptr, col, in, 0.f, post_b);
    load_vector<T>(a.pre_g, col, in, 1.f, pre_g);
    load_vector<T>(a.gate_kind == DS_GATE_COL ? a.gate : nullptr, col, in, 1.f, cgate);
    float s0[8], s1[8], s2[8], s3[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) s0[j] = s1[j] = s2[j] = s3[j] = 0.f;
    Raw8<T> ndy, ndu, ny, nh, ng;
    int nvalid = 0;
    float nhm = 0.f, nhr = 1.f, nym = 0.f, nyr = 0.f;
    auto fetch = [&](int row) {
        if (row >= a.rows) return;
        nvalid = a.row_valid ? a.row_valid[row] : 0;
        if (post) {
            nhm = a.stats[row];
            nhr = a.stats[(size_t)a.rows + row];
        }
        if (pre) {
            nym = a.stats[2 * (size_t)a.rows + row];
            nyr = a.stats[3 * (size_t)a.rows + row];
        }
        if (!in) return;
        const size_t at = (size_t)row * d + col;
        if (a.dy) ndy.load((const T*)a.dy + at);
        if (pre) {
            ndu.load((const T*)a.du + at);
            ny.load((const T*)a.y + at);
        }
        if (need_h) nh.load((const T*)a.h + at);
        if (row_gate) ng.load((const T*)a.gate + at);
    };
    const int step = gridDim.x * RA;
    fetch(blockIdx.x * RA + slot);
    int par = 0;
    for (int r0 = blockIdx.x * RA; r0 < a.rows; r0 += step, par ^= 1) {
        const int row = r0 + slot;
        const bool exists = row < a.rows, valid = nvalid >= 0, use = in && exists && valid;
        const float hm = nhm, hr = nhr, ym = nym, yr = nyr;
        float dt[8], du[8], yh[8], hh[8], gate[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            dt[j] = use && a.dy ? ndy.at(j) : 0.f;
            du[j] = use && pre ? ndu.at(j) : 0.f;
            yh[j] = use && pre ? (ny.at(j) - ym) * yr : 0.f;
            hh[j] = use && need_h ? (post ? (nh.at(j) - hm) * hr : nh.at(j)) : 0.f;
            gate[j] = use && row_gate ? ng.at(j) : cgate[j];
        }
        fetch(row + step);
        if (pre) {
            float c1 = 0.f, c2 = 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float c = du[j] * pre_g[j];
                if (!RMS) c1 += c;
                c2 += c * yh[j];
                s2[j] += du[j] * yh[j];
                s3[j] += du[j];
            }
            row_sums<NW>(c1, c2, !RMS, red[par][0], slot, part, lane);
            c1 *= inv_d;
            c2 *= inv_d;
#pragma unroll
            for (int j = 0; j < 8; ++j) dt[j] += use ? yr * (du[j] * pre_g[j] - (RMS ? 0.f : c1) - yh[j] * c2) : 0.f;
        }
        const size_t at = (size_t)row * d + col;
        float o[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) o[j] = a.resid_scale * dt[j];
        if (in && exists) Vec8<T>::store((T*)a.dx + at, o);
        float q[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float t = a.branch_scale * dt[j];
            q[j] = t * gate[j];
            const float s = row_gate ? q[j] : t;
            s0[j] += s * hh[j];
            s1[j] += s;
            if (row_gate) o[j] = t * (post ? hh[j] * post_g[j] + post_b[j] : hh[j]);
        }
        if (row_gate && in && exists) Vec8<T>::store((T*)a.dgate + at, o);
        if (post) {
            float c1 = 0.f, c2 = 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                q[j] *= post_g[j];
                if (!RMS) c1 += q[j];
                c2 += q[j] * hh[j];
            }
            row_sums<NW>(c1, c2, !RMS, red[par][1], slot, part, lane);
            c1 *= inv_d;
            c2 *= inv_d;
#pragma unroll
            for (int j = 0; j < 8; ++j) q[j] = use ? hr * (q[j] - (RMS ? 0.f : c1) - hh[j] * c2) : 0.f;
        }
        if (in && exists) Vec8<T>::store((T*)a.dh + at, q);
    }
    // the rows that the work-group took side by side are added through LDS, in order
    __shared__ float comb[RA > 1 ? RA - 1 : 1][RA > 1 ? 64 * NW * 8 : 1];
    auto finish = [&](float (&s)[8], int k) {
        if constexpr (RA > 1) {
            __syncthreads();
            if (slot > 0)
#pragma unroll
                for (int j = 0; j < 8; ++j) comb[slot - 1][(part * 64 + lane) * 8 + j] = s[j];
            __syncthreads();
            if (slot == 0)
#pragma unroll
                for (int i = 0; i < RA - 1; ++i)
#pragma unroll
                    for (int j = 0; j < 8; ++j) s[j] += comb[i][(part * 64 + lane) * 8 + j];
        }
        if (slot == 0 && in) Vec8<float>::store(a.partial + ((size_t)blockIdx.x * 4 + k) * d + col, s);
    };
    finish(s0, 0);
    if (!RMS) finish(s1, 1);
    if (pre) {
        finish(s2, 2);
        if (!RMS) finish(s3, 3);
    }
}

// out = (accumulate ? out : 0) + the work-groups' sums, in a fixed order: 16 columns per work-group, 64 threads take every 64th of
// the n partial rows of a column, and 4 of the sums at a time.
struct ResidSumArgs {
    int32_t n, d, gate_kind, accumulate, rms;
    const float* partial;
    const void *post_g, *post_b, *gate;
    float *dgate, *dpost_g, *dpost_b, *dpre_g, *dpre_b;
};
template <class T>
__global__ __launch_bounds__(1024) void resid_norm_sums_kernel(ResidSumArgs a) {
    __shared__ float part[4][64][17];
    const int c = threadIdx.x & 15, g = threadIdx.x >> 4, col = blockIdx.x * 16 + c;
    float s[4] = {0.f, 0.f, 0.f, 0.f};
    if (col < a.d) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if ((a.rms && (k & 1)) || (k >= 2 && !a.dpre_g)) continue;
            for (int i = g; i < a.n; i += 64) s[k] += a.partial[((size_t)i * 4 + k) * a.d + col];
        }
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) part[k][g][c] = s[k];
    for (int w = 32; w >= 1; w >>= 1) {
        __syncthreads();
        if (g < w)
#pragma unroll
            for (int k = 0; k < 4; ++k) part[k][g][c] += part[k][g + w][c];
    }
    if (g > 0 || col >= a.d) return;
#pragma unroll
    for (int k = 0; k < 4; ++k) s[k] = part[k][0][c];
    auto out = [&](float* p, float v) { p[col] = (a.accumulate ? p[col] : 0.f) + v; };
    const float gate = a.gate_kind == DS_GATE_COL ? to_f32(((const T*)a.gate)[col]) : 1.f;
    if (a.dpost_g) out(a.dpost_g, gate * s[0]);
    if (a.dpost_b) out(a.dpost_b, gate * s[1]);
    if (a.dgate) out(a.dgate, a.post_g ? to_f32(((const T*)a.post_g)[col]) * s[0] + (a.rms ? 0.f : to_f32(((const T*)a.post_b)[col]) * s[1]) : s[0]);
    if (a.dpre_g) out(a.dpre_g, s[2]);
    if (a.dpre_b) out(a.dpre_b, s[3]);
}

int row_waves(int d) { return d <= 512 ? 1 : d <= 1024 ? 2 : d <= 2048 ? 4 : d <= 4096 ? 8 : 16; }
int rows_per_group(int d) { const int nw = row_waves(d); return nw >= 4 ? 1 : 4 / nw; }

// work-groups of the backward kernel = rows of partial sums: enough to fill the chip, eight rows and more each, and at most 2^24
// floats of partial sums
int bwd_groups(int rows, int d) {
    const int at_once = rows_per_group(d);
    long long n = ((long long)rows + 8 * at_once - 1) / (8 * at_once);
    const long long most = d <= 4096 ? 1024 : 512;
    if (n > most) n = most;
    return (int)(n < 1 ? 1 : n);
}

template <class T, bool RMS>
ds_status fwd_launch(const ResidNormArgs& a, hipStream_t st) {
    const int nw = row_waves(a.d), ra = rows_per_group(a.d);
    long long groups = ((long long)a.rows + ra - 1) / ra;
    const long long most = 256 * 8;
    const dim3 grid((unsigned)(groups < most ? groups : most)), block(nw > 4 ? 64 * nw : 256);
    switch (nw) {
        case 1: hipLaunchKernelGGL((resid_norm_fwd_kernel<T, RMS, 1>), grid, block, 0, st, a); break;
        case 2: hipLaunchKernelGGL((resid_norm_fwd_kernel<T, RMS, 2>), grid, block, 0, st, a); break;
        case 4: hipLaunchKernelGGL((resid_norm_fwd_kernel<T, RMS, 4>), grid, block, 0, st, a); break;
        case 8: hipLaunchKernelGGL((resid_norm_fwd_kernel<T, RMS, 8>), grid, block, 0, st, a); break;
        default: hipLaunchKernelGGL((resid_norm_fwd_kernel<T, RMS, 16>), grid, block, 0, st, a); break;
    }
    DS_LAUNCH_CHECK();
    return DS_OK;
}

template <class T, bool RMS>
ds_status bwd_launch(const ResidNormArgs& a, hipStream_t st) {
    const int nw = row_waves(a.d);
    const dim3 grid((unsigned)bwd_groups(a.rows, a.d)), block(nw > 4 ? 64 * nw : 256);
    switch (nw) {
        case 1: hipLaunchKernelGGL((resid_norm_bwd_kernel<T, RMS, 1>), grid, block, 0, st, a); break;
        case 2: hipLaunchKernelGGL((resid_norm_bwd_kernel<T, RMS, 2>), grid, block, 0, st, a); break;
        case 4: hipLaunchKernelGGL((resid_norm_bwd_kernel<T, RMS, 4>), grid, block, 0, st, a); break;
        case 8: hipLaunchKernelGGL((resid_norm_bwd_kernel<T, RMS, 8>), grid, block, 0, st, a); break;
        default: hipLaunchKernelGGL((resid_norm_bwd_kernel<T, RMS, 16>), grid, block, 0, st, a); break;
    }
    DS_LAUNCH_CHECK();
    return DS_OK;
}

bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

// what forward and backward ask of their common arguments
bool common_ok(int32_t dtype, int32_t rms, int32_t rows, int32_t d, const void* h, const void* post_g, const void* post_b, int32_t gate_kind,
               const void* gate, const void* pre_g, const float* stats) {
    if (dtype != DS_DTYPE_F32 && dtype != DS_DTYPE_BF16) return false;
    if ((rms != 0 && rms != 1) || rows < 0 || rows > kMaxRows || d <= 0 || d % 8 || d > kMaxCols || !h || !stats) return false;
    if (gate_kind != DS_GATE_NONE && gate_kind != DS_GATE_COL && gate_kind != DS_GATE_ROW) return false;
    if ((gate_kind != DS_GATE_NONE) != (gate != nullptr)) return false;
    if (post_g && !rms && !post_b) return false;
    return aligned16(h) && aligned16(post_g) && aligned16(post_b) && aligned16(gate) && aligned16(pre_g);
}

}  // namespace

extern "C" int64_t ds_resid_norm_bwd_scratch_floats(int32_t rows, int32_t d) {
    if (rows <= 0 || d <= 0 || d > kMaxCols) return 0;
    return (int64_t)bwd_groups(rows, d) * 4 * d;
}

extern "C" ds_status ds_resid_norm_fwd(int32_t dtype, int32_t rms, int32_t rows, int32_t d, const void* x, const void* h, const int32_t* row_valid,
                                       const void* post_g, const void* post_b, int32_t gate_kind, const void* gate, float resid_scale,
                                       float branch_scale, const void* pre_g, const void* pre_b, void* y, void* u, float* stats, void* hip_stream) {
    if (!common_ok(dtype, rms, rows, d, h, post_g, post_b, gate_kind, gate, pre_g, stats) || !x || !y) return DS_EINVAL;
    if (pre_g && (!u || (!rms && !pre_b))) return DS_EINVAL;
    if (!aligned16(x) || !aligned16(y) || !aligned16(u) || !aligned16(pre_b)) return DS_EINVAL;
    if (rows == 0) return DS_OK;
    ResidNormArgs a = {};
    a.rows = rows; a.d = d; a.gate_kind = gate_kind;
    a.resid_scale = resid_scale; a.branch_scale = branch_scale;
    a.row_valid = row_valid;
    a.x = x; a.h = h; a.post_g = post_g; a.post_b = rms || !post_g ? nullptr : post_b; a.gate = gate; a.pre_g = pre_g; a.pre_b = rms || !pre_g ? nullptr : pre_b;
    a.y = y; a.u = u; a.stats = stats;
    hipStream_t st = (hipStream_t)hip_stream;
    if (dtype == DS_DTYPE_BF16) return rms ? fwd_launch<bf16_t, true>(a, st) : fwd_launch<bf16_t, false>(a, st);
    return rms ? fwd_launch<float, true>(a, st) : fwd_launch<float, false>(a, st);
}

extern "C" ds_status ds_resid_norm_bwd(int32_t dtype, int32_t rms, int32_t rows, int32_t d, const void* dy, const void* du, const void* y, const void* h,
                                       const int32_t* row_valid, const void* post_g, const void* post_b, int32_t gate_kind, const void* gate,
                                       float resid_scale, float branch_scale, const void* pre_g, const float* stats, void* dx, void* dh, void* dgate,
                                       float* dpost_g, float* dpost_b, float* dpre_g, float* dpre_b, float* partial, int32_t accumulate,
                                       void* hip_stream) {
    if (!common_ok(dtype, rms, rows, d, h, post_g, post_b, gate_kind, gate, pre_g, stats) || rows == 0 || !dx || !dh || !partial) return DS_EINVAL;
    if (accumulate != 0 && accumulate != 1) return DS_EINVAL;
    if (!dy && !pre_g) return DS_EINVAL;
    if (pre_g && (!du || !y || !dpre_g || (!rms && !dpre_b))) return DS_EINVAL;
    if (post_g && (!dpost_g || (!rms && !dpost_b))) return DS_EINVAL;
    if (gate_kind != DS_GATE_NONE && !dgate) return DS_EINVAL;
    if (!aligned16(dy) || !aligned16(du) || !aligned16(y) || !aligned16(dx) || !aligned16(dh) || !aligned16(dgate) || !aligned16(partial)) return DS_EINVAL;
    ResidNormArgs a = {};
    a.rows = rows; a.d = d; a.gate_kind = gate_kind;
    a.resid_scale = resid_scale; a.branch_scale = branch_scale;
    a.row_valid = row_valid;
    a.h = h; a.post_g = post_g; a.post_b = rms || !post_g ? nullptr : post_b; a.gate = gate; a.pre_g = pre_g;
    a.dy = dy; a.du = du; a.y = const_cast<void*>(y);
    a.dx = dx; a.dh = dh; a.dgate = gate_kind == DS_GATE_ROW ? dgate : nullptr;
    a.stats = const_cast<float*>(stats);
    a.partial = partial;
    hipStream_t st = (hipStream_t)hip_stream;
    ds_status r;
    if (dtype == DS_DTYPE_BF16) r = rms ? bwd_launch<bf16_t, true>(a, st) : bwd_launch<bf16_t, false>(a, st);
    else r = rms ? bwd_launch<float, true>(a, st) : bwd_launch<float, false>(a, st);
    if (r != DS_OK) return r;
    ResidSumArgs s = {};
    s.n = bwd_groups(rows, d); s.d = d; s.gate_kind = gate_kind; s.accumulate = accumulate; s.rms = rms;
    s.partial = partial;
    s.post_g = post_g; s.post_b = post_b; s.gate = gate;
    s.dgate = gate_kind == DS_GATE_COL ? (float*)dgate : nullptr;
    s.dpost_g = post_g ? dpost_g : nullptr;
    s.dpost_b = post_g && !rms ? dpost_b : nullptr;
    s.dpre_g = pre_g ? dpre_g : nullptr;
    s.dpre_b = pre_g && !rms ? dpre_b : nullptr;
    if (!s.dgate && !s.dpost_g && !s.dpre_g) return DS_OK;
    const dim3 grid((unsigned)((d + 15) / 16));
    if (dtype == DS_DTYPE_BF16) hipLaunchKernelGGL(resid_norm_sums_kernel<bf16_t>, grid, dim3(1024), 0, st, s);
    else hipLaunchKernelGGL(resid_norm_sums_kernel<float>, grid, dim3(1024), 0, st, s);
    DS_LAUNCH_CHECK();
    return DS_OK;
}
