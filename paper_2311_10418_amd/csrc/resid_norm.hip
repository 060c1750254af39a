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
//
// Measured with both norms: bf16, 65 582 x 2048, column gate, forward 211 us (5.1 TB/s; a large copy 5.0); bf16, 131 072 x 4096, a gate per token,
// backward 1 624 us (5.3 TB/s), of which the second stage of the column sums takes 10; 65 629 x 1024, column gate, RMSNorm, backward 160 us (5.0 TB/s);
// fp32, 517 x 256, forward 4 us, which is what a launch and two trips to memory take.
#include "common.hpp"
#include "gemm.hpp"

namespace {

constexpr int kMaxCols = 4096;                          // as ds_norm_fwd / ds_norm_bwd
constexpr int kMaxRows = 0x7fffffff - (1 << 16);        // a turn further is still an int

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
    u32x4_t v = {0u, 0u, 0u, 0u};
    __device__ __forceinline__ void load(const bf16_t* p) { v = *reinterpret_cast<const u32x4_t*>(p); }
    __device__ __forceinline__ void clear() { v = u32x4_t{0u, 0u, 0u, 0u}; }
    __device__ __forceinline__ float at(int j) const { return __builtin_bit_cast(float, (j & 1) ? v[j >> 1] & 0xFFFF0000u : v[j >> 1] << 16); }
};
template <> struct Raw8<float> {
    f32x4_t a = {0.f, 0.f, 0.f, 0.f}, b = {0.f, 0.f, 0.f, 0.f};
    __device__ __forceinline__ void load(const float* p) { a = *reinterpret_cast<const f32x4_t*>(p); b = *reinterpret_cast<const f32x4_t*>(p + 4); }
    __device__ __forceinline__ void clear() { a = b = f32x4_t{0.f, 0.f, 0.f, 0.f}; }
    __device__ __forceinline__ float at(int j) const { return j < 4 ? a[j & 3] : b[j & 3]; }
};

template <class T> __device__ __forceinline__ void load_vector(const void* p, int col, bool in, float fill, float (&v)[8]) {
    if (p && in) Vec8<T>::load((const T*)p + col, v);
    else
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = fill;
}
template <class T> __device__ __forceinline__ void store_row(void* p, size_t at, const float (&v)[8], bool valid) {
    const float none[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (valid) Vec8<T>::store((T*)p + at, v);
    else Vec8<T>::store((T*)p + at, none);
}

template <int NW> constexpr int rows_at_once() { return NW >= 4 ? 1 : 4 / NW; }

// Sum over the wavefront, the same in every lane, with the adder's own lane exchange (six additions; through LDS shuffles the kernels' vector and LDS
// work took as long as their memory traffic): pairs, fours, halves of 16, 16, then 16 to 16 upwards into lane 63.
template <int CTRL, int ROWS> __device__ __forceinline__ float add_lanes(float v) {
    return v + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, ROWS, 0xF, false));
}
__device__ __forceinline__ float lanes_sum(float v) {
    v = add_lanes<0xB1, 0xF>(v);                        // lane ^ 1
    v = add_lanes<0x4E, 0xF>(v);                        // lane ^ 2
    v = add_lanes<0x141, 0xF>(v);                       // mirrored within 8
    v = add_lanes<0x140, 0xF>(v);                       // mirrored within 16
    v = add_lanes<0x142, 0xA>(v);                       // lane 15 of rows 0 and 2 to rows 1 and 3
    v = add_lanes<0x143, 0xC>(v);                       // lane 31 to rows 2 and 3
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 63));
}

// 1 / sqrt(v), v >= 1e-6: the hardware's estimate (one unit in the last place) and one step of Newton's method; 0 for the infinity that the sum of
// squares of a row of large values becomes, where the step would make inf x 0 (ds_norm_fwd has 0 there, too: the row is its bias)
__device__ __forceinline__ float inv_sqrt(float v) {
    const float r = __builtin_amdgcn_rsqf(v);
    return r == 0.f ? 0.f : r * __builtin_fmaf(-0.5f * v * r, r, 1.5f);
}

// The columns of a wavefront's row: `n` of them here, of d in all
struct RowShare {
    int d, part, lane;
    float n, inv_n, inv_d;
    bool in;
};
template <int NW> __device__ __forceinline__ float share_of(int d, int w) { return (float)min(512, max(0, d - 512 * w)); }

// t = v - mean, and rstd, of the rows of a work-group; v: this lane's columns, red: LDS of this use
template <bool RMS, int NW>
__device__ __forceinline__ void row_moments(const float (&v)[8], float (&t)[8], const RowShare& c, float2* red, float& mean, float& rstd) {
    float q = 0.f, m = 0.f;
    if (!RMS) {
        float s = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) s += v[j];
        m = lanes_sum(c.in ? s : 0.f) * c.inv_n;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        t[j] = RMS ? v[j] : v[j] - m;
        q = __builtin_fmaf(t[j], t[j], q);
    }
    q = lanes_sum(c.in ? q : 0.f);
    mean = m;
    if constexpr (NW > 1) {
        if (c.lane == 0) red[c.part] = make_float2(m, q);
        __syncthreads();
        float all = 0.f;
        q = 0.f;
        if (!RMS) {
#pragma unroll
            for (int w = 0; w < NW; ++w) all = __builtin_fmaf(share_of<NW>(c.d, w), red[w].x, all);
            all *= c.inv_d;
        }
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            const float2 r = red[w];
            const float off = r.x - all;
            q += RMS ? r.y : __builtin_fmaf(share_of<NW>(c.d, w) * off, off, r.y);
        }
        if (!RMS) {
            mean = all;
#pragma unroll
            for (int j = 0; j < 8; ++j) t[j] = v[j] - all;
        }
    }
    rstd = inv_sqrt(__builtin_fmaf(q, c.inv_d, RMS ? kRmsEps : kLnEps));
}

template <int NW> __device__ __forceinline__ RowShare row_share(int d) {
    RowShare c;
    c.d = d;
    c.part = (threadIdx.x >> 6) % NW;
    c.lane = threadIdx.x & 63;
    c.n = share_of<NW>(d, c.part);
    c.inv_n = c.n > 0.f ? 1.0f / c.n : 0.f;
    c.inv_d = 1.0f / (float)d;
    c.in = c.part * 512 + c.lane * 8 < d;
    return c;
}

// ------------------------------------------------------------------ forward
template <class T, bool RMS, int NW>
__global__ __launch_bounds__(NW == 8 ? 512 : 256) void resid_norm_fwd_kernel(ResidNormArgs a) {
    constexpr int RA = rows_at_once<NW>();
    __shared__ float2 red[2][2][RA][NW];
    const RowShare c = row_share<NW>(a.d);
    const int slot = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) / NW, col = c.part * 512 + c.lane * 8;
    const bool post = a.post_g != nullptr, pre = a.pre_g != nullptr, row_gate = a.gate_kind == DS_GATE_ROW;
    float post_g[8], post_b[8], pre_g[8], pre_b[8], gate[8];
    load_vector<T>(a.post_g, col, c.in, 1.f, post_g);
    load_vector<T>(a.post_b, col, c.in, 0.f, post_b);
    load_vector<T>(a.pre_g, col, c.in, 1.f, pre_g);
    load_vector<T>(a.pre_b, col, c.in, 0.f, pre_b);
    load_vector<T>(a.gate_kind == DS_GATE_COL ? a.gate : nullptr, col, c.in, 1.f, gate);
#pragma unroll
    for (int j = 0; j < 8; ++j) {                       // y = a_r x + post_g . unit row + post_b: the gate and a_b are part of the vectors
        gate[j] *= a.branch_scale;
        post_g[j] *= gate[j];
        post_b[j] *= gate[j];
    }
    Raw8<T> nx, nh, ng;
    int nvalid = 0;
    auto fetch = [&](int row) {
        if (row >= a.rows) return;
        nvalid = a.row_valid ? a.row_valid[row] : 0;
        if (!c.in) return;
        const size_t at = (size_t)row * a.d + col;
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
        float z[8], y[8], t[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            z[j] = nh.at(j);
            y[j] = a.resid_scale * nx.at(j);
        }
        if (row_gate)
#pragma unroll
            for (int j = 0; j < 8; ++j) gate[j] = ng.at(j);
        fetch(row + step);
        float hm = 0.f, hr = 0.f, ym = 0.f, yr = 0.f;
        if (post) {
            row_moments<RMS, NW>(z, t, c, red[par][0][slot], hm, hr);
#pragma unroll
            for (int j = 0; j < 8; ++j) z[j] = __builtin_fmaf(t[j] * hr, post_g[j], post_b[j]);
        }
        if (row_gate || !post)
#pragma unroll
            for (int j = 0; j < 8; ++j) z[j] *= gate[j];
        if (row_gate && !post)
#pragma unroll
            for (int j = 0; j < 8; ++j) z[j] *= a.branch_scale;
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = to_f32(from_f32<T>(y[j] + z[j]));      // the stream as it is stored: u is its norm
        const size_t at = (size_t)row * a.d + col;
        if (c.in && exists) store_row<T>(a.y, at, y, valid);
        if (pre) {
            row_moments<RMS, NW>(y, t, c, red[par][1][slot], ym, yr);
#pragma unroll
            for (int j = 0; j < 8; ++j) y[j] = __builtin_fmaf(t[j] * yr, pre_g[j], pre_b[j]);
            if (c.in && exists) store_row<T>(a.u, at, y, valid);
        }
        if (c.lane == 0 && c.part == 0 && exists) {
            a.stats[row] = valid ? hm : 0.f;
            a.stats[(size_t)a.rows + row] = valid ? hr : 0.f;
            a.stats[2 * (size_t)a.rows + row] = valid ? ym : 0.f;
            a.stats[3 * (size_t)a.rows + row] = valid ? yr : 0.f;
        }
    }
}

// ------------------------------------------------------------------ backward
// sums of two values over the columns of a row
template <bool TWO, int NW>
__device__ __forceinline__ void row_sums(float& p, float& q, const RowShare& c, float2* red) {
    p = TWO ? lanes_sum(c.in ? p : 0.f) : 0.f;
    q = lanes_sum(c.in ? q : 0.f);
    if constexpr (NW > 1) {
        if (c.lane == 0) red[c.part] = make_float2(p, q);
        __syncthreads();
        p = q = 0.f;
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            p += red[w].x;
            q += red[w].y;
        }
    }
    p *= c.inv_d;
    q *= c.inv_d;
}

// With dt = dy + N_pre'(du . pre_g) the gradient of y:  dx = a_r dt,  t = a_b dt,  q = gate . t,  dh = N_post'(q . post_g),  where
// N'(c) = rstd (c - mean(c) - hat mean(c hat))  (RMSNorm: no mean(c)).
// Column sums over the rows of a work-group: 0: sum s . hhat, 1: sum s, 2: sum du . yhat, 3: sum du, with s = q under a gate per
// token and s = t otherwise (without N_post hhat stands for h); the gains' and the column gate's gradients are products of the
// first two with vectors, taken once in the end: dpost_g = gate S0, dpost_b = gate S1, dgate = post_g S0 + post_b S1.
template <class T, bool RMS, int NW>
__global__ __launch_bounds__(NW == 8 ? 512 : 256) void resid_norm_bwd_kernel(ResidNormArgs a) {
    constexpr int RA = rows_at_once<NW>();
    __shared__ float2 red[2][2][RA][NW];
    const RowShare c = row_share<NW>(a.d);
    const int slot = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) / NW, col = c.part * 512 + c.lane * 8;
    const bool post = a.post_g != nullptr, pre = a.pre_g != nullptr, row_gate = a.gate_kind == DS_GATE_ROW;
    const bool need_h = post || a.gate_kind != DS_GATE_NONE;
    float post_g[8], post_b[8], pre_g[8], gate[8];
    load_vector<T>(a.post_g, col, c.in, 1.f, post_g);
    load_vector<T>(row_gate ? a.post_b : nullptr, col, c.in, 0.f, post_b);
    load_vector<T>(a.pre_g, col, c.in, 1.f, pre_g);
    load_vector<T>(a.gate_kind == DS_GATE_COL ? a.gate : nullptr, col, c.in, 1.f, gate);
    float s0[8], s1[8], s2[8], s3[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) s0[j] = s1[j] = s2[j] = s3[j] = 0.f;
    Raw8<T> ndy, ndu, ny, nh, ng;
    int nvalid = 0;
    float nhm = 0.f, nhr = 1.f, nym = 0.f, nyr = 0.f;
    auto fetch = [&](int row) {
        nvalid = -1;
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
        if (!c.in) return;
        const size_t at = (size_t)row * a.d + col;
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
        const bool exists = row < a.rows;
        if (nvalid < 0) {                               // a row that does not count: zeros throughout
            ndy.clear();
            ndu.clear();
            ny.clear();
            nh.clear();
            ng.clear();
            nhm = nhr = nym = nyr = 0.f;
        }
        float dt[8], hh[8], o[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            dt[j] = ndy.at(j);
            hh[j] = nh.at(j);
        }
        if (row_gate)
#pragma unroll
            for (int j = 0; j < 8; ++j) gate[j] = ng.at(j);
        const float hm = nhm, hr = nhr;
        if (pre) {
            float yh[8], k[8], c1 = 0.f, c2 = 0.f;
            const float shift = RMS ? 0.f : -nym * nyr, yr = nyr;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float du = ndu.at(j);
                yh[j] = __builtin_fmaf(ny.at(j), yr, shift);
                s2[j] = __builtin_fmaf(du, yh[j], s2[j]);
                s3[j] += du;
                k[j] = du * pre_g[j];
                c1 += k[j];
                c2 = __builtin_fmaf(k[j], yh[j], c2);
            }
            fetch(row + step);
            row_sums<!RMS, NW>(c1, c2, c, red[par][0][slot]);
#pragma unroll
            for (int j = 0; j < 8; ++j) dt[j] = __builtin_fmaf(yr, __builtin_fmaf(-yh[j], c2, RMS ? k[j] : k[j] - c1), dt[j]);
        } else {
            fetch(row + step);
        }
        const size_t at = (size_t)row * a.d + col;
#pragma unroll
        for (int j = 0; j < 8; ++j) o[j] = a.resid_scale * dt[j];
        if (c.in && exists) Vec8<T>::store((T*)a.dx + at, o);
        if (post) {
            const float shift = RMS ? 0.f : -hm * hr;
#pragma unroll
            for (int j = 0; j < 8; ++j) hh[j] = __builtin_fmaf(hh[j], hr, shift);
        }
        if (row_gate) {
#pragma unroll
            for (int j = 0; j < 8; ++j) o[j] = a.branch_scale * dt[j] * (post ? __builtin_fmaf(hh[j], post_g[j], post_b[j]) : hh[j]);
            if (c.in && exists) Vec8<T>::store((T*)a.dgate + at, o);
        }
        float q[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float t = a.branch_scale * dt[j];
            q[j] = t * gate[j];
            const float s = row_gate ? q[j] : t;
            s0[j] = __builtin_fmaf(s, hh[j], s0[j]);
            s1[j] += s;
        }
        if (post) {
            float c1 = 0.f, c2 = 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                q[j] *= post_g[j];
                c1 += q[j];
                c2 = __builtin_fmaf(q[j], hh[j], c2);
            }
            row_sums<!RMS, NW>(c1, c2, c, red[par][1][slot]);
#pragma unroll
            for (int j = 0; j < 8; ++j) q[j] = hr * __builtin_fmaf(-hh[j], c2, RMS ? q[j] : q[j] - c1);
        }
        if (c.in && exists) Vec8<T>::store((T*)a.dh + at, q);
    }
    // the rows that the work-group took side by side are added through LDS, in order
    __shared__ float comb[RA > 1 ? RA - 1 : 1][RA > 1 ? 64 * NW * 8 : 1];
    auto finish = [&](float (&s)[8], int k) {
        if constexpr (RA > 1) {
            __syncthreads();
            if (slot > 0)
#pragma unroll
                for (int j = 0; j < 8; ++j) comb[slot - 1][(c.part * 64 + c.lane) * 8 + j] = s[j];
            __syncthreads();
            if (slot == 0)
#pragma unroll
                for (int i = 0; i < RA - 1; ++i)
#pragma unroll
                    for (int j = 0; j < 8; ++j) s[j] += comb[i][(c.part * 64 + c.lane) * 8 + j];
        }
        if (slot == 0 && c.in) Vec8<float>::store(a.partial + ((size_t)blockIdx.x * 4 + k) * a.d + col, s);
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
            const float* p = a.partial + (size_t)k * a.d + col;
            int i = g;
            for (; i + 7 * 64 < a.n; i += 8 * 64) {     // eight loads in flight
                float v[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = p[(size_t)(i + 64 * j) * 4 * a.d];
#pragma unroll
                for (int j = 0; j < 8; ++j) s[k] += v[j];
            }
            for (; i < a.n; i += 64) s[k] += p[(size_t)i * 4 * a.d];
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

int row_waves(int d) { return d <= 512 ? 1 : d <= 1024 ? 2 : d <= 2048 ? 4 : 8; }
int rows_per_group(int d) { const int nw = row_waves(d); return nw >= 4 ? 1 : 4 / nw; }

// Work-groups of `kern` that the GPU holds at once.  The kernels walk rows, so with more of them than that the last ones would run while most of the
// chip is idle (backward 131 072 x 4 096: 1 024 work-groups where 768 fit took a third longer for the rows of the last 256).
template <class Kern>
int resident_groups(Kern kern, int threads, int& cached) {
    int per_cu = __atomic_load_n(&cached, __ATOMIC_RELAXED);
    if (per_cu == 0) {
        if (hipOccupancyMaxActiveBlocksPerMultiprocessor(&per_cu, reinterpret_cast<const void*>(kern), threads, 0) != hipSuccess || per_cu < 1) per_cu = 1;
        __atomic_store_n(&cached, per_cu, __ATOMIC_RELAXED);
    }
    return gemm_cu_count() * per_cu;
}

// most work-groups of the backward kernel = rows of partial sums: at most eight rows for each slot of a work-group until there are 1 024 of them (or what
// the GPU holds), and so at most 2^24 floats of partial sums
int bwd_most_groups(int rows, int d) {
    const int at_once = rows_per_group(d);
    const long long n = ((long long)rows + 8 * at_once - 1) / (8 * at_once), most = 1024;
    return (int)(n < 1 ? 1 : n < most ? n : most);
}

template <class T, bool RMS, int NW>
ds_status fwd_launch_nw(const ResidNormArgs& a, hipStream_t st) {
    static int cached = 0;
    constexpr int RA = rows_at_once<NW>(), threads = NW == 8 ? 512 : 256;
    auto kern = resid_norm_fwd_kernel<T, RMS, NW>;
    const long long need = ((long long)a.rows + RA - 1) / RA, fit = resident_groups(kern, threads, cached);
    hipLaunchKernelGGL(kern, dim3((unsigned)(need < fit ? need : fit)), dim3(threads), 0, st, a);
    DS_LAUNCH_CHECK();
    return DS_OK;
}
// groups: the rows of partial sums that were written
template <class T, bool RMS, int NW>
ds_status bwd_launch_nw(const ResidNormArgs& a, hipStream_t st, int& groups) {
    static int cached = 0;
    constexpr int threads = NW == 8 ? 512 : 256;
    auto kern = resid_norm_bwd_kernel<T, RMS, NW>;
    const int most = bwd_most_groups(a.rows, a.d), fit = resident_groups(kern, threads, cached);
    groups = most < fit ? most : fit;
    hipLaunchKernelGGL(kern, dim3((unsigned)groups), dim3(threads), 0, st, a);
    DS_LAUNCH_CHECK();
    return DS_OK;
}

template <class T, bool RMS>
ds_status fwd_launch(const ResidNormArgs& a, hipStream_t st) {
    switch (row_waves(a.d)) {
        case 1: return fwd_launch_nw<T, RMS, 1>(a, st);
        case 2: return fwd_launch_nw<T, RMS, 2>(a, st);
        case 4: return fwd_launch_nw<T, RMS, 4>(a, st);
        default: return fwd_launch_nw<T, RMS, 8>(a, st);
    }
}

template <class T, bool RMS>
ds_status bwd_launch(const ResidNormArgs& a, hipStream_t st, int& groups) {
    switch (row_waves(a.d)) {
        case 1: return bwd_launch_nw<T, RMS, 1>(a, st, groups);
        case 2: return bwd_launch_nw<T, RMS, 2>(a, st, groups);
        case 4: return bwd_launch_nw<T, RMS, 4>(a, st, groups);
        default: return bwd_launch_nw<T, RMS, 8>(a, st, groups);
    }
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
    return (int64_t)bwd_most_groups(rows, d) * 4 * d;
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
    int groups = 0;
    if (dtype == DS_DTYPE_BF16) r = rms ? bwd_launch<bf16_t, true>(a, st, groups) : bwd_launch<bf16_t, false>(a, st, groups);
    else r = rms ? bwd_launch<float, true>(a, st, groups) : bwd_launch<float, false>(a, st, groups);
    if (r != DS_OK) return r;
    ResidSumArgs s = {};
    s.n = groups; s.d = d; s.gate_kind = gate_kind; s.accumulate = accumulate; s.rms = rms;
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
