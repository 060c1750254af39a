// Rotary positions: the columns of a head are taken in pairs, and pair p of a token at position t is turned by the angle
// t freq[p]:  (x0, x1) -> amplitude (x0 cos - x1 sin, x1 cos + x0 sin).  The inverse turns by the negative angle with the same
// amplitude, which is also the gradient.  Pairs are (2p, 2p + 1), interleaved, or (p, p + rot / 2), halves.
//
// Bound by memory: every value is read and written once.  An angle is the same for all heads of a row, so a thread keeps the
// cosines and sines of its pairs in registers and walks over heads (about four: more of them would leave too few threads for the transfers).
// Measured: bf16, 65 582 rows of 64 heads of 64, 205 us (5.2 TB/s; a large copy 5.0); fp32, interleaved, half of every head of 128, 7 685 rows of 8,
// 13.3 us (4.8 TB/s); 64 rows of 64 heads of 64 4 us, a launch.
#include "common.hpp"

#include <cmath>

namespace {

// cos and sin of t * f.  The product is taken in 64 bits and reduced to a part of one turn there: at t = 2^20 and f = 1 a product in
// 32 bits is 0.03 rad off.  What is left is an eighth of a turn at most, where the series to x^10 (cosine) and x^9 (sine) end below
// 2^-27 of the largest value.
__device__ __forceinline__ void turn(int32_t t, double f, float amplitude, float& c, float& s) {
    const double x = (double)t * f;
    const double n = __builtin_rint(x * 0.63661977236758134308);             // quarter turns
    const float r = (float)__builtin_fma(n, -6.123233995736766e-17, __builtin_fma(n, -1.5707963267948966, x));
    const float w = r * r;
    float sn = __builtin_fmaf(w, 2.7557319e-6f, -1.9841270e-4f);
    sn = __builtin_fmaf(w, sn, 8.3333333e-3f);
    sn = __builtin_fmaf(w, sn, -1.6666667e-1f);
    sn = __builtin_fmaf(r * w, sn, r);
    float cs = __builtin_fmaf(w, -2.7557319e-7f, 2.4801587e-5f);
    cs = __builtin_fmaf(w, cs, -1.3888889e-3f);
    cs = __builtin_fmaf(w, cs, 4.1666667e-2f);
    cs = __builtin_fmaf(w, cs, -0.5f);
    cs = __builtin_fmaf(w, cs, 1.0f);
    const int q = (int)((long long)n) & 3;
    const float a = (q & 1) ? sn : cs, b = (q & 1) ? cs : sn;
    c = amplitude * ((q == 1 || q == 2) ? -a : a);
    s = amplitude * ((q & 2) ? -b : b);
}

struct RopeArgs {
    int32_t rows, n_heads, head_dim, rot, inverse;
    const int32_t* pos;
    const double* freq;
    float amplitude;
    const void* x;
    void* y;
    long long ldx, ldy;
    int32_t lanes, per_row;                             // threads side by side over a head's pairs; threads per row
};

// V pairs per thread: 8 (16-byte accesses) or 1.
template <class T, bool INTERLEAVED, int V>
__global__ __launch_bounds__(256) void rope_kernel(RopeArgs a) {
    const long long id = (long long)blockIdx.x * 256 + threadIdx.x;
    const int row = (int)(id / a.per_row), in_row = (int)(id - (long long)row * a.per_row);
    if (row >= a.rows) return;
    const int32_t t = a.pos[row];
    if (t < 0) return;
    const int chunk = in_row % a.lanes, h0 = in_row / a.lanes, hs = a.per_row / a.lanes;
    const int half = a.rot / 2, n_turn = half / V;
    const T* x = (const T*)a.x + (long long)row * a.ldx;
    T* y = (T*)a.y + (long long)row * a.ldy;
    if (chunk >= n_turn) {                              // columns behind the turned ones
        if (x == y) return;
        const int c = a.rot + (chunk - n_turn) * V;
        if (c >= a.head_dim) return;
        for (int h = h0; h < a.n_heads; h += hs) {
            if constexpr (V == 8) {
                float v[8];
                Vec8<T>::load(x + h * a.head_dim + c, v);
                Vec8<T>::store(y + h * a.head_dim + c, v);
            } else {
                y[h * a.head_dim + c] = x[h * a.head_dim + c];
            }
        }
        return;
    }
    float cs[V], sn[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
        turn(t, a.freq[chunk * V + j], a.amplitude, cs[j], sn[j]);
        if (a.inverse) sn[j] = -sn[j];
    }
    for (int h = h0; h < a.n_heads; h += hs) {
        const int base = h * a.head_dim;
        if constexpr (V == 8) {
            const int c0 = INTERLEAVED ? chunk * 16 : chunk * 8, c1 = INTERLEAVED ? chunk * 16 + 8 : half + chunk * 8;
            float p[8], q[8], o0[8], o1[8];
            Vec8<T>::load(x + base + c0, p);
            Vec8<T>::load(x + base + c1, q);
            if constexpr (INTERLEAVED) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    o0[2 * j] = p[2 * j] * cs[j] - p[2 * j + 1] * sn[j];
                    o0[2 * j + 1] = p[2 * j + 1] * cs[j] + p[2 * j] * sn[j];
                    o1[2 * j] = q[2 * j] * cs[j + 4] - q[2 * j + 1] * sn[j + 4];
                    o1[2 * j + 1] = q[2 * j + 1] * cs[j + 4] + q[2 * j] * sn[j + 4];
                }
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    o0[j] = p[j] * cs[j] - q[j] * sn[j];
                    o1[j] = q[j] * cs[j] + p[j] * sn[j];
                }
            }
            Vec8<T>::store(y + base + c0, o0);
            Vec8<T>::store(y + base + c1, o1);
        } else {
            const int c0 = INTERLEAVED ? 2 * chunk : chunk, c1 = INTERLEAVED ? 2 * chunk + 1 : half + chunk;
            const float p = to_f32(x[base + c0]), q = to_f32(x[base + c1]);
            y[base + c0] = from_f32<T>(p * cs[0] - q * sn[0]);
            y[base + c1] = from_f32<T>(q * cs[0] + p * sn[0]);
        }
    }
}

template <class T, int V>
ds_status rope_launch(RopeArgs a, bool interleaved, hipStream_t st) {
    const bool copies = a.x != a.y && a.rot < a.head_dim;
    a.lanes = a.rot / 2 / V + (copies ? (a.head_dim - a.rot) / V : 0);
    a.per_row = a.lanes * ((a.n_heads + 3) / 4);        // about four heads per thread
    // a launch has fewer than 2^32 threads, and per_row is below 2^30: a range of rows each
    const long long rows = a.rows, most = (0xffffffffLL / 256) * 256 / a.per_row;
    for (long long r0 = 0; r0 < rows; r0 += most) {
        RopeArgs part = a;
        part.rows = (int32_t)(rows - r0 < most ? rows - r0 : most);
        part.pos = a.pos + r0;
        part.x = (const T*)a.x + r0 * a.ldx;
        part.y = (T*)a.y + r0 * a.ldy;
        const dim3 grid((unsigned)(((long long)part.rows * a.per_row + 255) / 256));
        if (interleaved) hipLaunchKernelGGL((rope_kernel<T, true, V>), grid, dim3(256), 0, st, part);
        else hipLaunchKernelGGL((rope_kernel<T, false, V>), grid, dim3(256), 0, st, part);
        DS_LAUNCH_CHECK();
    }
    return DS_OK;
}

}  // namespace

extern "C" ds_status ds_rope(int32_t dtype, int32_t rows, int32_t n_heads, int32_t head_dim, int32_t rot_dim, int32_t interleaved, int32_t inverse,
                             const int32_t* pos, const double* freq, float amplitude, const void* x, int64_t ldx, void* y, int64_t ldy,
                             void* hip_stream) {
    if (dtype != DS_DTYPE_F32 && dtype != DS_DTYPE_BF16) return DS_EINVAL;
    if (rows < 0 || n_heads <= 0 || head_dim <= 0 || rot_dim <= 0 || rot_dim % 2 || rot_dim > head_dim) return DS_EINVAL;
    if ((interleaved != 0 && interleaved != 1) || (inverse != 0 && inverse != 1) || !pos || !freq || !x || !y) return DS_EINVAL;
    const int64_t width = (int64_t)n_heads * head_dim;
    if (width > 0x7fffffffLL || ldx < width || ldy < width || (x == y && ldx != ldy)) return DS_EINVAL;
    const size_t size = dtype_size(dtype);
    if ((uintptr_t)x % size || (uintptr_t)y % size || (uintptr_t)pos % 4 || (uintptr_t)freq % 8) return DS_EINVAL;
    if (rows == 0) return DS_OK;
    RopeArgs a = {};
    a.rows = rows; a.n_heads = n_heads; a.head_dim = head_dim; a.rot = rot_dim; a.inverse = inverse;
    a.pos = pos; a.freq = freq; a.amplitude = amplitude;
    a.x = x; a.y = y; a.ldx = ldx; a.ldy = ldy;
    hipStream_t st = (hipStream_t)hip_stream;
    const bool wide = rot_dim % 16 == 0 && head_dim % 8 == 0 && ldx % 8 == 0 && ldy % 8 == 0 && ((uintptr_t)x & 15) == 0 && ((uintptr_t)y & 15) == 0;
    if (dtype == DS_DTYPE_BF16) return wide ? rope_launch<bf16_t, 8>(a, interleaved, st) : rope_launch<bf16_t, 1>(a, interleaved, st);
    return wide ? rope_launch<float, 8>(a, interleaved, st) : rope_launch<float, 1>(a, interleaved, st);
}

// Host: freq[p] = base^(-2p / rot_dim), then scaled for contexts longer than the one trained on.
extern "C" ds_status ds_rope_freqs(int32_t rot_dim, double base, int32_t scaling, double factor, double context, double low_turns, double high_turns,
                                   double* freq) {
    if (rot_dim <= 0 || rot_dim % 2 || !(base > 0.0) || !std::isfinite(base) || !freq) return DS_EINVAL;
    if (scaling < DS_ROPE_PLAIN || scaling > DS_ROPE_BANDS) return DS_EINVAL;
    if (scaling != DS_ROPE_PLAIN && (!(factor > 0.0) || !std::isfinite(factor))) return DS_EINVAL;
    if (scaling == DS_ROPE_BASE && rot_dim <= 2) return DS_EINVAL;
    if (scaling == DS_ROPE_BANDS && (!(context > 0.0) || !(high_turns > low_turns) || !std::isfinite(context) || !std::isfinite(low_turns) || !std::isfinite(high_turns))) return DS_EINVAL;
    if (scaling == DS_ROPE_BASE) base *= std::pow(factor, (double)rot_dim / (rot_dim - 2));
    for (int p = 0; p < rot_dim / 2; ++p) {
        double f = std::pow(base, -2.0 * p / rot_dim);
        if (scaling == DS_ROPE_LINEAR) f /= factor;
        if (scaling == DS_ROPE_BANDS) {
            const double turns = context * f / 6.283185307179586;             // turns the pair makes over the context trained on
            double w = (turns - low_turns) / (high_turns - low_turns);
            w = w < 0.0 ? 0.0 : w > 1.0 ? 1.0 : w;
            f *= w + (1.0 - w) / factor;
        }
        freq[p] = f;
    }
    return DS_OK;
}

// Host: the position of every stream row within its sequence, -1 in padding rows.
extern "C" ds_status ds_layout_positions(const ds_layout* layout, int32_t which, int32_t* pos) {
    ds_layout_view v;
    if (!pos || (which != 0 && which != 1)) return DS_EINVAL;
    const ds_status r = ds_layout_get(layout, &v);
    if (r != DS_OK) return r;
    const int32_t rows = which ? v.total_rows_tgt : v.total_rows;
    const int32_t* row = which ? v.seq_row_tgt : v.seq_row;
    const int32_t* len = which ? v.seq_len_tgt : v.seq_len;
    if (!row || !len) return DS_ELAYOUT;
    for (int32_t i = 0; i < rows; ++i) pos[i] = -1;
    for (int32_t s = 0; s < v.n_seq; ++s)
        for (int32_t i = 0; i < len[s]; ++i) pos[row[s] + i] = i;
    return DS_OK;
}
