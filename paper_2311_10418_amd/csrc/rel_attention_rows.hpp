// Attention with a relative position bias under a causal mask one row at a time, reading exactly the rows of the other side that belong together: what the
// general kernels fall back to where sums are not finite.  A wavefront per row, lane i with the features i and i + 64 (of at most 128).
#pragma once
#include "rel_attention.hpp"

namespace {

struct RelPair { float a, b; };
template <class T> __device__ __forceinline__ RelPair rel_pair(const void* base, long long row, long long ld, int h, int hd, int lane) {
    const T* p = (const T*)base + row * ld + (long long)h * hd;
    return {lane < hd ? to_f32(p[lane]) : 0.f, lane + 64 < hd ? to_f32(p[lane + 64]) : 0.f};
}
template <class T> __device__ __forceinline__ void rel_put(T* p, int hd, int lane, RelPair v) {
    if (lane < hd) p[lane] = from_f32<T>(v.a);
    if (lane + 64 < hd) p[lane + 64] = from_f32<T>(v.b);
}
__device__ __forceinline__ float rel_dot(RelPair x, RelPair y) { return wave_sum(__builtin_fmaf(x.a, y.a, x.b * y.b)); }
__device__ __forceinline__ RelPair rel_axpy(float w, RelPair x, RelPair y) { return {__builtin_fmaf(w, x.a, y.a), __builtin_fmaf(w, x.b, y.b)}; }
// whether a row's sums are NaN throughout, which nothing changes any more
__device__ __forceinline__ bool rel_all_nan(RelPair v, int hd, int lane) {
    return __builtin_amdgcn_ballot_w64((lane < hd && v.a == v.a) || (lane + 64 < hd && v.b == v.b)) == 0;
}

// sum of exp2(S - e) V over keys first .. first + n - 1 that a query at position p sees
template <class T> __device__ __forceinline__ RelPair rel_fwd_row(const RelAttnArgs& a, int s, int h, int qi, int p, int first, int n, float e, int lane) {
    const int hd = a.head_dim;
    const long long kr0 = a.k_row[s];
    const RelPair q = rel_pair<T>(a.q, (long long)a.q_row[s] + qi, a.ldq, h, hd, lane);
    const float c = a.scale * 1.4426950408889634f;
    RelPair o = {0.f, 0.f};
    for (int j = first; j < min(first + n, p + 1); ++j) {
        const float x = __builtin_fmaf(rel_dot(q, rel_pair<T>(a.k, kr0 + j, a.ldk, h, hd, lane)), c, rel_bias(a, h, j - p + a.reach));
        o = rel_axpy(__builtin_amdgcn_exp2f(x - e), rel_pair<T>(a.v, kr0 + j, a.ldv, h, hd, lane), o);
        if (j % 16 == 15 && rel_all_nan(o, hd, lane)) break;
    }
    return o;
}
// dQ of query qi, and its dS by distance into sums[distance + reach + pad]
template <class T>
__device__ __forceinline__ void rel_dq_row(const RelAttnArgs& a, int s, int h, int qi, int p, int kl, float e, float d, float* sums, int lane) {
    const int hd = a.head_dim;
    const long long qr = (long long)a.q_row[s] + qi, kr0 = a.k_row[s];
    const RelPair q = rel_pair<T>(a.q, qr, a.ldq, h, hd, lane), g = rel_pair<T>(a.d_o, qr, a.ldo, h, hd, lane);
    const float c = a.scale * 1.4426950408889634f;
    RelPair o = {0.f, 0.f};
    for (int j = 0; j < min(kl, p + 1); ++j) {
        const RelPair k = rel_pair<T>(a.k, kr0 + j, a.ldk, h, hd, lane);
        const int i = min(max(j - p + a.reach, 0), 2 * a.reach);
        const float x = __builtin_fmaf(rel_dot(q, k), c, rel_bias(a, h, i));
        const float w = __builtin_amdgcn_exp2f(x - e) * (rel_dot(g, rel_pair<T>(a.v, kr0 + j, a.ldv, h, hd, lane)) - d);
        o = rel_axpy(w, k, o);
        if (lane == 0) sums[i] += w;
    }
    rel_put<T>((T*)a.dq + qr * a.ldq + (long long)h * hd, hd, lane, {o.a * a.scale, o.b * a.scale});
}
// dK and dV of key kj
template <class T> __device__ __forceinline__ void rel_dkv_row(const RelAttnArgs& a, int s, int h, int kj, int pos, int ql, int lane) {
    const int hd = a.head_dim;
    const long long kr = (long long)a.k_row[s] + kj, qr0 = a.q_row[s];
    const RelPair k = rel_pair<T>(a.k, kr, a.ldk, h, hd, lane), v = rel_pair<T>(a.v, kr, a.ldv, h, hd, lane);
    const float c = a.scale * 1.4426950408889634f;
    RelPair dk = {0.f, 0.f}, dv = {0.f, 0.f};
    for (int i = max(kj - pos, 0); i < ql; ++i) {
        const RelPair q = rel_pair<T>(a.q, qr0 + i, a.ldq, h, hd, lane), g = rel_pair<T>(a.d_o, qr0 + i, a.ldo, h, hd, lane);
        const size_t at = (size_t)h * a.q_total_rows + qr0 + i;
        const float x = __builtin_fmaf(rel_dot(q, k), c, rel_bias(a, h, kj - pos - i + a.reach));
        const float w = __builtin_amdgcn_exp2f(x - rel_lse2(a.lse[at]));
        dv = rel_axpy(w, g, dv);
        dk = rel_axpy(w * (rel_dot(g, v) - a.d[at]), q, dk);
        if (i % 16 == 15 && rel_all_nan(dk, hd, lane) && rel_all_nan(dv, hd, lane)) break;
    }
    rel_put<T>((T*)a.dk + kr * a.ldk + (long long)h * hd, hd, lane, {dk.a * a.scale, dk.b * a.scale});
    rel_put<T>((T*)a.dv + kr * a.ldv + (long long)h * hd, hd, lane, dv);
}

}  // namespace
