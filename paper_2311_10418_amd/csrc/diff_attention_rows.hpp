// Differential attention under a causal mask one row at a time, reading exactly the rows of the other side that belong together: what the general
// kernels fall back to where sums are not finite.  A wavefront per row, lane i with the features i and i + 64 (of at most 128).
#pragma once
#include "diff_attention.hpp"

namespace {

constexpr float kLog2eRows = 1.4426950408889634f;

struct Pair { float a, b; };
template <class T> __device__ __forceinline__ Pair pair_of(const void* base, long long row, long long ld, int h, int hd, int lane) {
    const T* p = (const T*)base + row * ld + (long long)h * hd;
    return {lane < hd ? to_f32(p[lane]) : 0.f, lane + 64 < hd ? to_f32(p[lane + 64]) : 0.f};
}
template <class T> __device__ __forceinline__ void put_pair(void* base, long long row, long long ld, int h, int hd, int lane, Pair v) {
    T* p = (T*)base + row * ld + (long long)h * hd;
    if (lane < hd) p[lane] = from_f32<T>(v.a);
    if (lane + 64 < hd) p[lane + 64] = from_f32<T>(v.b);
}
__device__ __forceinline__ float dot_pairs(Pair x, Pair y) { return wave_sum(__builtin_fmaf(x.a, y.a, x.b * y.b)); }
// probabilities of both maps from a query's and a key's features and the log-sum-exps (exp2 domain); half a head is at most 64 features
__device__ __forceinline__ Pair both_maps(const DiffAttnArgs& a, Pair q, Pair k, float e1, float e2, int lane) {
    const float c = a.scale * kLog2eRows, both = q.a * k.a;
    const bool first = lane < a.head_dim / 2;
    return {__builtin_amdgcn_exp2f(__builtin_fmaf(wave_sum(first ? both : 0.f), c, -e1)),
            __builtin_amdgcn_exp2f(__builtin_fmaf(wave_sum(__builtin_fmaf(q.b, k.b, first ? 0.f : both)), c, -e2))};
}

// Whether a row's sums are NaN throughout, which nothing changes any more: asked for every 16 rows, so that a sequence of NaN takes no longer than another.
__device__ __forceinline__ bool all_nan(Pair v, int hd, int lane) {
    return __builtin_amdgcn_ballot_w64((lane < hd && v.a == v.a) || (lane + 64 < hd && v.b == v.b)) == 0;
}

// outputs of query qi
template <class T> __device__ __forceinline__ void diff_fwd_row(const DiffAttnArgs& a, int s, int h, int qi, float e1, float e2, int lane) {
    const int hd = a.head_dim, nk = min(a.k_len[s], qi + 1);
    const long long qr = (long long)a.q_row[s] + qi, kr0 = a.k_row[s];
    const Pair q = pair_of<T>(a.q, qr, a.ldq, h, hd, lane);
    Pair o1 = {0.f, 0.f}, o2 = {0.f, 0.f};
    for (int j = 0; j < nk; ++j) {
        const Pair p = both_maps(a, q, pair_of<T>(a.k, kr0 + j, a.ldk, h, hd, lane), e1, e2, lane), v = pair_of<T>(a.v, kr0 + j, a.ldv, h, hd, lane);
        o1 = {__builtin_fmaf(p.a, v.a, o1.a), __builtin_fmaf(p.a, v.b, o1.b)};
        o2 = {__builtin_fmaf(p.b, v.a, o2.a), __builtin_fmaf(p.b, v.b, o2.b)};
        if (j % 16 == 15 && all_nan(o1, hd, lane) && all_nan(o2, hd, lane)) break;
    }
    const float lam = a.lambda[h];
    put_pair<T>(a.o, qr, a.ldo, h, hd, lane, {o1.a - o2.a * lam, o1.b - o2.b * lam});
    if (a.o2) put_pair<T>(a.o2, qr, a.ldo, h, hd, lane, o2);
}

// gradient of query qi; returns the sum of P_2 G
template <class T> __device__ __forceinline__ float diff_dq_row(const DiffAttnArgs& a, int s, int h, int qi, float e1, float e2, float d1, float d2, int lane) {
    const int hd = a.head_dim, nk = min(a.k_len[s], qi + 1);
    const long long qr = (long long)a.q_row[s] + qi, kr0 = a.k_row[s];
    const Pair q = pair_of<T>(a.q, qr, a.ldq, h, hd, lane), d_o = pair_of<T>(a.d_o, qr, a.ldo, h, hd, lane);
    const float lam = a.lambda[h];
    const bool first = lane < hd / 2;
    Pair g = {0.f, 0.f};
    float lam_sum = 0.f;
    for (int j = 0; j < nk; ++j) {
        const Pair k = pair_of<T>(a.k, kr0 + j, a.ldk, h, hd, lane), p = both_maps(a, q, k, e1, e2, lane);
        const float dp = dot_pairs(d_o, pair_of<T>(a.v, kr0 + j, a.ldv, h, hd, lane)), ds1 = p.a * (dp - d1), ds2 = p.b * (d2 - dp) * lam;
        g = {__builtin_fmaf(first ? ds1 : ds2, k.a, g.a), __builtin_fmaf(ds2, k.b, g.b)};
        lam_sum = __builtin_fmaf(p.b, dp, lam_sum);
        if (j % 16 == 15 && lam_sum != lam_sum && all_nan(g, hd, lane)) break;
    }
    put_pair<T>(a.dq, qr, a.ldq, h, hd, lane, {g.a * a.scale, g.b * a.scale});
    return lam_sum;
}

// gradients of key kj
template <class T> __device__ __forceinline__ void diff_dkv_row(const DiffAttnArgs& a, int s, int h, int kj, int lane) {
    const int hd = a.head_dim, ql = a.q_len[s];
    const long long kr = (long long)a.k_row[s] + kj, qr0 = a.q_row[s];
    const Pair k = pair_of<T>(a.k, kr, a.ldk, h, hd, lane), v = pair_of<T>(a.v, kr, a.ldv, h, hd, lane);
    const float lam = a.lambda[h];
    const bool first = lane < hd / 2;
    Pair gk = {0.f, 0.f}, gv = {0.f, 0.f};
    for (int i = kj; i < ql; ++i) {
        const long long qr = qr0 + i;
        const Pair q = pair_of<T>(a.q, qr, a.ldq, h, hd, lane), d_o = pair_of<T>(a.d_o, qr, a.ldo, h, hd, lane);
        const Pair p = both_maps(a, q, k, a.lse[(size_t)(2 * h) * a.lse_stride + qr] * kLog2eRows, a.lse[(size_t)(2 * h + 1) * a.lse_stride + qr] * kLog2eRows, lane);
        const float dp = dot_pairs(d_o, v), d1 = a.d1[(size_t)h * a.q_total_rows + qr], d2 = a.d2[(size_t)h * a.q_total_rows + qr];
        const float ds1 = p.a * (dp - d1), p2 = lam * p.b, ds2 = p2 * (d2 - dp), both = p.a - p2;
        gk = {__builtin_fmaf(first ? ds1 : ds2, q.a, gk.a), __builtin_fmaf(ds2, q.b, gk.b)};
        gv = {__builtin_fmaf(both, d_o.a, gv.a), __builtin_fmaf(both, d_o.b, gv.b)};
        if ((i - kj) % 16 == 15 && all_nan(gk, hd, lane) && all_nan(gv, hd, lane)) break;
    }
    put_pair<T>(a.dk, kr, a.ldk, h, hd, lane, {gk.a * a.scale, gk.b * a.scale});
    put_pair<T>(a.dv, kr, a.ldv, h, hd, lane, gv);
}

}  // namespace
