// Attention with a relative position bias for single tokens on a cache (one query to a sequence), in fp32 and in bf16 at the head sizes that the matrix-core kernels
// do not take (at those that they take they are as fast: their tiles come from memory just as well): bound by the bytes of the keys and values, which
// nothing is done with twice, so that there is nothing to stage and no matrix instruction to feed.
//
// A work-group has one query of one head and a share of the keys.  LANES lanes hold a row, 16 bytes each; a wavefront takes 64 / LANES keys a load and eight loads of
// keys and as many of values at once, all of them on their way before the first is looked at.  The lanes of a row add their products up among themselves (shifts of
// lanes); each group of lanes keeps a softmax of its own (maximum, sum, output) and they meet in LDS at the end, those of the work-groups in rel_join.
// fp32 arithmetic throughout.  Keys that a mask hides are not read.
//
// fp32, 16 heads, us (TB/s), before with the general kernels -> now: heads of 64, one sequence of 1 024 keys 10.1 -> 7.3, of 32 768 72 -> 52 (5.2), 16 of 1 019 40 -> 27 (4.9), 16 of 16 384
// 458 -> 400 (5.4); heads of 128, 13.3 -> 8.0, 208 -> 108 (5.0), 106 -> 49 (5.4), 1 579 -> 699 (6.1).
#include "rel_attention.hpp"
#include <initializer_list>

namespace {

constexpr int kLoads = 8, kMostTable = 2 * 1024 + 1;

template <class T> struct Piece;                        // 16 bytes of a row
template <> struct Piece<float> {
    static constexpr int N = 4;
    float4 v;
    __device__ __forceinline__ void load(const float* p) { v = *reinterpret_cast<const float4*>(p); }
    __device__ __forceinline__ void get(float (&f)[4]) const { f[0] = v.x; f[1] = v.y; f[2] = v.z; f[3] = v.w; }
};
template <> struct Piece<bf16_t> {
    static constexpr int N = 8;
    bf16x8_t v;
    __device__ __forceinline__ void load(const bf16_t* p) { v = *reinterpret_cast<const bf16x8_t*>(p); }
    __device__ __forceinline__ void get(float (&f)[8]) const {
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = (float)v[j];
    }
};

template <int CTRL> __device__ __forceinline__ float lanes(float v) {
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}
// the sum over LANES neighbouring lanes, in all of them
template <int LANES> __device__ __forceinline__ float sum_lanes(float v) {
    v += lanes<0xB1>(v);                                // quad_perm 1 0 3 2
    v += lanes<0x4E>(v);                                // quad_perm 2 3 0 1
    if constexpr (LANES >= 8) v += lanes<0x141>(v);     // row_half_mirror: the other four of eight
    if constexpr (LANES >= 16) v += lanes<0x140>(v);    // row_mirror: the other eight of sixteen
    if constexpr (LANES >= 32) v += __shfl_xor(v, 16, 64);
    return v;
}

template <class T, int LANES> __global__ __launch_bounds__(256) void rel_few_kernel(RelAttnArgs a) {
    constexpr int N = Piece<T>::N, KEYS = 64 / LANES, GROUPS = 4 * KEYS, WIDE = LANES * N;
    __shared__ float table[kMostTable];
    __shared__ __attribute__((aligned(16))) float part[GROUPS * WIDE];
    __shared__ float top[GROUPS], total[GROUPS];
    const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const int s = a.n_seq - 1 - blockIdx.z, h = blockIdx.y, qi = blockIdx.x / a.k_splits, split = blockIdx.x - qi * a.k_splits;
    const int ql = __builtin_amdgcn_readfirstlane(a.q_len[s]);
    if (qi >= ql) return;
    const int pos = __builtin_amdgcn_readfirstlane(rel_position(a, s)) + qi, hd = a.head_dim;
    const int seen = a.mask ? min(__builtin_amdgcn_readfirstlane(a.k_len[s]), max(0, pos + 1)) : __builtin_amdgcn_readfirstlane(a.k_len[s]);
    const long long run = a.k_splits == 1 ? seen : ((long long)seen + 64LL * a.k_splits - 1) / (64LL * a.k_splits) * 64;
    const int first = (int)min(run * split, (long long)seen), end = (int)min((long long)first + run, (long long)seen);
    const long long qrow = (long long)a.q_row[s] + qi;
    const int piece = lane % LANES, key = wave * KEYS * kLoads + lane / LANES;
    const bool in = piece * N < hd;                     // (a head of 24, 40, ...: the last lanes of a row have nothing)
    const int col = in ? piece * N : 0;
    const T* K = (const T*)a.k + (long long)a.k_row[s] * a.ldk + (long long)h * hd + col;
    const T* V = (const T*)a.v + (long long)a.k_row[s] * a.ldv + (long long)h * hd + col;
    Piece<T> k[kLoads], v[kLoads], qp;
    auto fetch = [&](int from) {
#pragma unroll
        for (int u = 0; u < kLoads; ++u) k[u].load(K + (long long)min(from + key + u * KEYS, end - 1) * a.ldk);
#pragma unroll
        for (int u = 0; u < kLoads; ++u) v[u].load(V + (long long)min(from + key + u * KEYS, end - 1) * a.ldv);
    };
    qp.load((const T*)a.q + qrow * a.ldq + (long long)h * hd + col);
    if (first < end) fetch(first);
    for (int i = t; i <= 2 * a.reach; i += 256) table[i] = rel_bias(a, h, i);
    __syncthreads();
    float q[N], o[N], m = -INFINITY, l = 0.f;
    const float c = a.scale * 1.4426950408889634f;      // (times the sum, as in the other kernels: times the query it might overflow where the score does not)
    qp.get(q);
#pragma unroll
    for (int j = 0; j < N; ++j) {
        q[j] = in ? q[j] : 0.f;
        o[j] = 0.f;
    }
    for (int from = first; from < end; from += GROUPS * kLoads) {
        float x[kLoads], up = m;
#pragma unroll
        for (int u = 0; u < kLoads; ++u) {
            float f[N];
            k[u].get(f);
            float dot = 0.f;
#pragma unroll
            for (int j = 0; j < N; ++j) dot = __builtin_fmaf(q[j], in ? f[j] : 0.f, dot);
            const int j = from + key + u * KEYS;
            x[u] = j < end ? __builtin_fmaf(sum_lanes<LANES>(dot), c, table[min(max(j - pos, -a.reach), a.reach) + a.reach]) : -INFINITY;
            up = fmaxf(up, x[u]);
        }
        const float use = up == -INFINITY ? 0.f : up, alpha = __builtin_amdgcn_exp2f(m - use);
        l *= alpha;
#pragma unroll
        for (int j = 0; j < N; ++j) o[j] *= alpha;
#pragma unroll
        for (int u = 0; u < kLoads; ++u) {
            float f[N];
            v[u].get(f);
            const float p = __builtin_amdgcn_exp2f(x[u] - use);
            l += p;
#pragma unroll
            for (int j = 0; j < N; ++j) o[j] = __builtin_fmaf(p, f[j], o[j]);
        }
        m = up;
        if (from + GROUPS * kLoads < end) fetch(from + GROUPS * kLoads);
    }
    const int group = wave * KEYS + lane / LANES;
    if (piece == 0) top[group] = m, total[group] = l;
#pragma unroll
    for (int j = 0; j < N; ++j) part[group * WIDE + piece * N + j] = o[j];
    __syncthreads();
    if (t >= hd) return;
    float all = -INFINITY, sum = 0.f, out = 0.f;
#pragma unroll
    for (int i = 0; i < GROUPS; ++i) all = fmaxf(all, top[i]);
    const float use = all == -INFINITY ? 0.f : all;
#pragma unroll
    for (int i = 0; i < GROUPS; ++i) {
        const float w = __builtin_amdgcn_exp2f(top[i] - use);
        sum = __builtin_fmaf(w, total[i], sum);
        out = __builtin_fmaf(w, part[i * WIDE + t], out);
    }
    if (a.k_splits > 1) {
        const RelPart to = rel_part(a, h, qrow, split);
        if (t == 0) to.stat[0] = all, to.stat[1] = sum;
        to.o[t] = out;
        return;
    }
    ((T*)a.o)[qrow * a.ldo + (long long)h * hd + t] = from_f32<T>(sum == 0.f ? 0.f : out / sum);
    if (t == 0) a.lse[(size_t)h * a.lse_stride + qrow] = (all + __builtin_amdgcn_logf(sum)) * 0.6931471805599453f;
}

}  // namespace

bool rel_few_supported(const RelAttnArgs& a) {
    const int n = a.dtype == DS_DTYPE_BF16 ? 8 : 4;
    if (a.max_q_len > 1 || a.ldq % n || a.ldk % n || a.ldv % n) return false;
    for (const void* p : {a.q, a.k, a.v})
        if ((uintptr_t)p & 15) return false;
    return true;
}

ds_status rel_fwd_few(const RelAttnArgs& a, hipStream_t st) {
    const dim3 grid(a.k_splits * a.max_q_len, a.n_heads, a.n_seq);
    const int lanes = rel_few_lanes(a.dtype, a.head_dim);
    if (a.dtype == DS_DTYPE_BF16) {
        auto kern = lanes == 4 ? rel_few_kernel<bf16_t, 4> : lanes == 8 ? rel_few_kernel<bf16_t, 8> : rel_few_kernel<bf16_t, 16>;
        hipLaunchKernelGGL(kern, grid, dim3(256), 0, st, a);
    } else {
        auto kern = lanes == 4 ? rel_few_kernel<float, 4> : lanes == 8 ? rel_few_kernel<float, 8> : lanes == 16 ? rel_few_kernel<float, 16> : rel_few_kernel<float, 32>;
        hipLaunchKernelGGL(kern, grid, dim3(256), 0, st, a);
    }
    DS_LAUNCH_CHECK();
    return a.k_splits == 1 ? DS_OK : rel_join(a, st);
}
