// Differential attention for every type, head size, stride and alignment the entry points take: v_mfma_f32_16x16x4_f32 on fp32 values
// (bf16 operands are widened as their tiles go to LDS), so that products, probabilities and sums are fp32 throughout.
//
// A wavefront owns 16 "column" items (queries in forward and dQ, keys in dK/dV) and computes transposed score blocks of both maps: 16
// rows of the other side x its 16 columns, lane = (column lane % 16, rows 4 g + e with g = lane / 16, e = 0..3).  Per column values
// are per-lane scalars, and register e of a block is, as it stands, the B operand of the second product for the rows {4 g + e}.
// Tiles of the other side are kept in LDS row by row, every half head padded with zeros to HH columns (a multiple of 16), V and dO too:
// the contraction over features does not see the order of the columns, and outputs go back through the same mapping.
//
// Causal masks and values that are not finite.  A score that a column does not see is replaced whatever it is; but the second products run over whole
// blocks of rows, probability 0 where a column does not see one, and 0 x Inf is NaN (dP of a hidden row may overflow, too).  A wavefront whose sums are not
// finite in the end therefore takes its columns one by one (diff_attention_rows.hpp), so that a row is affected by the rows it sees and by no others.
// (Looking the rows over as their tiles go to LDS took 2 to 7 % of the kernels' time; this takes about 1 %.)
//
// Bound by issue: the matrix pipe is busy 60 % of the SIMD cycles and vector instructions, more than two for each matrix instruction, take the rest.
// Measured in fp32: 16 heads of 64, 31 sequences of 366 to 523, unmasked, forward 398 us, backward 967 (93 and 90 TFLOP/s
// of the products they form, where a large product of matrices reaches 154); 16 heads of 128, 8 of 1 639 to 2 048, causal, 1 791 and 6 036 (92 and 63: 32-row
// tiles backward); 4 heads of 64, 23 sequences of 88 to 177, causal, backward 42.
#include "diff_attention.hpp"
#include "diff_attention_rows.hpp"
#include "gemm.hpp"
#include <type_traits>

namespace {

constexpr float kLog2eG = 1.4426950408889634f;
constexpr float kLn2G = 0.6931471805599453f;

__device__ __forceinline__ f32x4_t mfma4(float a, float b, f32x4_t c) { return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4_t zero4() { f32x4_t z = {0.f, 0.f, 0.f, 0.f}; return z; }

template <class T> __device__ __forceinline__ float4 load4(const T* p, bool vec);
template <> __device__ __forceinline__ float4 load4<float>(const float* p, bool vec) {
    return vec ? *reinterpret_cast<const float4*>(p) : make_float4(p[0], p[1], p[2], p[3]);
}
template <> __device__ __forceinline__ float4 load4<bf16_t>(const bf16_t* p, bool vec) {
    if (vec) {
        const bf16x4_t v = *reinterpret_cast<const bf16x4_t*>(p);
        return make_float4((float)v[0], (float)v[1], (float)v[2], (float)v[3]);
    }
    return make_float4((float)p[0], (float)p[1], (float)p[2], (float)p[3]);
}
__device__ __forceinline__ void store4(float* p, const f32x4_t& v, bool vec) {
    if (vec) *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
    else
        for (int j = 0; j < 4; ++j) p[j] = v[j];
}
__device__ __forceinline__ void store4(bf16_t* p, const f32x4_t& v, bool vec) {
    if (vec) {
        bf16x4_t b;
#pragma unroll
        for (int j = 0; j < 4; ++j) b[j] = (bf16_t)v[j];
        *reinterpret_cast<bf16x4_t*>(p) = b;
    } else
        for (int j = 0; j < 4; ++j) p[j] = (bf16_t)v[j];
}

template <class T, int HH, int THREADS> struct Tile {
    static constexpr int ROWS = HH <= 48 ? 64 : 32, HD = 2 * HH, LD = HD + 4, NV = ROWS * HD / 4 / THREADS;
    static constexpr int FLOATS = ROWS * LD;
    float4 v[NV];
    __device__ __forceinline__ void load(const T* src, long long ld, int r0, int n_rows, int half, bool vec) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int u = threadIdx.x + THREADS * i, r = r0 + u / (HD / 4), d = (u % (HD / 4)) * 4, m = d >= HH;
            v[i] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (r < n_rows && d - m * HH < half) v[i] = load4<T>(src + (long long)r * ld + m * half + (d - m * HH), vec);
        }
    }
    __device__ __forceinline__ void store(float* tile) const {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int u = threadIdx.x + THREADS * i;
            *reinterpret_cast<float4*>(tile + (u / (HD / 4)) * LD + (u % (HD / 4)) * 4) = v[i];
        }
    }
};

// this lane's column item: features 16 s + 4 g .. + 3, padded like the tiles
template <class T, int HH>
__device__ __forceinline__ void load_column(const T* row, int half, int g, bool vec, float4 (&f)[HH / 8]) {
#pragma unroll
    for (int s = 0; s < HH / 8; ++s) {
        const int m = s >= HH / 16, d = 16 * s + 4 * g - m * HH;
        f[s] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (d < half) f[s] = load4<T>(row + m * half + d, vec);
    }
}
template <class T, int HH>
__device__ __forceinline__ void store_column(const f32x4_t (&acc)[HH / 8], float mul, T* row, int half, int g, bool vec) {
#pragma unroll
    for (int s = 0; s < HH / 8; ++s) {
        const int m = s >= HH / 16, d = 16 * s + 4 * g - m * HH;
        if (d < half) store4(row + m * half + d, acc[s] * mul, vec);
    }
}

// rows rb .. rb+15 of a tile times this lane's column item, contracted over the feature steps S0 .. S1-1
template <int HH, int S0, int S1>
__device__ __forceinline__ f32x4_t first_product(const float* tile, int rb, int lane, const float4 (&f)[HH / 8]) {
    const float* p = tile + (rb + (lane & 15)) * (2 * HH + 4) + 4 * (lane >> 4);
    f32x4_t acc = zero4();
#pragma unroll
    for (int s = S0; s < S1; ++s) {
        const float4 x = *reinterpret_cast<const float4*>(p + 16 * s);
        acc = mfma4(x.x, f[s].x, acc);
        acc = mfma4(x.y, f[s].y, acc);
        acc = mfma4(x.z, f[s].z, acc);
        acc = mfma4(x.w, f[s].w, acc);
    }
    return acc;
}
// out^T[feature step S0 .. S1-1][column] += tile[rows rb .. rb+15]^T * w
template <int HH, int S0, int S1>
__device__ __forceinline__ void second_product(const float* tile, int rb, int lane, const f32x4_t& w, f32x4_t (&out)[HH / 8]) {
    const float* p = tile + (rb + 4 * (lane >> 4)) * (2 * HH + 4) + (lane & 15);
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int s = S0; s < S1; ++s) out[s] = mfma4(p[e * (2 * HH + 4) + 16 * s], w[e], out[s]);
}

template <int N> __device__ __forceinline__ bool any_not_finite(const f32x4_t (&acc)[N]) {       // of the wavefront's sums
    float nothing = 0.f;                                // 0, or NaN
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) nothing = __builtin_fmaf(acc[i][j], 0.f, nothing);
    return __builtin_amdgcn_ballot_w64(nothing != 0.f) != 0;
}

__device__ __forceinline__ float groups_max(float v) { v = fmaxf(v, __shfl_xor(v, 16, 64)); return fmaxf(v, __shfl_xor(v, 32, 64)); }
__device__ __forceinline__ float groups_sum(float v) { v += __shfl_xor(v, 16, 64); return v + __shfl_xor(v, 32, 64); }

// A work-group's COLS columns: sequence, head, first column (negative: nothing to do).  Sequences last to first: a plan lists them by
// ascending length, and the longest chains of tiles should start first.
struct ColumnBlock { int s, h, first; };
template <int COLS = 64> __device__ __forceinline__ ColumnBlock column_block(const AttnArgs& a, const int32_t* len, bool last_first, int z) {
    ColumnBlock c = {a.n_seq - 1 - z, (int)blockIdx.y, -1};
    const int n = (len[c.s] + COLS - 1) / COLS, b = blockIdx.x;
    if (b < n) c.first = COLS * (last_first ? n - 1 - b : b);
    return c;
}
// an odd number of blocks per grid row: work-groups go to the eight XCDs in turn, and the longest of every sequence should not meet on one
dim3 column_grid(const AttnArgs& a, int max_len, int cols = 64) { return dim3((max_len / cols + (max_len % cols != 0)) | 1, a.n_heads, a.n_seq); }

// ---------------------------------------------------------------- forward
template <class T, int HH>
__global__ __launch_bounds__(256, HH <= 32 ? 3 : 2) void diff_fwd_kernel(DiffAttnArgs a) {
    typedef Tile<T, HH, 256> Tl;
    constexpr int KT = Tl::ROWS, NB = KT / 16, NS = HH / 8;
    __shared__ __attribute__((aligned(16))) float sK[Tl::FLOATS];
    __shared__ __attribute__((aligned(16))) float sV[Tl::FLOATS];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4;
    ColumnBlock cb = column_block(a, a.q_len, a.mask != 0, blockIdx.z);
    const int split = a.k_splits > 1 ? blockIdx.x : 0;                 // (one block of queries then)
    if (a.k_splits > 1) cb.first = a.q_len[cb.s] > 0 ? 0 : -1;
    if (cb.first < 0) return;
    const int s = cb.s, h = cb.h, q0 = cb.first, ql = a.q_len[s], hd = a.head_dim, half = hd / 2;
    const KeyRange range = split_keys(a, a.k_len[s], split);
    const int kl = range.count;
    const bool vec = a.vec;
    const long long qrow0 = a.q_row[s], krow0 = (long long)a.k_row[s] + range.first;
    const T* K = (const T*)a.k + krow0 * a.ldk + (long long)h * hd;
    const T* V = (const T*)a.v + krow0 * a.ldv + (long long)h * hd;
    const int qw0 = q0 + wave * 16, qi = qw0 + (lane & 15), qi_c = qi < ql ? qi : ql - 1;
    float4 qf[NS];
    load_column<T, HH>((const T*)a.q + (qrow0 + qi_c) * a.ldq + (long long)h * hd, half, g, vec, qf);
    f32x4_t o1[NS], o2[NS];
#pragma unroll
    for (int i = 0; i < NS; ++i) { o1[i] = zero4(); o2[i] = zero4(); }
    const float c = a.scale * kLog2eG;
    float m1 = -INFINITY, m2 = -INFINITY, l1 = 0.f, l2 = 0.f;          // running maxima (exp2 domain), this lane's part of the sums
    const int kv_end = a.mask ? min(kl, q0 + 64) : kl;
    const int wave_last = a.mask ? min(kl - 1, qw0 + 15) : kl - 1;     // last key this wavefront can see
    Tl tk, tv;
    if (kv_end > 0) {
        tk.load(K, a.ldk, 0, kl, half, vec);
        tv.load(V, a.ldv, 0, kl, half, vec);
    }
    for (int k0 = 0; k0 < kv_end; k0 += KT) {
        __syncthreads();                                               // the previous tile has been read by everybody
        tk.store(sK);
        tv.store(sV);
        __syncthreads();
        if (k0 + KT < kv_end) {
            tk.load(K, a.ldk, k0 + KT, kl, half, vec);
            tv.load(V, a.ldv, k0 + KT, kl, half, vec);
        }
        if (k0 > wave_last || qw0 >= ql) continue;
        // one map after the other, strictly so above head size 32, where the scores of both would take the registers of the second or third wavefront
        // of a SIMD (16 heads of 64, 31 sequences of about 445 in fp32: 473 -> 430 us; 16 heads of 128, 8 of about 1 820, causal: 3 184 -> 1 940)
        auto map = [&](auto first, float& m, float& l, f32x4_t (&o)[NS]) {
            constexpr int S0 = decltype(first)::value, S1 = S0 + NS / 2;
            f32x4_t p[NB];
            float x = -INFINITY;
#pragma unroll
            for (int kt = 0; kt < NB; ++kt) {
                p[kt] = first_product<HH, S0, S1>(sK, 16 * kt, lane, qf);
                const int kb = k0 + 16 * kt;
                if (kb + 16 > kl || (a.mask && kb + 15 > qw0))         // (a branch: most blocks need no mask)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int key = kb + 4 * g + e;
                        if (key >= kl || (a.mask && key > qi)) p[kt][e] = -INFINITY;
                    }
#pragma unroll
                for (int e = 0; e < 4; ++e) x = fmaxf(x, p[kt][e]);
            }
            const float m_new = fmaxf(m, groups_max(x) * c), m_use = m_new == -INFINITY ? 0.f : m_new;
            const float alpha = __builtin_amdgcn_exp2f(m - m_use);
            float rs = 0.f;
#pragma unroll
            for (int kt = 0; kt < NB; ++kt)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    p[kt][e] = __builtin_amdgcn_exp2f(__builtin_fmaf(p[kt][e], c, -m_use));
                    rs += p[kt][e];
                }
            l = l * alpha + rs;
            m = m_new;
#pragma unroll
            for (int i = 0; i < NS; ++i) o[i] *= alpha;
#pragma unroll
            for (int kt = 0; kt < NB; ++kt) second_product<HH, 0, NS>(sV, 16 * kt, lane, p[kt], o);
        };
        map(std::integral_constant<int, 0>{}, m1, l1, o1);
        if constexpr (HH >= 32) __builtin_amdgcn_sched_barrier(0);
        map(std::integral_constant<int, NS / 2>{}, m2, l2, o2);
    }
    l1 = groups_sum(l1);
    l2 = groups_sum(l2);
    if (a.mask && (any_not_finite(o1) || any_not_finite(o2))) {
        const float e1 = m1 + __builtin_amdgcn_logf(l1), e2 = m2 + __builtin_amdgcn_logf(l2);
        for (int i = 0; i < min(16, ql - qw0); ++i) diff_fwd_row<T>(a, s, h, qw0 + i, __shfl(e1, i, 64), __shfl(e2, i, 64), lane);
        if (g == 0 && qi < ql) {
            a.lse[(size_t)(2 * h) * a.lse_stride + qrow0 + qi] = e1 * kLn2G;
            a.lse[(size_t)(2 * h + 1) * a.lse_stride + qrow0 + qi] = e2 * kLn2G;
        }
        return;
    }
    if (qi >= ql) return;
    const long long row = qrow0 + qi;
    if (a.k_splits > 1) {
        const SplitPart to = split_part(a, h, row, split);
        if (g == 0) *reinterpret_cast<float4*>(to.stat) = make_float4(m1, l1, m2, l2);
        store_column<float, HH>(o1, 1.0f, to.o[0], half, g, true);
        store_column<float, HH>(o2, 1.0f, to.o[1], half, g, true);
        return;
    }
    const float lam = a.lambda[h], r1 = kl > 0 ? 1.0f / l1 : 0.f, r2 = kl > 0 ? 1.0f / l2 : 0.f;      // (no keys: zeros)
#pragma unroll
    for (int i = 0; i < NS; ++i) {
        o2[i] *= r2;
        o1[i] = o1[i] * r1 - o2[i] * lam;
    }
    store_column<T, HH>(o1, 1.0f, (T*)a.o + row * a.ldo + (long long)h * hd, half, g, vec);
    if (a.o2) store_column<T, HH>(o2, 1.0f, (T*)a.o2 + row * a.ldo + (long long)h * hd, half, g, vec);
    if (g == 0) {
        a.lse[(size_t)(2 * h) * a.lse_stride + row] = (m1 + __builtin_amdgcn_logf(l1)) * kLn2G;
        a.lse[(size_t)(2 * h + 1) * a.lse_stride + row] = (m2 + __builtin_amdgcn_logf(l2)) * kLn2G;
    }
}

// What the work-groups that shared a head's keys found, put together: a wavefront per query, lane i with the statistics of work-group i, then four
// columns of one of the outputs per lane.  A work-group without keys has sum 0, and its maximum does not count.  A chain of two trips to memory and no
// more for up to kAtOnce work-groups, whose outputs are on their way before the statistics are there.
template <class T> __global__ __launch_bounds__(256) void diff_join_kernel(DiffAttnArgs a) {
    constexpr int kAtOnce = 16;
    const int lane = threadIdx.x & 63, q = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = blockIdx.y, s = blockIdx.z;
    if (q >= a.q_len[s]) return;
    const long long row = (long long)a.q_row[s] + q;
    const int hd = a.head_dim, n = a.k_splits, quarter = hd / 4;
    const size_t step = 2 * hd + 4;
    const SplitPart p = split_part(a, h, row, 0);
    const int m = lane >= quarter, col = 4 * (lane - m * quarter);     // this lane's output and columns
    const bool on = lane < 2 * quarter;
    const float* from = p.o[0] + 4 * (on ? lane : 0);
    auto load = [&](int i) { return *reinterpret_cast<const f32x4_t*>(from + min(i, n - 1) * step); };
    f32x4_t v[kAtOnce];
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) v[i] = load(i);
    const f32x4_t st = lane < n ? *reinterpret_cast<const f32x4_t*>(p.stat + lane * step) : zero4();
    float w[2], r[2], lse[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const float l = st[2 * i + 1], top = l == 0.f ? -INFINITY : st[2 * i];
        float up = top;
#pragma unroll
        for (int j = 1; j < 64; j *= 2) up = fmaxf(up, __shfl_xor(up, j, 64));
        w[i] = l == 0.f ? 0.f : __builtin_amdgcn_exp2f(top - up);
        float sum = w[i] * l;
#pragma unroll
        for (int j = 1; j < 64; j *= 2) sum += __shfl_xor(sum, j, 64);
        r[i] = sum == 0.f ? 0.f : 1.0f / sum;
        lse[i] = (up + __builtin_amdgcn_logf(sum)) * kLn2G;
    }
    auto weight = [&](int i) {                          // (lanes n and above hold 0)
        const float w1 = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, w[0]), i));
        const float w2 = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, w[1]), i));
        return m ? w2 : w1;
    };
    f32x4_t o = zero4();
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i)
        if (i < n) o += v[i] * weight(i);
#pragma unroll 8
    for (int i = kAtOnce; i < n; ++i) o += load(i) * weight(i);
    o *= r[m];
    const float lam = a.lambda[h];
    f32x4_t other;
#pragma unroll
    for (int j = 0; j < 4; ++j) other[j] = __shfl(o[j], lane + quarter, 64);
    if (m == 0) o -= other * lam;
    T* to = (T*)(m ? a.o2 : a.o);
    if (on && to) store4(to + row * a.ldo + (long long)h * hd + col, o, a.vec);
    if (lane < 2) a.lse[(size_t)(2 * h + lane) * a.lse_stride + row] = lane ? lse[1] : lse[0];
}

// ---------------------------------------------------------------- backward: dQ, D_1, D_2, the parts of dlambda
// Eight wavefronts, SPLITS = 2 or 4 for each 16 columns: they take every SPLITS-th 16 rows of a tile, and what they have is added up in the end, by
// halves.  A work-group has 64 columns, or 32 where that makes too few of them for the compute units (see narrow()).
template <int COLS> struct Share {
    static constexpr int GROUPS = COLS / 16, SPLITS = 8 / GROUPS;
};
template <int COLS, int N> __device__ __forceinline__ void join_shares(float* lds, int split, int t, f32x4_t (&acc)[N]) {
#pragma unroll
    for (int half = Share<COLS>::SPLITS / 2; half >= 1; half /= 2) {
        f32x4_t* p = reinterpret_cast<f32x4_t*>(lds) + (t - (split >= half ? half : 0) * (4 * COLS));
        __syncthreads();                                // what the memory held before has been read
        if (split >= half && split < 2 * half)
#pragma unroll
            for (int i = 0; i < N; ++i) p[256 * i] = acc[i];
        __syncthreads();
        if (split < half)
#pragma unroll
            for (int i = 0; i < N; ++i) acc[i] += p[256 * i];
    }
}

template <class T, int HH, int COLS>
__global__ __launch_bounds__(512, HH <= 32 ? 4 : 2) void diff_bwd_dq_kernel(DiffAttnArgs a) {
    typedef Tile<T, HH, 512> Tl;
    constexpr int KT = Tl::ROWS, NS = HH / 8;
    __shared__ __attribute__((aligned(16))) float lds[2 * Tl::FLOATS];
    static_assert(2 * Tl::FLOATS >= 256 * 4 * NS, "the sums of four wavefronts");
    float *const sK = lds, *const sV = lds + Tl::FLOATS;
    const int t = threadIdx.x, lane = t & 63, wave8 = __builtin_amdgcn_readfirstlane(t >> 6), g = lane >> 4;
    const int wave = wave8 % Share<COLS>::GROUPS, split = wave8 / Share<COLS>::GROUPS;
    const ColumnBlock cb = column_block<COLS>(a, a.q_len, a.mask != 0, blockIdx.z);
    if (cb.first < 0) return;
    const int s = cb.s, h = cb.h, q0 = cb.first, ql = a.q_len[s], kl = a.k_len[s], hd = a.head_dim, half = hd / 2;
    const bool vec = a.vec;
    const long long qrow0 = a.q_row[s], krow0 = a.k_row[s];
    const T* K = (const T*)a.k + krow0 * a.ldk + (long long)h * hd;
    const T* V = (const T*)a.v + krow0 * a.ldv + (long long)h * hd;
    const int qw0 = q0 + wave * 16, qi = qw0 + (lane & 15), qi_c = qi < ql ? qi : ql - 1;
    const long long row = qrow0 + qi_c;
    const float lam = a.lambda[h];
    float4 qf[NS], dof[NS];
    load_column<T, HH>((const T*)a.q + row * a.ldq + (long long)h * hd, half, g, vec, qf);
    load_column<T, HH>((const T*)a.d_o + row * a.ldo + (long long)h * hd, half, g, vec, dof);
    float d1 = 0.f, d2 = 0.f;
    {
        float4 f[NS];
        load_column<T, HH>((const T*)a.o + row * a.ldo + (long long)h * hd, half, g, vec, f);
#pragma unroll
        for (int i = 0; i < NS; ++i) d1 += (f[i].x * dof[i].x + f[i].y * dof[i].y) + (f[i].z * dof[i].z + f[i].w * dof[i].w);
        load_column<T, HH>((const T*)a.o2 + row * a.ldo + (long long)h * hd, half, g, vec, f);
#pragma unroll
        for (int i = 0; i < NS; ++i) d2 += (f[i].x * dof[i].x + f[i].y * dof[i].y) + (f[i].z * dof[i].z + f[i].w * dof[i].w);
        d2 = groups_sum(d2);
        d1 = groups_sum(d1) + lam * d2;
        if (g == 0 && qi < ql && split == 0) {
            a.d1[(size_t)h * a.q_total_rows + row] = d1;
            a.d2[(size_t)h * a.q_total_rows + row] = d2;
        }
    }
    const float e1 = a.lse[(size_t)(2 * h) * a.lse_stride + row] * kLog2eG, e2 = a.lse[(size_t)(2 * h + 1) * a.lse_stride + row] * kLog2eG;
    const float c = a.scale * kLog2eG;
    f32x4_t gacc[NS];
#pragma unroll
    for (int i = 0; i < NS; ++i) gacc[i] = zero4();
    float lam_sum = 0.f;
    const int kv_end = a.mask ? min(kl, q0 + COLS) : kl;
    const int wave_last = a.mask ? min(kl - 1, qw0 + 15) : kl - 1;
    Tl tk, tv;
    if (kv_end > 0) {
        tk.load(K, a.ldk, 0, kl, half, vec);
        tv.load(V, a.ldv, 0, kl, half, vec);
    }
    for (int k0 = 0; k0 < kv_end; k0 += KT) {
        __syncthreads();
        tk.store(sK);
        tv.store(sV);
        __syncthreads();
        if (k0 + KT < kv_end) {
            tk.load(K, a.ldk, k0 + KT, kl, half, vec);
            tv.load(V, a.ldv, k0 + KT, kl, half, vec);
        }
        if (qw0 >= ql) continue;
#pragma unroll
        for (int i = 0; i < KT / 16 / Share<COLS>::SPLITS; ++i) {
            const int kt = Share<COLS>::SPLITS * i + split;
            if (k0 + 16 * kt > wave_last) break;
            f32x4_t p1 = first_product<HH, 0, NS / 2>(sK, 16 * kt, lane, qf);
            f32x4_t p2 = first_product<HH, NS / 2, NS>(sK, 16 * kt, lane, qf);
            const f32x4_t gr = first_product<HH, 0, NS>(sV, 16 * kt, lane, dof);
            const int kb = k0 + 16 * kt;
            if (kb + 16 > kl || (a.mask && kb + 15 > qw0))
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int key = kb + 4 * g + e;
                    if (key >= kl || (a.mask && key > qi)) p1[e] = p2[e] = -INFINITY;
                }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float u1 = __builtin_amdgcn_exp2f(__builtin_fmaf(p1[e], c, -e1)), u2 = __builtin_amdgcn_exp2f(__builtin_fmaf(p2[e], c, -e2));
                lam_sum = __builtin_fmaf(u2, gr[e], lam_sum);
                p1[e] = u1 * (gr[e] - d1);
                p2[e] = u2 * (d2 - gr[e]) * lam;
            }
            second_product<HH, 0, NS / 2>(sK, 16 * kt, lane, p1, gacc);
            second_product<HH, NS / 2, NS>(sK, 16 * kt, lane, p2, gacc);
        }
    }
    join_shares<COLS>(lds, split, t, gacc);
    f32x4_t lam_join[1] = {{lam_sum, 0.f, 0.f, 0.f}};
    join_shares<COLS>(lds, split, t, lam_join);
    if (split != 0) return;
    const bool by_rows = a.mask && (any_not_finite(gacc) || any_not_finite(lam_join));
    if (by_rows) {
        lam_sum = 0.f;
        for (int i = 0; i < min(16, ql - qw0); ++i)
            lam_sum += diff_dq_row<T>(a, s, h, qw0 + i, __shfl(e1, i, 64), __shfl(e2, i, 64), __shfl(d1, i, 64), __shfl(d2, i, 64), lane);
    } else {
        lam_sum = wave_sum(qi < ql ? lam_join[0][0] : 0.f);
    }
    if (lane == 0 && qw0 < ql) a.lam_part[(size_t)h * a.q_total_rows + qrow0 + qw0] = lam_sum;
    if (qi < ql && !by_rows) store_column<T, HH>(gacc, a.scale, (T*)a.dq + (qrow0 + qi) * a.ldq + (long long)h * hd, half, g, vec);
}

// ---------------------------------------------------------------- backward: dK, dV
template <class T, int HH, int COLS>
__global__ __launch_bounds__(512, HH <= 32 && COLS == 64 ? 4 : 2) void diff_bwd_dkv_kernel(DiffAttnArgs a) {
    typedef Tile<T, HH, 512> Tl;
    constexpr int QT = Tl::ROWS, NS = HH / 8;
    __shared__ __attribute__((aligned(16))) float lds[2 * Tl::FLOATS];
    static_assert(2 * Tl::FLOATS >= 256 * 4 * NS, "the sums of four wavefronts");
    float *const sQ = lds, *const sO = lds + Tl::FLOATS;
    __shared__ __attribute__((aligned(16))) float stat[4][QT];         // log-sum-exps (exp2 domain), D_1, D_2 of the tile's queries
    const int t = threadIdx.x, lane = t & 63, wave8 = __builtin_amdgcn_readfirstlane(t >> 6), g = lane >> 4;
    const int wave = wave8 % Share<COLS>::GROUPS, split = wave8 / Share<COLS>::GROUPS;
    if (blockIdx.z == 0) {                              // a layer of work-groups more, which start first: one for each head sums up dlambda
        if (blockIdx.x == 0) sum_dlambda<16, 512>(a, blockIdx.y, lds);
        return;
    }
    const ColumnBlock cb = column_block<COLS>(a, a.k_len, false, blockIdx.z - 1);
    if (cb.first < 0) return;
    const int s = cb.s, h = cb.h, k0 = cb.first, ql = a.q_len[s], kl = a.k_len[s], hd = a.head_dim, half = hd / 2;
    const bool vec = a.vec;
    const long long qrow0 = a.q_row[s], krow0 = a.k_row[s];
    const T* Q = (const T*)a.q + qrow0 * a.ldq + (long long)h * hd;
    const T* dO = (const T*)a.d_o + qrow0 * a.ldo + (long long)h * hd;
    const int kw0 = k0 + wave * 16, ki = kw0 + (lane & 15), ki_c = ki < kl ? ki : kl - 1;
    float4 kf[NS], vf[NS];
    load_column<T, HH>((const T*)a.k + (krow0 + ki_c) * a.ldk + (long long)h * hd, half, g, vec, kf);
    load_column<T, HH>((const T*)a.v + (krow0 + ki_c) * a.ldv + (long long)h * hd, half, g, vec, vf);
    const float c = a.scale * kLog2eG, lam = a.lambda[h];
    f32x4_t dk[NS], dv[NS];
#pragma unroll
    for (int i = 0; i < NS; ++i) { dk[i] = zero4(); dv[i] = zero4(); }
    const int q_begin = a.mask ? k0 : 0;                               // causal: only queries at or after the key see it
    Tl tq, to;
    float st[4];
    auto fetch = [&](int q0) {
        tq.load(Q, a.ldq, q0, ql, half, vec);
        to.load(dO, a.ldo, q0, ql, half, vec);
        const bool in = t < QT && q0 + t < ql;
        const long long row = qrow0 + q0 + t;
        st[0] = in ? a.lse[(size_t)(2 * h) * a.lse_stride + row] * kLog2eG : 0.f;
        st[1] = in ? a.lse[(size_t)(2 * h + 1) * a.lse_stride + row] * kLog2eG : 0.f;
        st[2] = in ? a.d1[(size_t)h * a.q_total_rows + row] : 0.f;
        st[3] = in ? a.d2[(size_t)h * a.q_total_rows + row] : 0.f;
    };
    if (q_begin < ql) fetch(q_begin);
    for (int q0 = q_begin; q0 < ql; q0 += QT) {
        __syncthreads();
        tq.store(sQ);
        to.store(sO);
        if (t < QT)
#pragma unroll
            for (int i = 0; i < 4; ++i) stat[i][t] = st[i];
        __syncthreads();
        if (q0 + QT < ql) fetch(q0 + QT);
        if (kw0 >= kl) continue;
#pragma unroll
        for (int i = 0; i < QT / 16 / Share<COLS>::SPLITS; ++i) {
            const int qt = Share<COLS>::SPLITS * i + split;
            const int qb = q0 + 16 * qt;
            if (qb >= ql || (a.mask && qb + 15 < kw0)) continue;       // no visible query
            f32x4_t p1 = first_product<HH, 0, NS / 2>(sQ, 16 * qt, lane, kf);
            f32x4_t p2 = first_product<HH, NS / 2, NS>(sQ, 16 * qt, lane, kf);
            const f32x4_t gr = first_product<HH, 0, NS>(sO, 16 * qt, lane, vf);
            f32x4_t p;
            const f32x4_t e1 = *reinterpret_cast<const f32x4_t*>(&stat[0][16 * qt + 4 * g]), e2 = *reinterpret_cast<const f32x4_t*>(&stat[1][16 * qt + 4 * g]);
            const f32x4_t d1 = *reinterpret_cast<const f32x4_t*>(&stat[2][16 * qt + 4 * g]), d2 = *reinterpret_cast<const f32x4_t*>(&stat[3][16 * qt + 4 * g]);
            // queries past the last one need no mask: they are zeros, their statistics too, so that a probability of 1 multiplies nothing
            if (a.mask && qb < kw0 + 15)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (qb + 4 * g + e < ki) p1[e] = p2[e] = -INFINITY;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float u1 = __builtin_amdgcn_exp2f(__builtin_fmaf(p1[e], c, -e1[e])), u2 = lam * __builtin_amdgcn_exp2f(__builtin_fmaf(p2[e], c, -e2[e]));
                p[e] = u1 - u2;
                p1[e] = u1 * (gr[e] - d1[e]);
                p2[e] = u2 * (d2[e] - gr[e]);
            }
            second_product<HH, 0, NS>(sO, 16 * qt, lane, p, dv);
            second_product<HH, 0, NS / 2>(sQ, 16 * qt, lane, p1, dk);
            second_product<HH, NS / 2, NS>(sQ, 16 * qt, lane, p2, dk);
        }
    }
    join_shares<COLS>(lds, split, t, dk);
    join_shares<COLS>(lds, split, t, dv);
    if (split != 0) return;
    if (a.mask && (any_not_finite(dk) || any_not_finite(dv))) {
        for (int i = 0; i < min(16, kl - kw0); ++i) diff_dkv_row<T>(a, s, h, kw0 + i, lane);
        return;
    }
    if (ki >= kl) return;
    store_column<T, HH>(dk, a.scale, (T*)a.dk + (krow0 + ki) * a.ldk + (long long)h * hd, half, g, vec);
    store_column<T, HH>(dv, 1.0f, (T*)a.dv + (krow0 + ki) * a.ldv + (long long)h * hd, half, g, vec);
}

template <class T, int HH> void fwd_launch(const DiffAttnArgs& a, hipStream_t st) {
    const dim3 grid = a.k_splits > 1 ? dim3(a.k_splits, a.n_heads, a.n_seq) : column_grid(a, a.max_q_len);
    hipLaunchKernelGGL((diff_fwd_kernel<T, HH>), grid, dim3(256), 0, st, a);
}
// Fewer work-groups of 64 columns than two for a compute unit: 32 columns each (up to head size 96: above, a tile has no 16 rows for each of four wavefronts).  64 -> 32, dQ and dK/dV together, fp32, heads of 64: 23 sequences of 88
// to 177, 4 heads, causal (276 work-groups) 59 -> 52 us; 3 of 100 to 200, 2 heads 50 -> 35; but 31 of 366 to 523, 16 heads (4 464) 1 114 -> 1 226.
bool narrow(const DiffAttnArgs& a, int max_len) { return diff_general_columns(a, max_len) == 32; }
template <class T, int HH> void dq_launch(const DiffAttnArgs& a, hipStream_t st) {
    if constexpr (HH <= 48)
        if (narrow(a, a.max_q_len)) {
            hipLaunchKernelGGL((diff_bwd_dq_kernel<T, HH, 32>), column_grid(a, a.max_q_len, 32), dim3(512), 0, st, a);
            return;
        }
    hipLaunchKernelGGL((diff_bwd_dq_kernel<T, HH, 64>), column_grid(a, a.max_q_len), dim3(512), 0, st, a);
}
dim3 and_dlambda(dim3 g) { return dim3(g.x, g.y, g.z + 1); }
template <class T, int HH> void dkv_launch(const DiffAttnArgs& a, hipStream_t st) {
    if constexpr (HH <= 48)
        if (narrow(a, a.max_k_len)) {
            hipLaunchKernelGGL((diff_bwd_dkv_kernel<T, HH, 32>), and_dlambda(column_grid(a, a.max_k_len, 32)), dim3(512), 0, st, a);
            return;
        }
    hipLaunchKernelGGL((diff_bwd_dkv_kernel<T, HH, 64>), and_dlambda(column_grid(a, a.max_k_len)), dim3(512), 0, st, a);
}

}  // namespace

int diff_general_columns(const DiffAttnArgs& a, int max_len) {
    return a.head_dim <= 96 && (long long)a.n_seq * a.n_heads * (max_len / 64 + 1) <= 2LL * kDiffUnits ? 32 : 64;
}

#define DS_DIFF_DISPATCH(launch)                                              \
    do {                                                                      \
        const bool bf = a.dtype == DS_DTYPE_BF16;                             \
        if (a.head_dim <= 32) bf ? launch<bf16_t, 16>(a, st) : launch<float, 16>(a, st);      \
        else if (a.head_dim <= 64) bf ? launch<bf16_t, 32>(a, st) : launch<float, 32>(a, st); \
        else if (a.head_dim <= 96) bf ? launch<bf16_t, 48>(a, st) : launch<float, 48>(a, st); \
        else bf ? launch<bf16_t, 64>(a, st) : launch<float, 64>(a, st);       \
    } while (0)

ds_status diff_fwd_general(const DiffAttnArgs& a, hipStream_t st) {
    DS_DIFF_DISPATCH(fwd_launch);
    DS_LAUNCH_CHECK();
    return a.k_splits > 1 ? diff_join(a, st) : DS_OK;
}

ds_status diff_join(const DiffAttnArgs& a, hipStream_t st) {
    const dim3 grid((a.max_q_len + 3) / 4, a.n_heads, a.n_seq);
    if (a.dtype == DS_DTYPE_BF16) hipLaunchKernelGGL((diff_join_kernel<bf16_t>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((diff_join_kernel<float>), grid, dim3(256), 0, st, a);
    DS_LAUNCH_CHECK();
    return DS_OK;
}

ds_status diff_bwd_general(const DiffAttnArgs& a, hipStream_t st) {
    DS_DIFF_DISPATCH(dq_launch);
    DS_LAUNCH_CHECK();
    DS_DIFF_DISPATCH(dkv_launch);
    DS_LAUNCH_CHECK();
    return DS_OK;
}
