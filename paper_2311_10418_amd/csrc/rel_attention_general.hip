// Attention with a relative position bias for every type, head size, stride and alignment the entry points take: v_mfma_f32_16x16x4_f32 on fp32 values (bf16
// operands are widened as their tiles go to LDS), so that products, probabilities and sums are fp32 throughout.
//
// A wavefront owns 16 "column" items (queries in forward and dQ, keys in dK/dV) and computes transposed score blocks: 16 rows of the other side x its 16
// columns, lane = (column lane % 16, rows 4 g + e with g = lane / 16, e = 0..3).  Per column values are per-lane scalars, and register e of a block is, as it
// stands, the B operand of the second product for the rows {4 g + e}.  Tiles of the other side are kept in LDS row by row, heads padded with zeros to HD columns.
//
// The bias.  A block of 16 x 16 pairs covers 31 distances; where all of them lie beyond reach on one side it is one number, the rest reads the table of the
// head in LDS (distances -reach - 31 .. reach + 31).  Sums of dS by distance: beyond reach a register per lane and side, near blocks add theirs to an array of
// the wavefront's own in LDS, 16 lanes (16 distances) at a time.
//
// Bound by the trips between memory, LDS and the products at short sequences (a tile of 64 rows costs 2.5 us of which the matrix instructions are 1, and a kernel has 5 us besides): fp32, 23
// sequences of 88 to 177, 4 heads of 64, causal, dQ 23 us and dK/dV 26 (matrix pipe 8 and 10 % of the cycles).  dK/dV with work-groups of 32 columns, which such calls take, has 136 registers
// at head size 64: three wavefronts to a SIMD, and so one work-group of eight to a compute unit.  With 64 columns it has 128 and spills 3 or 4.
//
// Causal masks and values that are not finite: as in the general kernels of differential attention, a wavefront whose sums are not finite in the end takes its
// columns one by one (rel_attention_rows.hpp), so that a row is affected by the rows it sees and by no others.
#include "rel_attention.hpp"
#include "rel_attention_rows.hpp"
#include "gemm.hpp"
#include <type_traits>

namespace {

constexpr float kLog2eG = 1.4426950408889634f;
constexpr float kLn2G = 0.6931471805599453f;
constexpr int kPad = 31;                                // distances that a near block may reach beyond `reach`

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

template <class T, int HD, int THREADS> struct Tile {
    static constexpr int ROWS = HD <= 96 ? 64 : 32, LD = HD + 4, NV = ROWS * HD / 4 / THREADS, FLOATS = ROWS * LD;
    float4 v[NV];
    __device__ __forceinline__ void load(const T* src, long long ld, int r0, int n_rows, int hd, bool vec) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int u = threadIdx.x + THREADS * i, r = r0 + u / (HD / 4), d = (u % (HD / 4)) * 4;
            v[i] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (r < n_rows && d < hd) v[i] = load4<T>(src + (long long)r * ld + d, vec);
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
template <class T, int HD> __device__ __forceinline__ void load_column(const T* row, int hd, int g, bool vec, float4 (&f)[HD / 16]) {
#pragma unroll
    for (int s = 0; s < HD / 16; ++s) {
        const int d = 16 * s + 4 * g;
        f[s] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (d < hd) f[s] = load4<T>(row + d, vec);
    }
}
template <class T, int HD> __device__ __forceinline__ void store_column(const f32x4_t (&acc)[HD / 16], float mul, T* row, int hd, int g, bool vec) {
#pragma unroll
    for (int s = 0; s < HD / 16; ++s) {
        const int d = 16 * s + 4 * g;
        if (d < hd) store4(row + d, acc[s] * mul, vec);
    }
}
// rows rb .. rb+15 of a tile times this lane's column item
template <int HD> __device__ __forceinline__ f32x4_t first_product(const float* tile, int rb, int lane, const float4 (&f)[HD / 16]) {
    const float* p = tile + (rb + (lane & 15)) * (HD + 4) + 4 * (lane >> 4);
    f32x4_t acc = zero4();
#pragma unroll
    for (int s = 0; s < HD / 16; ++s) {
        const float4 x = *reinterpret_cast<const float4*>(p + 16 * s);
        acc = mfma4(x.x, f[s].x, acc);
        acc = mfma4(x.y, f[s].y, acc);
        acc = mfma4(x.z, f[s].z, acc);
        acc = mfma4(x.w, f[s].w, acc);
    }
    return acc;
}
// out^T[feature step][column] += tile[rows rb .. rb+15]^T * w
template <int HD> __device__ __forceinline__ void second_product(const float* tile, int rb, int lane, const f32x4_t& w, f32x4_t (&out)[HD / 16]) {
    const float* p = tile + (rb + 4 * (lane >> 4)) * (HD + 4) + (lane & 15);
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int s = 0; s < HD / 16; ++s) out[s] = mfma4(p[e * (HD + 4) + 16 * s], w[e], out[s]);
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

// A work-group's COLS columns: sequence, head, block (negative: nothing to do).  Sequences last to first: a plan lists them by ascending length, and the
// longest chains of tiles should start first.
struct ColumnBlock { int s, h, block; };
template <int COLS> __device__ __forceinline__ ColumnBlock column_block(const RelAttnArgs& a, const int32_t* len, bool last_first, int z) {
    ColumnBlock c = {a.n_seq - 1 - z, (int)blockIdx.y, -1};
    const int n = (len[c.s] + COLS - 1) / COLS, b = blockIdx.x;
    if (b < n) c.block = last_first ? n - 1 - b : b;
    return c;
}
// an odd number of blocks per grid row: work-groups go to the eight XCDs in turn, and the longest of every sequence should not meet on one
dim3 column_grid(const RelAttnArgs& a, int max_len, int cols) { return dim3((max_len / cols + (max_len % cols != 0)) | 1, a.n_heads, a.n_seq); }

// The table of a head, entry i = distance + reach + kPad, in three parts: its two trips to memory (the buckets, then their biases) go beside those that a work-group
// begins with anyway.  The last entries of a long reach are made in the end.
template <class T, int THREADS> struct TableFill {
    int bucket;
    float bias;
    __device__ __forceinline__ void buckets(const RelAttnArgs& a) { bucket = a.bucket[min(max((int)threadIdx.x - kPad, 0), 2 * a.reach)]; }
    __device__ __forceinline__ void biases(const RelAttnArgs& a, int h) {
        bias = kLog2eG * to_f32(((const T*)a.bias)[(size_t)min(max(bucket, 0), a.n_buckets - 1) * a.n_heads + h]);
    }
    __device__ __forceinline__ void store(const RelAttnArgs& a, int h, float* table) const {
        const int n = 2 * (a.reach + kPad) + 1;
        if ((int)threadIdx.x < n) table[threadIdx.x] = bias;
        for (int i = threadIdx.x + THREADS; i < n; i += THREADS) table[i] = rel_bias(a, h, i - kPad);
    }
};
// Where a block of 16 rows and 16 columns lies whose distances are first .. first + 30: -1 / 1: beyond reach on one side, 0: near
__device__ __forceinline__ int side_of(int first, int reach) { return first + 30 <= -reach ? -1 : first >= reach ? 1 : 0; }

__host__ __device__ constexpr int table_floats(int reach) { return (2 * (reach + kPad) + 1 + 3) & ~3; }

// ---------------------------------------------------------------- forward
template <class T, int HD>
__global__ __launch_bounds__(256, HD <= 64 ? 3 : 2) void rel_fwd_kernel(RelAttnArgs a) {
    typedef Tile<T, HD, 256> Tl;
    constexpr int KT = Tl::ROWS, NB = KT / 16, NS = HD / 16;
    extern __shared__ __attribute__((aligned(16))) float lds[];
    float *const sK = lds, *const sV = lds + Tl::FLOATS, *const table = lds + 2 * Tl::FLOATS;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4;
    TableFill<T, 256> fill;
    fill.buckets(a);
    ColumnBlock cb = column_block<64>(a, a.q_len, a.mask != 0, blockIdx.z);
    const int split = a.k_splits > 1 ? blockIdx.x : 0;                 // (one block of queries then)
    if (a.k_splits > 1) cb.block = a.q_len[cb.s] > 0 ? 0 : -1;
    if (cb.block < 0) return;
    fill.biases(a, cb.h);
    const int s = cb.s, h = cb.h, q0 = 64 * cb.block, ql = a.q_len[s], hd = a.head_dim, pos = rel_position(a, s);
    int kl = rel_keys(a, a.k_len[s], ql, pos), kfirst = 0;
    if (a.k_splits > 1) {                                              // keys kfirst .. kfirst + kl - 1: whole tiles of 64, as evenly as they go
        const long long run = ((long long)kl + 64LL * a.k_splits - 1) / (64LL * a.k_splits) * 64;
        kfirst = (int)min(run * split, (long long)kl);
        kl = (int)min(run, (long long)kl - kfirst);
    }
    const bool vec = a.vec;
    const long long qrow0 = a.q_row[s], krow0 = (long long)a.k_row[s] + kfirst;
    const T* K = (const T*)a.k + krow0 * a.ldk + (long long)h * hd;
    const T* V = (const T*)a.v + krow0 * a.ldv + (long long)h * hd;
    const int qw0 = q0 + wave * 16, qi = qw0 + (lane & 15), qi_c = qi < ql ? qi : ql - 1;
    const int pw0 = pos - kfirst + qw0, pi = pw0 + (lane & 15);        // positions, keys counted from the first of this work-group
    float4 qf[NS];
    load_column<T, HD>((const T*)a.q + (qrow0 + qi_c) * a.ldq + (long long)h * hd, hd, g, vec, qf);
    f32x4_t o[NS];
#pragma unroll
    for (int i = 0; i < NS; ++i) o[i] = zero4();
    const float c = a.scale * kLog2eG;
    float m = -INFINITY, l = 0.f;                                      // running maximum (exp2 domain), this lane's part of the sum
    const int kv_end = a.mask ? min(kl, max(0, pos - kfirst + min(q0 + 64, ql))) : kl;
    const int wave_last = a.mask ? min(kl - 1, pw0 + 15) : kl - 1;     // last key this wavefront can see
    Tl tk, tv;
    if (kv_end > 0) {
        tk.load(K, a.ldk, 0, kl, hd, vec);
        tv.load(V, a.ldv, 0, kl, hd, vec);
    }
    fill.store(a, h, table);
    __syncthreads();
    const float *const near = table + a.reach + kPad + 4 * g - pi;     // [key tile row e]: near[kb + e]
    const float side_bias[2] = {table[0], table[2 * (a.reach + kPad)]};
    for (int k0 = 0; k0 < kv_end; k0 += KT) {
        __syncthreads();                                               // the previous tile has been read by everybody
        tk.store(sK);
        tv.store(sV);
        __syncthreads();
        if (k0 + KT < kv_end) {
            tk.load(K, a.ldk, k0 + KT, kl, hd, vec);
            tv.load(V, a.ldv, k0 + KT, kl, hd, vec);
        }
        if (k0 > wave_last || qw0 >= ql) continue;
        f32x4_t p[NB];
        float x = -INFINITY;
#pragma unroll
        for (int kt = 0; kt < NB; ++kt) {
            p[kt] = first_product<HD>(sK, 16 * kt, lane, qf);
            const int kb = k0 + 16 * kt, side = side_of(kb - pw0 - 15, a.reach);
            if (side == 0) {
#pragma unroll
                for (int e = 0; e < 4; ++e) p[kt][e] = __builtin_fmaf(p[kt][e], c, near[kb + e]);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) p[kt][e] = __builtin_fmaf(p[kt][e], c, side < 0 ? side_bias[0] : side_bias[1]);
            }
            if (kb + 16 > kl || (a.mask && kb + 15 > pw0))             // (a branch: most blocks need no mask)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int key = kb + 4 * g + e;
                    if (key >= kl || (a.mask && key > pi)) p[kt][e] = -INFINITY;
                }
#pragma unroll
            for (int e = 0; e < 4; ++e) x = fmaxf(x, p[kt][e]);
        }
        const float m_new = fmaxf(m, groups_max(x)), m_use = m_new == -INFINITY ? 0.f : m_new;
        const float alpha = __builtin_amdgcn_exp2f(m - m_use);
        float rs = 0.f;
#pragma unroll
        for (int kt = 0; kt < NB; ++kt)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                p[kt][e] = __builtin_amdgcn_exp2f(p[kt][e] - m_use);
                rs += p[kt][e];
            }
        l = l * alpha + rs;
        m = m_new;
#pragma unroll
        for (int i = 0; i < NS; ++i) o[i] *= alpha;
#pragma unroll
        for (int kt = 0; kt < NB; ++kt) second_product<HD>(sV, 16 * kt, lane, p[kt], o);
    }
    l = groups_sum(l);
    if (a.mask && any_not_finite(o)) {
        const float e2 = a.k_splits > 1 ? (m == -INFINITY ? 0.f : m) : m + __builtin_amdgcn_logf(l);
        for (int i = 0; i < min(16, ql - qw0); ++i) {
            const long long row = qrow0 + qw0 + i;
            const float e = __shfl(e2, i, 64), li = __shfl(l, i, 64), mi = __shfl(m, i, 64);
            const RelPair r = li == 0.f ? RelPair{0.f, 0.f} : rel_fwd_row<T>(a, s, h, qw0 + i, pos + qw0 + i, kfirst, kl, e, lane);
            if (a.k_splits > 1) {
                const RelPart to = rel_part(a, h, row, split);
                rel_put<float>(to.o, hd, lane, r);
                if (lane == 0) to.stat[0] = mi, to.stat[1] = li;
            } else {
                rel_put<T>((T*)a.o + row * a.ldo + (long long)h * hd, hd, lane, r);
                if (lane == 0) a.lse[(size_t)h * a.lse_stride + row] = (mi + __builtin_amdgcn_logf(li)) * kLn2G;
            }
        }
        return;
    }
    if (qi >= ql) return;
    const long long row = qrow0 + qi;
    if (l == 0.f)                                                      // sees nothing
#pragma unroll
        for (int i = 0; i < NS; ++i) o[i] = zero4();
    if (a.k_splits > 1) {
        const RelPart to = rel_part(a, h, row, split);
        if (g == 0) to.stat[0] = m, to.stat[1] = l;
        store_column<float, HD>(o, 1.0f, to.o, hd, g, true);
        return;
    }
    store_column<T, HD>(o, l == 0.f ? 0.f : 1.0f / l, (T*)a.o + row * a.ldo + (long long)h * hd, hd, g, vec);
    if (g == 0) a.lse[(size_t)h * a.lse_stride + row] = (m + __builtin_amdgcn_logf(l)) * kLn2G;
}

// What the work-groups that shared a head's keys found, put together: a wavefront per query, lane i with the statistics of work-group i, then two columns
// of the output per lane.  A work-group without keys has sum 0, and its maximum does not count.
template <class T> __global__ __launch_bounds__(256) void rel_join_kernel(RelAttnArgs a) {
    const int lane = threadIdx.x & 63, q = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = blockIdx.y, s = blockIdx.z;
    if (q >= a.q_len[s]) return;
    const long long row = (long long)a.q_row[s] + q;
    const int hd = a.head_dim, n = a.k_splits;
    const size_t step = hd + 4;
    const RelPart p = rel_part(a, h, row, 0);
    // outputs on their way together, the first of them before the statistics are there (those beyond 16 one by one: single tokens of 4 heads of 64, fp32, two caches of 8 192 keys 22.9 -> 13.2 us;
    // 16 heads, one of 32 768 61 -> 52)
    constexpr int kAtOnce = 16;
    const bool on = 2 * lane < hd;
    const float* from = p.o + (on ? 2 * lane : 0);
    auto load = [&](int i) { return *reinterpret_cast<const float2*>(from + min(i, n - 1) * step); };
    float2 v[kAtOnce];
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) v[i] = load(i);
    const float2 st = lane < n ? *reinterpret_cast<const float2*>(p.stat + lane * step) : make_float2(0.f, 0.f);
    const float top = st.y == 0.f ? -INFINITY : st.x, up = wave_max(top);
    const float w = st.y == 0.f ? 0.f : __builtin_amdgcn_exp2f(top - up), sum = wave_sum(w * st.y);
    auto weight = [&](int i) { return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, w), i)); };
    float o0 = 0.f, o1 = 0.f;
    auto add = [&](float2 x, float wt) { o0 = __builtin_fmaf(x.x, wt, o0); o1 = __builtin_fmaf(x.y, wt, o1); };
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i)
        if (i < n) add(v[i], weight(i));
    for (int first = kAtOnce; first < n; first += kAtOnce) {
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) v[i] = load(first + i);
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i)
            if (first + i < n) add(v[i], weight(first + i));
    }
    const float r = sum == 0.f ? 0.f : 1.0f / sum;
    if (on) {
        T* to = (T*)a.o + row * a.ldo + (long long)h * hd + 2 * lane;
        to[0] = from_f32<T>(o0 * r);
        to[1] = from_f32<T>(o1 * r);
    }
    if (lane == 0) a.lse[(size_t)h * a.lse_stride + row] = (up + __builtin_amdgcn_logf(sum)) * kLn2G;
}

// ---------------------------------------------------------------- backward: dQ, D, the slots of dbias
// Eight wavefronts, SPLITS = 2 or 4 for each 16 columns: they take every SPLITS-th 16 rows of a tile, and what they have is added up in the end, by
// halves.  A work-group has 64 columns, or 32 where that makes too few of them for the compute units (rel_general_columns).
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

template <class T, int HD, int COLS>
__global__ __launch_bounds__(512, HD <= 64 ? 4 : 2) void rel_bwd_dq_kernel(RelAttnArgs a) {
    typedef Tile<T, HD, 512> Tl;
    constexpr int KT = Tl::ROWS, NS = HD / 16;
    extern __shared__ __attribute__((aligned(16))) float lds[];
    static_assert(2 * Tl::FLOATS >= 256 * 4 * NS, "the sums of four wavefronts");
    const int wide = table_floats(a.reach);
    float *const sK = lds, *const sV = lds + Tl::FLOATS, *const table = lds + 2 * Tl::FLOATS;
    const int t = threadIdx.x, lane = t & 63, wave8 = __builtin_amdgcn_readfirstlane(t >> 6), g = lane >> 4;
    float *const sums = table + wide * (1 + wave8);                    // this wavefront's sums of dS by distance
    const int wave = wave8 % Share<COLS>::GROUPS, split = wave8 / Share<COLS>::GROUPS;
    TableFill<T, 512> fill;
    fill.buckets(a);
    const int before = blocks_part<COLS, 512>(a, a.n_seq - 1 - blockIdx.z);
    const ColumnBlock cb = column_block<COLS>(a, a.q_len, a.mask != 0, blockIdx.z);
    if (cb.block < 0) return;
    fill.biases(a, cb.h);
    const int s = cb.s, h = cb.h, q0 = COLS * cb.block, ql = a.q_len[s], pos = rel_position(a, s), kl = rel_keys(a, a.k_len[s], ql, pos), hd = a.head_dim;
    const bool vec = a.vec;
    const long long qrow0 = a.q_row[s], krow0 = a.k_row[s];
    const T* K = (const T*)a.k + krow0 * a.ldk + (long long)h * hd;
    const T* V = (const T*)a.v + krow0 * a.ldv + (long long)h * hd;
    const int qw0 = q0 + wave * 16, qi = qw0 + (lane & 15), qi_c = qi < ql ? qi : ql - 1, pw0 = pos + qw0, pi = pos + qi;
    const long long row = qrow0 + qi_c;
    const int kv_end = a.mask ? min(kl, max(0, pos + q0 + COLS)) : kl;
    const int wave_last = a.mask ? min(kl - 1, pw0 + 15) : kl - 1;
    Tl tk, tv;
    if (kv_end > 0) {
        tk.load(K, a.ldk, 0, kl, hd, vec);
        tv.load(V, a.ldv, 0, kl, hd, vec);
    }
    float4 qf[NS], dof[NS];
    load_column<T, HD>((const T*)a.q + row * a.ldq + (long long)h * hd, hd, g, vec, qf);
    load_column<T, HD>((const T*)a.d_o + row * a.ldo + (long long)h * hd, hd, g, vec, dof);
    float d = 0.f;
    {
        float4 f[NS];
        load_column<T, HD>((const T*)a.o + row * a.ldo + (long long)h * hd, hd, g, vec, f);
#pragma unroll
        for (int i = 0; i < NS; ++i) d += (f[i].x * dof[i].x + f[i].y * dof[i].y) + (f[i].z * dof[i].z + f[i].w * dof[i].w);
        d = groups_sum(d);
        if (g == 0 && qi < ql && split == 0) a.d[(size_t)h * a.q_total_rows + row] = d;
    }
    const float e2 = rel_lse2(a.lse[(size_t)h * a.lse_stride + row]), c = a.scale * kLog2eG;
    fill.store(a, h, table);
    for (int i = t; i < 8 * wide; i += 512) table[wide + i] = 0.f;
    const int slot = blocks_sum<512>(before, reinterpret_cast<int*>(sK)) + cb.block;
    const int near = a.reach + kPad + 4 * g - pi;                      // [key tile row e]: entry near + kb + e
    const float side_bias[2] = {table[0], table[2 * (a.reach + kPad)]};
    const float live = qi < ql ? 1.f : 0.f;             // (a lane past the last query repeats the last one: its sums do not count)
    float beyond[2] = {0.f, 0.f};
    f32x4_t gacc[NS];
#pragma unroll
    for (int i = 0; i < NS; ++i) gacc[i] = zero4();
    for (int k0 = 0; k0 < kv_end; k0 += KT) {
        __syncthreads();
        tk.store(sK);
        tv.store(sV);
        __syncthreads();
        if (k0 + KT < kv_end) {
            tk.load(K, a.ldk, k0 + KT, kl, hd, vec);
            tv.load(V, a.ldv, k0 + KT, kl, hd, vec);
        }
        if (qw0 >= ql) continue;
#pragma unroll
        for (int i = 0; i < (KT / 16 + Share<COLS>::SPLITS - 1) / Share<COLS>::SPLITS; ++i) {
            const int kt = Share<COLS>::SPLITS * i + split, kb = k0 + 16 * kt;
            if (16 * kt >= KT || kb > wave_last) break;
            f32x4_t p = first_product<HD>(sK, 16 * kt, lane, qf);
            const f32x4_t gr = first_product<HD>(sV, 16 * kt, lane, dof);
            const int side = side_of(kb - pw0 - 15, a.reach);
            const float flat = (side < 0 ? side_bias[0] : side_bias[1]) - e2;
#pragma unroll
            for (int e = 0; e < 4; ++e) p[e] = __builtin_fmaf(p[e], c, side ? flat : table[near + kb + e] - e2);
            if (kb + 16 > kl || (a.mask && kb + 15 > pw0))
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int key = kb + 4 * g + e;
                    if (key >= kl || (a.mask && key > pi)) p[e] = -INFINITY;
                }
#pragma unroll
            for (int e = 0; e < 4; ++e) p[e] = __builtin_amdgcn_exp2f(p[e]) * (gr[e] - d);
            if (side) {
                const float add = live * ((p[0] + p[1]) + (p[2] + p[3]));
                beyond[0] += side < 0 ? add : 0.f;
                beyond[1] += side < 0 ? 0.f : add;
            } else {
                // rows 4 g + e of 16 columns: two sums a lane, of distances 16 apart; the four groups of lanes overlap and add theirs one after the other
                float minus = 0.f, around = 0.f;
                add_diagonals<0>(live * p[0], minus, around);
                add_diagonals<1>(live * p[1], minus, around);
                add_diagonals<2>(live * p[2], minus, around);
                add_diagonals<3>(live * p[3], minus, around);
                float* to = &sums[kb - pw0 + 4 * g - (lane & 15) + a.reach + kPad];
#pragma unroll
                for (int part = 0; part < 4; ++part)
                    if (g == part) {
                        lds_add(to, minus);
                        if ((lane & 15) > 12) lds_add(to + 16, around);
                    }
            }
            second_product<HD>(sK, 16 * kt, lane, p, gacc);
        }
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const float all = wave_sum(beyond[i]);
        if (lane == 0) lds_add(&sums[kPad + 2 * a.reach * i], all);
    }
    join_shares<COLS>(lds, split, t, gacc);
    // sums that are not finite: this block's columns one by one, and all it has of dbias with them
    int* flag = reinterpret_cast<int*>(lds);
    __syncthreads();
    if (t == 0) flag[0] = 0;
    __syncthreads();
    bool odd = split == 0 && qw0 < ql && any_not_finite(gacc);
    if (a.mask) {                                       // (a sum of dS may overflow or be NaN where those of dQ are finite: 0 x NaN is not)
        float nothing = 0.f;
        for (int i = lane; i < wide; i += 64) nothing = __builtin_fmaf(sums[i], 0.f, nothing);
        odd = odd || __builtin_amdgcn_ballot_w64(nothing != 0.f) != 0;
        if (odd && lane == 0) flag[0] = 1;
    }
    __syncthreads();
    const bool by_rows = a.mask && flag[0] != 0;
    if (by_rows) {
        for (int i = lane; i < wide; i += 64) sums[i] = 0.f;
        wave_lds_sync();
        if (split == 0)
            for (int i = 0; i < min(16, ql - qw0); ++i)
                rel_dq_row<T>(a, s, h, qw0 + i, pw0 + i, kl, __shfl(e2, i, 64), __shfl(d, i, 64), sums + kPad, lane);
    } else if (split == 0 && qi < ql) {
        store_column<T, HD>(gacc, a.scale, (T*)a.dq + (qrow0 + qi) * a.ldq + (long long)h * hd, hd, g, vec);
    }
    __syncthreads();
    // the block's slot: what the wavefronts have, distances beyond reach with those at it
    float* to = a.slots + ((size_t)slot * a.n_heads + h) * (2 * a.reach + 1);
    for (int i = t; i <= 2 * (a.reach + kPad); i += 512) {
        float sum = 0.f;
#pragma unroll
        for (int w = 0; w < 8; ++w) sum += table[wide * (1 + w) + i];
        const int at = i - kPad;
        if (at > 0 && at < 2 * a.reach) to[at] = sum;
        else table[i] = sum;
    }
    __syncthreads();
    if (wave8 < 2) {
        float sum = lane <= kPad ? table[wave8 * (2 * a.reach + kPad) + lane] : 0.f;
        sum = wave_sum(sum);
        if (lane == 0) to[wave8 * 2 * a.reach] = sum;
    }
}

// ---------------------------------------------------------------- backward: dK, dV
template <class T, int HD, int COLS>
__global__ __launch_bounds__(512, HD <= 64 && COLS == 64 ? 4 : 2) void rel_bwd_dkv_kernel(RelAttnArgs a, int slot_cols) {
    typedef Tile<T, HD, 512> Tl;
    constexpr int QT = Tl::ROWS, NS = HD / 16;
    extern __shared__ __attribute__((aligned(16))) float lds[];
    static_assert(2 * Tl::FLOATS >= 256 * 4 * NS, "the sums of four wavefronts");
    float *const sQ = lds, *const sO = lds + Tl::FLOATS, *const stat = lds + 2 * Tl::FLOATS, *const table = stat + 2 * QT;      // stat: log-sum-exps (exp2 domain), D
    const int t = threadIdx.x, lane = t & 63, wave8 = __builtin_amdgcn_readfirstlane(t >> 6), g = lane >> 4;
    const int wave = wave8 % Share<COLS>::GROUPS, split = wave8 / Share<COLS>::GROUPS;
    if (blockIdx.z == 0) {                              // a layer of work-groups more, which start first: one for each head sums up dbias
        if (blockIdx.x != 0) return;
        int* words = reinterpret_cast<int*>(lds);
        const int n = blocks_sum<512>(slot_cols == 32 ? blocks_part<32, 512>(a, a.n_seq) : blocks_part<64, 512>(a, a.n_seq), words);
        sum_dbias<512>(a, blockIdx.y, n, lds);
        return;
    }
    TableFill<T, 512> fill;
    fill.buckets(a);
    const ColumnBlock cb = column_block<COLS>(a, a.k_len, false, blockIdx.z - 1);
    if (cb.block < 0) return;
    fill.biases(a, cb.h);
    const int s = cb.s, h = cb.h, k0 = COLS * cb.block, ql = a.q_len[s], kl = a.k_len[s], hd = a.head_dim, pos = rel_position(a, s);
    const bool vec = a.vec;
    const long long qrow0 = a.q_row[s], krow0 = a.k_row[s];
    const T* Q = (const T*)a.q + qrow0 * a.ldq + (long long)h * hd;
    const T* dO = (const T*)a.d_o + qrow0 * a.ldo + (long long)h * hd;
    const int kw0 = k0 + wave * 16, ki = kw0 + (lane & 15), ki_c = ki < kl ? ki : kl - 1;
    const int q_begin = a.mask ? max(0, k0 - pos) : 0;                 // causal: only queries at or after the key see it
    Tl tq, to;
    float st[2];
    auto fetch = [&](int q0) {
        tq.load(Q, a.ldq, q0, ql, hd, vec);
        to.load(dO, a.ldo, q0, ql, hd, vec);
        const bool in = t < QT && q0 + t < ql;
        const long long row = qrow0 + q0 + t;
        st[0] = in ? rel_lse2(a.lse[(size_t)h * a.lse_stride + row]) : INFINITY;       // (past the last query: probabilities of 0)
        st[1] = in ? a.d[(size_t)h * a.q_total_rows + row] : 0.f;
    };
    if (q_begin < ql) fetch(q_begin);
    float4 kf[NS], vf[NS];
    load_column<T, HD>((const T*)a.k + (krow0 + ki_c) * a.ldk + (long long)h * hd, hd, g, vec, kf);
    load_column<T, HD>((const T*)a.v + (krow0 + ki_c) * a.ldv + (long long)h * hd, hd, g, vec, vf);
    const float c = a.scale * kLog2eG;
    f32x4_t dk[NS], dv[NS];
#pragma unroll
    for (int i = 0; i < NS; ++i) { dk[i] = zero4(); dv[i] = zero4(); }
    fill.store(a, h, table);
    __syncthreads();
    const float side_bias[2] = {table[0], table[2 * (a.reach + kPad)]};
    const int near = a.reach + kPad + ki - pos - 4 * g;                // [query tile row e]: entry near - qb - e
    for (int q0 = q_begin; q0 < ql; q0 += QT) {
        __syncthreads();
        tq.store(sQ);
        to.store(sO);
        if (t < QT) {
            stat[t] = st[0];
            stat[QT + t] = st[1];
        }
        __syncthreads();
        if (q0 + QT < ql) fetch(q0 + QT);
        if (kw0 >= kl) continue;
#pragma unroll
        for (int i = 0; i < (QT / 16 + Share<COLS>::SPLITS - 1) / Share<COLS>::SPLITS; ++i) {
            const int qt = Share<COLS>::SPLITS * i + split, qb = q0 + 16 * qt;
            if (16 * qt >= QT || qb >= ql || (a.mask && pos + qb + 15 < kw0)) continue;       // no visible query
            f32x4_t p = first_product<HD>(sQ, 16 * qt, lane, kf);
            f32x4_t gr = first_product<HD>(sO, 16 * qt, lane, vf);
            const f32x4_t e2 = *reinterpret_cast<const f32x4_t*>(&stat[16 * qt + 4 * g]), d = *reinterpret_cast<const f32x4_t*>(&stat[QT + 16 * qt + 4 * g]);
            const int side = side_of(kw0 - pos - qb - 15, a.reach);
            const float flat = side < 0 ? side_bias[0] : side_bias[1];
#pragma unroll
            for (int e = 0; e < 4; ++e) p[e] = __builtin_fmaf(p[e], c, (side ? flat : table[near - qb - e]) - e2[e]);
            if (a.mask && pos + qb < kw0 + 15)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (pos + qb + 4 * g + e < ki) p[e] = -INFINITY;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                p[e] = __builtin_amdgcn_exp2f(p[e]);
                gr[e] = p[e] * (gr[e] - d[e]);
            }
            second_product<HD>(sO, 16 * qt, lane, p, dv);
            second_product<HD>(sQ, 16 * qt, lane, gr, dk);
        }
    }
    join_shares<COLS>(lds, split, t, dk);
    join_shares<COLS>(lds, split, t, dv);
    if (split != 0) return;
    if (a.mask && (any_not_finite(dk) || any_not_finite(dv))) {
        for (int i = 0; i < min(16, kl - kw0); ++i) rel_dkv_row<T>(a, s, h, kw0 + i, pos, ql, lane);
        return;
    }
    if (ki >= kl) return;
    store_column<T, HD>(dk, a.scale, (T*)a.dk + (krow0 + ki) * a.ldk + (long long)h * hd, hd, g, vec);
    store_column<T, HD>(dv, 1.0f, (T*)a.dv + (krow0 + ki) * a.ldv + (long long)h * hd, hd, g, vec);
}

constexpr int kAllLds = 160 * 1024;                     // (calls of a long reach ask for nearly as much)
template <class T, int HD> ds_status fwd_launch(const RelAttnArgs& a, hipStream_t st) {
    static std::atomic<uint64_t> allowed{0};
    auto kern = rel_fwd_kernel<T, HD>;
    const ds_status r = allow_dynamic_lds(kern, kAllLds, allowed);
    if (r != DS_OK) return r;
    const dim3 grid = a.k_splits > 1 ? dim3(a.k_splits, a.n_heads, a.n_seq) : column_grid(a, a.max_q_len, 64);
    hipLaunchKernelGGL(kern, grid, dim3(256), (2 * Tile<T, HD, 256>::FLOATS + table_floats(a.reach)) * 4, st, a);
    DS_LAUNCH_CHECK();
    return DS_OK;
}
template <class T, int HD, int COLS> ds_status dq_launch(const RelAttnArgs& a, hipStream_t st) {
    static std::atomic<uint64_t> allowed{0};
    auto kern = rel_bwd_dq_kernel<T, HD, COLS>;
    const ds_status r = allow_dynamic_lds(kern, kAllLds, allowed);
    if (r != DS_OK) return r;
    hipLaunchKernelGGL(kern, column_grid(a, a.max_q_len, COLS), dim3(512), (2 * Tile<T, HD, 512>::FLOATS + 9 * table_floats(a.reach)) * 4, st, a);
    DS_LAUNCH_CHECK();
    return DS_OK;
}
template <class T, int HD, int COLS> ds_status dkv_launch(const RelAttnArgs& a, int slot_cols, hipStream_t st) {
    static std::atomic<uint64_t> allowed{0};
    auto kern = rel_bwd_dkv_kernel<T, HD, COLS>;
    const ds_status r = allow_dynamic_lds(kern, kAllLds, allowed);
    if (r != DS_OK) return r;
    dim3 grid = column_grid(a, a.max_k_len, COLS);
    grid.z += 1;
    hipLaunchKernelGGL(kern, grid, dim3(512), (2 * Tile<T, HD, 512>::FLOATS + 2 * Tile<T, HD, 512>::ROWS + table_floats(a.reach)) * 4, st, a, slot_cols);
    DS_LAUNCH_CHECK();
    return DS_OK;
}
template <class T, int HD> ds_status bwd_launch(const RelAttnArgs& a, hipStream_t st) {
    const int q_cols = rel_general_columns(a, a.max_q_len), k_cols = rel_general_columns(a, a.max_k_len);
    const ds_status r = q_cols == 32 ? dq_launch<T, HD, 32>(a, st) : dq_launch<T, HD, 64>(a, st);
    if (r != DS_OK) return r;
    return k_cols == 32 ? dkv_launch<T, HD, 32>(a, q_cols, st) : dkv_launch<T, HD, 64>(a, q_cols, st);
}

template <class F> ds_status by_size(const RelAttnArgs& a, F&& f) {
    auto of = [&](auto zero) {
        if (a.head_dim <= 32) return f(zero, std::integral_constant<int, 32>{});
        if (a.head_dim <= 64) return f(zero, std::integral_constant<int, 64>{});
        if (a.head_dim <= 96) return f(zero, std::integral_constant<int, 96>{});
        return f(zero, std::integral_constant<int, 128>{});
    };
    return a.dtype == DS_DTYPE_BF16 ? of(bf16_t{}) : of(float{});
}

}  // namespace

int rel_general_columns(const RelAttnArgs& a, int max_len) {
    return a.head_dim <= 96 && (long long)a.n_seq * a.n_heads * (max_len / 64 + 1) <= 2LL * kRelUnits ? 32 : 64;
}

ds_status rel_join(const RelAttnArgs& a, hipStream_t st) {
    const dim3 grid((a.max_q_len + 3) / 4, a.n_heads, a.n_seq);
    if (a.dtype == DS_DTYPE_BF16) hipLaunchKernelGGL((rel_join_kernel<bf16_t>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((rel_join_kernel<float>), grid, dim3(256), 0, st, a);
    DS_LAUNCH_CHECK();
    return DS_OK;
}

ds_status rel_fwd_general(const RelAttnArgs& a, hipStream_t st) {
    const ds_status r = by_size(a, [&](auto zero, auto hd) { return fwd_launch<decltype(zero), decltype(hd)::value>(a, st); });
    return r != DS_OK || a.k_splits == 1 ? r : rel_join(a, st);
}

ds_status rel_bwd_general(const RelAttnArgs& a, hipStream_t st) {
    return by_size(a, [&](auto zero, auto hd) { return bwd_launch<decltype(zero), decltype(hd)::value>(a, st); });
}
