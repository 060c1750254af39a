// Arguments shared by the kernels of attention with a learned relative position bias.
//
// Query i of a sequence stands at position p_i = q_pos + i, key j at position j.  With b(d) = bias[bucket[clamp(d, -reach, reach) + reach]][h], the bias of
// head h at distance d = j - p_i:
//     S = s Q K^T + b(j - p_i)   (mask 1: -inf where j > p_i),   P = softmax(S),   O = P V,   lse = log sum exp S.
// Backward, D = rowsum(dO O) with O as it is stored:
//     dS = P (dO V^T - D),  dQ = s dS K,  dK = s dS^T Q,  dV = P^T dO,  dbias[c][h] = sum of dS over the pairs whose distance has bucket c.
// A row that sees no key (none there, all hidden by the mask, or by biases of -inf) has O = 0, lse = -inf, and no gradient.
//
// Beyond `reach` the bias is one number on each side, so that only blocks of pairs near the diagonal look anything up: by distance, in a table in LDS that
// holds the bias of one head in the exp2 domain.  What dbias sums goes by distance too, first in LDS, then to one slot in the scratch for each block of queries
// (sum_dbias puts the slots together, in a fixed order): no atomics whose order could change a result.
#pragma once
#include "attention.hpp"
#include "common.hpp"

struct RelAttnArgs : AttnArgs {
    const void* bias;                                   // [n_buckets][n_heads], of the tensors' type
    const int32_t* bucket;                              // [2 reach + 1]
    int32_t n_buckets, reach;
    const int32_t* q_pos;                               // [n_seq] or NULL: zeros
    float* dbias;                                       // [n_buckets][n_heads]
    int32_t accumulate;
    int32_t vec;                                        // general kernels: rows of four elements may be accessed at once
    int32_t k_splits;                                   // forward: work-groups that share the keys of a head (1: one has them all)
    float* d;                                           // general kernels: D, [n_heads][q_total_rows]
    float* slots;                                       // sums of dS by distance, [block of queries][n_heads][2 reach + 1]
    float* split_part;                                  // see RelPart
    int32_t b_splits;                                   // backward, matrix-core kernels: work-groups that share the keys (queries) of a block of queries (keys), and where they leave
    float *part_q, *part_k;                             // their sums: dQ [share][q_total_rows][wide], dK and dV [share][k_total_rows][2][wide], wide = n_heads * head_dim
    char* aug;                                          // matrix-core kernels: what the dQ kernel hands to the dK/dV kernel
    int32_t direct, direct_k;                           // matrix-core kernels: blocks of 128 queries / keys that a sequence may have, and work-groups go by them; 0: by a list
    int32_t first_group, groups;                        // dK/dV grid: work-groups in front that sum up dbias, work-groups behind them
};

constexpr int kRelShares = 8;                           // most work-groups that share a block of 128 rows in the matrix-core kernels
// Work-groups that share the keys of a sequence and head leave, for each query, its maximum (exp2 domain), sum and unscaled output.
struct RelPart { float *stat, *o; };
__device__ __forceinline__ RelPart rel_part(const RelAttnArgs& a, int h, long long row, int split) {
    float* p = a.split_part + ((size_t)(h * (long long)a.q_total_rows + row) * a.k_splits + split) * (a.head_dim + 4);
    return {p, p + 4};
}
ds_status rel_join(const RelAttnArgs& a, hipStream_t st);

// Position of a sequence's first query.  Lengths stay below 2^28 and reach below 2^11, so that what lies beyond 2^30 may as well lie there.
__device__ __forceinline__ int rel_position(const RelAttnArgs& a, int s) { return a.q_pos ? min(max(a.q_pos[s], -(1 << 30)), 1 << 30) : 0; }
// keys of a sequence that its last query sees
__device__ __forceinline__ int rel_keys(const RelAttnArgs& a, int kl, int ql, int pos) { return a.mask ? min(kl, max(0, pos + ql)) : kl; }
// bias of head h at table entry i = distance + reach, clamped, in the exp2 domain
__device__ __forceinline__ float rel_bias(const RelAttnArgs& a, int h, int i) {
    const int b = min(max(a.bucket[min(max(i, 0), 2 * a.reach)], 0), a.n_buckets - 1);
    const size_t at = (size_t)b * a.n_heads + h;
    return 1.4426950408889634f * (a.dtype == DS_DTYPE_BF16 ? (float)((const bf16_t*)a.bias)[at] : ((const float*)a.bias)[at]);
}
// log-sum-exp as the backward kernels subtract it (exp2 domain): rows that see nothing get probabilities of 0
__device__ __forceinline__ float rel_lse2(float lse) { return lse == -INFINITY ? INFINITY : lse * 1.4426950408889634f; }

// lds[i] += v without a return, by the lanes of one wavefront and with no two of them at one address: LDS operations of a wavefront take effect in order, so
// that the sum does not depend on timing as long as other wavefronts keep off it
__device__ __forceinline__ void lds_add(float* lds, float v) {
    __builtin_amdgcn_ds_faddf((__attribute__((address_space(3))) float*)lds, v, 0, 0, false);
}

// v of the lane N above (row_shl) or below (row_shr) within each 16 lanes, 0 where there is none: rides on the addition that uses it
template <int N> __device__ __forceinline__ float lanes_above(float v) {
    if constexpr (N == 0) return v;
    else return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0x100 + N, 0xf, 0xf, true));
}
template <int N> __device__ __forceinline__ float lanes_below(float v) {
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0x110 + N, 0xf, 0xf, true));
}
// Sums along the diagonals of a block whose columns are 16 lanes: the value of row r (a constant) in lane c belongs to distance r - c, which is -d for the lane d
// that it is shifted to where d = c - r is a lane, and 16 - d where it comes in again at the other end.
template <int R> __device__ __forceinline__ void add_diagonals(float x, float& minus, float& around) {
    minus += lanes_above<R>(x);
    if constexpr (R != 0) around += lanes_below<16 - R>(x);
}

// blocks of `cols` queries of all sequences before s (slots are numbered by sequence): this thread's part, and the sum of all
template <int COLS, int THREADS> __device__ __forceinline__ int blocks_part(const RelAttnArgs& a, int s) {
    int n = 0;
    for (int i = threadIdx.x; i < s; i += THREADS) n += max(a.q_len[i] + COLS - 1, 0) / COLS;
    return n;
}
template <int THREADS> __device__ __forceinline__ int blocks_sum(int n, int* lds) {
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) n += __shfl_xor(n, m, 64);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = n;
    __syncthreads();
    n = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) n += lds[w];
    __syncthreads();
    return n;
}
// dbias[.][h] = (accumulate ? itself : 0) + the sums in n slots, in a fixed order: a work-group of the dK/dV launch for each head.  Up to 320 distances each wavefront
// takes every so-manieth slot, five distances a lane; more go by thread.  Eight threads to a bucket then look for its distances.  (With a thread to a distance and to a
// bucket this took 12 us of every backward call.)  lds: 2 reach + 1 pairs and, up to 320, as many floats for each wavefront.
template <int THREADS> __device__ __forceinline__ void sum_dbias(const RelAttnArgs& a, int h, int n, float* lds) {
    constexpr int WAVES = THREADS / 64, MOST = 5;
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6, w = 2 * a.reach + 1;
    const size_t step = (size_t)a.n_heads * w;
    const float* from = a.slots + (size_t)h * w;
    const bool shared = w <= 64 * MOST;
    float2* pair = reinterpret_cast<float2*>(lds + (shared ? WAVES * w : 0));
    if (shared) {
        float sum[MOST];
#pragma unroll
        for (int j = 0; j < MOST; ++j) sum[j] = 0.f;
#pragma unroll 4
        for (int k = wave; k < n; k += WAVES)
#pragma unroll
            for (int j = 0; j < MOST; ++j) sum[j] += from[(size_t)k * step + min(lane + 64 * j, w - 1)];
#pragma unroll
        for (int j = 0; j < MOST; ++j)
            if (lane + 64 * j < w) lds[wave * w + lane + 64 * j] = sum[j];
        __syncthreads();
    }
    for (int i = t; i < w; i += THREADS) {
        float sum = 0.f;
        if (shared) {
#pragma unroll
            for (int j = 0; j < WAVES; ++j) sum += lds[j * w + i];
        } else {
#pragma unroll 8
            for (int k = 0; k < n; ++k) sum += from[(size_t)k * step + i];
        }
        pair[i] = make_float2(sum, __builtin_bit_cast(float, min(max(a.bucket[i], 0), a.n_buckets - 1)));
    }
    __syncthreads();
    for (int b0 = 0; b0 < a.n_buckets; b0 += THREADS / 8) {
        const int b = b0 + (t >> 3);
        float sum = 0.f;
#pragma unroll 8
        for (int i = t & 7; i < w; i += 8) {
            const float2 x = pair[i];
            sum += __builtin_bit_cast(int, x.y) == b ? x.x : 0.f;
        }
#pragma unroll
        for (int m = 1; m < 8; m *= 2) sum += __shfl_xor(sum, m, 64);
        if ((t & 7) == 0 && b < a.n_buckets) {
            float* to = a.dbias + (size_t)b * a.n_heads + h;
            *to = (a.accumulate ? *to : 0.f) + sum;
        }
    }
}

// Compute units that the rules of choice count on: an MI355X's, and not those of the current device, since the scratch is sized by one of them.
constexpr int kRelUnits = 256;
int rel_general_columns(const RelAttnArgs& a, int max_len);

ds_status rel_fwd_general(const RelAttnArgs& a, hipStream_t st);
ds_status rel_bwd_general(const RelAttnArgs& a, hipStream_t st);
// bf16 matrix-core kernels; what they do not take (see rel_mfma_supported) the general ones do
bool rel_mfma_supported(const RelAttnArgs& a);
ds_status rel_fwd_mfma(const RelAttnArgs& a, hipStream_t st);
ds_status rel_bwd_mfma(const RelAttnArgs& a, hipStream_t st);
// one query to a sequence, rows of 16-byte pieces (rel_attention_few.hip); keys that a work-group takes at a time
bool rel_few_supported(const RelAttnArgs& a);
ds_status rel_fwd_few(const RelAttnArgs& a, hipStream_t st);
constexpr int rel_few_lanes(int32_t dtype, int head_dim) {                  // lanes that hold a row: a power of two
    int n = 4;
    while (n * (dtype == DS_DTYPE_BF16 ? 8 : 4) < head_dim) n *= 2;
    return n;
}
constexpr int rel_few_keys(int32_t dtype, int head_dim) { return 2048 / rel_few_lanes(dtype, head_dim); }
