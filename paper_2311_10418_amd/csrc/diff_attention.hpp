// Arguments shared by the kernels of differential attention.
//
// Head h owns columns h * head_dim .. of q, k, v, o.  The first half of its q and k columns makes the scores of map 1, the second
// half those of map 2:  P_i = softmax(Q_i K_i^T / sqrt(head_dim / 2)),  O_2 = P_2 V,  O = P_1 V - lambda_h O_2.
// Backward, with G = dO V^T, D_2 = rowsum(dO O_2), D_1 = rowsum(dO O) + lambda_h D_2 (= rowsum(dO O_1)):
//     dS_1 = P_1 (G - D_1),  dS_2 = -lambda_h P_2 (G - D_2),  dQ_i = s dS_i K_i,  dK_i = s dS_i^T Q_i,
//     dV = (P_1 - lambda_h P_2)^T dO,  dlambda_h = - sum P_2 G.
// (dlambda is summed from the probabilities themselves, in fp32, and not from O_2, which is rounded to the tensors' type.)
#pragma once
#include "attention.hpp"
#include "common.hpp"

struct DiffAttnArgs : AttnArgs {                        // scale: 1 / sqrt(head_dim / 2); lse: [2 n_heads][lse_stride], map m of head h at row 2h + m
    const float* lambda;                                // [n_heads]
    void* o2;                                           // forward: NULL or where O_2 goes; backward: O_2
    float* dlambda;
    int32_t accumulate;
    float *d1, *d2;                                     // general kernels: D_1, D_2, [n_heads][q_total_rows]
    float* lam_part;                                    // sums of P_2 G of the queries of a wavefront, at the row of its first query
    int32_t vec;                                        // general kernels: rows of four elements may be accessed at once
    char* aug;                                          // matrix-core kernels: see diff_attention_bwd.hip
    int32_t k_splits;                                   // forward: work-groups that share the keys of a head (1: one has them all)
    int32_t direct;                                     // matrix-core kernels: sequences have one block of 128 rows, and work-groups go by sequence and head without a list
    float* split_part;                                  // what each of them found: see SplitPart
};

// Few short queries over long keys (single tokens on a cache): the keys of a sequence and head are dealt out to k_splits work-groups, in runs of
// whole tiles, and each leaves for every query its maxima and sums (exp2 domain) and its two unscaled outputs; diff_join_kernel puts them together.
struct SplitPart {
    float *stat, *o[2];                                 // {maximum 1, sum 1, maximum 2, sum 2}; [head_dim] each
};
__device__ __forceinline__ SplitPart split_part(const DiffAttnArgs& a, int h, long long row, int split) {
    float* p = a.split_part + ((size_t)(h * (long long)a.q_total_rows + row) * a.k_splits + split) * (2 * a.head_dim + 4);
    return {p, {p + 4, p + 4 + a.head_dim}};
}
// keys first .. first + count - 1 of kl are those of work-group `split`
struct KeyRange { int first, count; };
__device__ __forceinline__ KeyRange split_keys(const DiffAttnArgs& a, int kl, int split) {
    if (a.k_splits == 1) return {0, kl};
    const long long run = ((long long)kl + 64LL * a.k_splits - 1) / (64LL * a.k_splits) * 64, first = min(run * split, (long long)kl);
    return {(int)first, (int)min(run, kl - first)};
}
ds_status diff_join(const DiffAttnArgs& a, hipStream_t st);

// Compute units that the rules of choice count on: an MI355X's, and not those of the current device, since the scratch is sized by one of them.
constexpr int kDiffUnits = 256;
// What a call takes (see DiffChoice in diff_attention_api.hip): wavefronts that share a block of queries, whether there is no work list; columns of a work-group
int diff_mfma_sharing(const DiffAttnArgs& a);
bool diff_mfma_direct(const DiffAttnArgs& a, bool backward);
int diff_general_columns(const DiffAttnArgs& a, int max_len);

size_t diff_scratch_bytes(int n_heads, int q_total_rows, int k_total_rows, int n_seq);
ds_status diff_fwd_general(const DiffAttnArgs& a, hipStream_t st);
ds_status diff_bwd_general(const DiffAttnArgs& a, hipStream_t st);
// bf16 matrix-core kernels; what they do not take (see diff_mfma_supported) the general ones do
bool diff_mfma_supported(const DiffAttnArgs& a);
ds_status diff_fwd_mfma(const DiffAttnArgs& a, hipStream_t st);
ds_status diff_bwd_mfma(const DiffAttnArgs& a, hipStream_t st);
// dlambda[h] = (accumulate ? dlambda[h] : 0) - the sums in lam_part, which stand QUERIES rows apart within a sequence: a work-group of the dK/dV launch
// for each head, 16 threads for a sequence, in a fixed order.  (A launch of its own took 4 us.)
template <int QUERIES, int THREADS> __device__ __forceinline__ void sum_dlambda(const DiffAttnArgs& a, int h, float* lds) {
    const int lane = threadIdx.x & 15;
    const float* p = a.lam_part + (size_t)h * a.q_total_rows;
    float sum = 0.f;
#pragma unroll 4
    for (int s = threadIdx.x >> 4; s < a.n_seq; s += THREADS / 16) {
        const int n = (a.q_len[s] + QUERIES - 1) / QUERIES;
        const float* q = p + a.q_row[s];
        for (int i = lane; i < n; i += 16) sum += q[(size_t)i * QUERIES];
    }
    sum = wave_sum(sum);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x != 0) return;
    sum = 0.f;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) sum += lds[w];
    a.dlambda[h] = (a.accumulate ? a.dlambda[h] : 0.f) - sum;
}
