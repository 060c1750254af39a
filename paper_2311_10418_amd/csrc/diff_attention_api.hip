// C-ABI entry points and dispatch of differential attention.
#include "diff_attention.hpp"
#include "gemm.hpp"
#include <algorithm>
#include <cmath>

// Work-groups that share the keys of a head, for sequences of at most 64 queries in a tensor of at most 64 rows for each of them (the shares go to
// scratch by row of that tensor, whose lengths the scratch's size does not know): as many as make one for every compute unit, with a least
// number of keys each; two, which head sizes up to 64 have the LDS for, with more keys each; at most one for a lane of the wavefront that joins them.
// Matrix-core kernels: 128 keys, from 321 on (300 keys at once take 9.3 us, three shares of them and their joining 9.7); two from 1024 each on.
// General kernels: 64 keys, for two as well.  One query of 16 heads of 64, us without -> with, bf16 / fp32:
//     1 sequence of 512, 1024, 4096 keys:  15 -> 10, 24 -> 10, 77 -> 12 / 39 -> 11, 74 -> 11, 287 -> 22; of 32768 keys: 575 -> 37 (3.6 TB/s)
//     16 sequences of 2048, 16384 keys:  44 -> 33, 295 -> 195 (5.5 TB/s; one work-group for a compute unit: 37, 322)
//     16 sequences of 33 queries and 1019 keys:  28 -> 23 (two work-groups with half of them each: 29)
static constexpr int kSplitQueries = 64, kSplitMost = 64;
static int most_splits(bool general, int n_heads, int head_dim, int q_total_rows, int max_k_len, int n_seq) {
    const int from = general ? 129 : 321, keys_one = general ? 64 : 128, keys_two = general ? 64 : 1024;
    const long long items = (long long)n_seq * n_heads;
    if (q_total_rows > (long long)kSplitQueries * n_seq || max_k_len < from) return 1;
    auto with = [&](long long groups, int keys) {
        return std::min({groups / items, (long long)kSplitMost, ((long long)max_k_len + keys - 1) / keys});
    };
    const long long one = with(kDiffUnits, keys_one), two = head_dim <= 64 ? with(2 * kDiffUnits, keys_two) : 1;
    return (int)std::max<long long>(std::max(one, two), 1);
}

// Scratch: the work lists of the matrix-core kernels, then what the dQ kernels hand to the dK/dV kernels, 32 bytes for each query of a head
// (the general ones use 8 of them, as two arrays of floats), then the parts of dlambda, one float each.  A forward call has the parts of split keys in
// the place of both.
static size_t lists_size(int q_total_rows, int k_total_rows, int n_seq) { return attn_scratch_bytes(0, 0, q_total_rows, k_total_rows, n_seq); }
size_t diff_scratch_bytes(int n_heads, int q_total_rows, int k_total_rows, int n_seq) {
    size_t of_row = 32 + 4;
    for (const int head_dim : {64, 128}) {
        const int splits = most_splits(true, n_heads, head_dim, q_total_rows, k_total_rows, n_seq);      // (never fewer than the others)
        if (splits > 1) of_row = std::max(of_row, (size_t)splits * (2 * head_dim + 4) * 4);
    }
    return lists_size(q_total_rows, k_total_rows, n_seq) + (size_t)n_heads * q_total_rows * of_row;
}

static bool four_at_once(const void* p, size_t size) { return !p || (uintptr_t)p % (4 * size) == 0; }

static ds_status check(DiffAttnArgs& a) {
    if (a.n_seq <= 0 || a.n_heads <= 0 || a.head_dim <= 0 || a.head_dim > 128 || a.head_dim % 16) return DS_EINVAL;
    if (a.dtype != DS_DTYPE_F32 && a.dtype != DS_DTYPE_BF16) return DS_EINVAL;
    if (a.mask != 0 && a.mask != 1) return DS_EINVAL;
    if (!a.q_row || !a.q_len || !a.k_row || !a.k_len || !a.q || !a.k || !a.v || !a.lambda || !a.o || !a.lse) return DS_EINVAL;
    if (a.max_q_len <= 0 || a.max_k_len <= 0 || a.q_total_rows <= 0 || a.k_total_rows <= 0) return DS_EINVAL;
    if (a.n_seq > 65534 || a.n_heads > 65535) return DS_EINVAL;
    const long long wide = (long long)a.n_heads * a.head_dim;
    if (a.ldq < wide || a.ldk < wide || a.ldv < wide || a.ldo < wide) return DS_EINVAL;
    if (!a.scratch || (uintptr_t)a.scratch % 16 || a.scratch_bytes < diff_scratch_bytes(a.n_heads, a.q_total_rows, a.k_total_rows, a.n_seq)) return DS_EINVAL;
    a.max_q_len = std::min(a.max_q_len, a.q_total_rows);
    a.max_k_len = std::min(a.max_k_len, a.k_total_rows);
    const size_t size = dtype_size(a.dtype);
    for (const void* p : {a.q, a.k, a.v, (const void*)a.o, (const void*)a.o2, a.d_o, (const void*)a.dq, (const void*)a.dk, (const void*)a.dv})
        if ((uintptr_t)p % size) return DS_EINVAL;
    a.vec = four_at_once(a.q, size) && four_at_once(a.k, size) && four_at_once(a.v, size) && four_at_once(a.o, size) && four_at_once(a.o2, size) &&
            four_at_once(a.d_o, size) && four_at_once(a.dq, size) && four_at_once(a.dk, size) && four_at_once(a.dv, size) &&
            a.ldq % 4 == 0 && a.ldk % 4 == 0 && a.ldv % 4 == 0 && a.ldo % 4 == 0;
    a.scale = 1.0f / sqrtf((float)(a.head_dim / 2));
    char* after_lists = (char*)a.scratch + lists_size(a.q_total_rows, a.k_total_rows, a.n_seq);
    const size_t entries = (size_t)a.n_heads * a.q_total_rows;
    a.aug = after_lists;
    a.d1 = (float*)after_lists;
    a.d2 = a.d1 + entries;
    a.k_splits = 1;
    a.n_items = (const int32_t*)a.scratch;              // (valid memory also where no list is made)
    a.split_part = (float*)after_lists;
    a.lam_part = (float*)(after_lists + entries * 32);
    return DS_OK;
}

// How a call goes to the kernels: fp32 arithmetic or bf16 matrix cores; bf16: whether there is no work list, wavefronts that share a block of queries; both:
// work-groups that share a head's keys (forward); fp32 backward: columns of a work-group of the dQ and of the dK/dV kernel.
struct DiffChoice { int32_t general, direct, sharing, k_splits, dq_columns, dkv_columns; };
static DiffChoice choose(const DiffAttnArgs& a, bool backward, bool force_generic) {
    DiffChoice c = {force_generic || !diff_mfma_supported(a), 0, 1, 1, 64, 64};
    if (!c.general) {
        c.direct = diff_mfma_direct(a, backward);
        c.sharing = diff_mfma_sharing(a);
    }
    if (backward) {
        c.dq_columns = diff_general_columns(a, a.max_q_len);
        c.dkv_columns = diff_general_columns(a, a.max_k_len);
    } else if (!a.mask && a.max_q_len <= kSplitQueries && (c.general || c.sharing > 1)) {
        c.k_splits = most_splits(c.general, a.n_heads, a.head_dim, a.q_total_rows, a.max_k_len, a.n_seq);
    }
    return c;
}
// the general kernels: 64 tokens to a work-group of 512 threads, fewer than 2^32 of them along a sequence
static bool too_long(const DiffAttnArgs& a) { return std::max(a.max_q_len, a.max_k_len) > 1 << 28; }
// For tests: what `choose` says of a call whose tensors have the least strides and are aligned, in the order of DiffChoice.  Not part of the C ABI's header.
extern "C" void ds_diff_attention_choice(int32_t dtype, int32_t n_seq, int32_t n_heads, int32_t head_dim, int32_t mask, int32_t max_q_len, int32_t max_k_len,
                                         int32_t q_total_rows, int32_t k_total_rows, int32_t backward, int32_t force_generic, int32_t* out) {
    DiffAttnArgs a = {};
    a.dtype = dtype; a.n_seq = n_seq; a.n_heads = n_heads; a.head_dim = head_dim; a.mask = mask;
    a.max_q_len = std::min(max_q_len, q_total_rows); a.max_k_len = std::min(max_k_len, k_total_rows);
    a.q_total_rows = q_total_rows; a.k_total_rows = k_total_rows;
    a.ldq = a.ldk = a.ldv = a.ldo = (long long)n_heads * head_dim;
    const DiffChoice c = choose(a, backward != 0, force_generic != 0);
    for (const int32_t v : {c.general, c.direct, c.sharing, c.k_splits, c.dq_columns, c.dkv_columns}) *out++ = v;
}

extern "C" int64_t ds_diff_attention_scratch_bytes(int32_t n_heads, int32_t q_total_rows, int32_t k_total_rows, int32_t n_seq) {
    if (n_heads <= 0 || q_total_rows <= 0 || k_total_rows <= 0 || n_seq <= 0) return 0;
    return (int64_t)diff_scratch_bytes(n_heads, q_total_rows, k_total_rows, n_seq);
}

extern "C" ds_status ds_diff_attention_fwd(int32_t dtype, int32_t n_seq, int32_t n_heads, int32_t head_dim, int32_t mask, const int32_t* q_row,
                                           const int32_t* q_len, const int32_t* k_row, const int32_t* k_len, int32_t max_q_len, int32_t max_k_len,
                                           const void* q, int32_t ldq, const void* k, int32_t ldk, const void* v, int32_t ldv, const float* lambda,
                                           void* o, void* o2, int32_t ldo, float* lse, int32_t q_total_rows, int32_t k_total_rows, void* scratch,
                                           int64_t scratch_bytes, int32_t force_generic, void* hip_stream) {
    DiffAttnArgs a = {};
    a.dtype = dtype; a.n_seq = n_seq; a.n_heads = n_heads; a.head_dim = head_dim; a.mask = mask;
    a.q_row = q_row; a.q_len = q_len; a.k_row = k_row; a.k_len = k_len;
    a.max_q_len = max_q_len; a.max_k_len = max_k_len;
    a.q = q; a.k = k; a.v = v; a.ldq = ldq; a.ldk = ldk; a.ldv = ldv;
    a.lambda = lambda;
    a.o = o; a.o2 = o2; a.ldo = ldo; a.lse = lse; a.lse_stride = q_total_rows;
    a.q_total_rows = q_total_rows; a.k_total_rows = k_total_rows;
    a.scratch = scratch; a.scratch_bytes = scratch_bytes < 0 ? 0 : (size_t)scratch_bytes;
    const ds_status r = check(a);
    if (r != DS_OK) return r;
    const DiffChoice c = choose(a, false, force_generic != 0);
    if (c.general && too_long(a)) return DS_EINVAL;
    a.k_splits = c.k_splits;
    if (!c.general) return diff_fwd_mfma(a, (hipStream_t)hip_stream);
    return diff_fwd_general(a, (hipStream_t)hip_stream);
}

extern "C" ds_status ds_diff_attention_bwd(int32_t dtype, int32_t n_seq, int32_t n_heads, int32_t head_dim, int32_t mask, const int32_t* q_row,
                                           const int32_t* q_len, const int32_t* k_row, const int32_t* k_len, int32_t max_q_len, int32_t max_k_len,
                                           const void* q, int32_t ldq, const void* k, int32_t ldk, const void* v, int32_t ldv, const float* lambda,
                                           const void* o, const void* o2, const void* d_o, int32_t ldo, const float* lse, void* dq, void* dk, void* dv,
                                           float* dlambda, int32_t accumulate, int32_t q_total_rows, int32_t k_total_rows, void* scratch,
                                           int64_t scratch_bytes, int32_t force_generic, void* hip_stream) {
    DiffAttnArgs a = {};
    a.dtype = dtype; a.n_seq = n_seq; a.n_heads = n_heads; a.head_dim = head_dim; a.mask = mask;
    a.q_row = q_row; a.q_len = q_len; a.k_row = k_row; a.k_len = k_len;
    a.max_q_len = max_q_len; a.max_k_len = max_k_len;
    a.q = q; a.k = k; a.v = v; a.ldq = ldq; a.ldk = ldk; a.ldv = ldv;
    a.lambda = lambda;
    a.o = const_cast<void*>(o); a.o2 = const_cast<void*>(o2); a.d_o = d_o; a.ldo = ldo;
    a.lse = const_cast<float*>(lse); a.lse_stride = q_total_rows;
    a.dq = dq; a.dk = dk; a.dv = dv; a.dlambda = dlambda; a.accumulate = accumulate;
    a.q_total_rows = q_total_rows; a.k_total_rows = k_total_rows;
    a.scratch = scratch; a.scratch_bytes = scratch_bytes < 0 ? 0 : (size_t)scratch_bytes;
    const ds_status r = check(a);
    if (r != DS_OK) return r;
    if (!o2 || !d_o || !dq || !dk || !dv || !dlambda || (accumulate != 0 && accumulate != 1)) return DS_EINVAL;
    if (!choose(a, true, force_generic != 0).general) return diff_bwd_mfma(a, (hipStream_t)hip_stream);
    if (too_long(a)) return DS_EINVAL;
    return diff_bwd_general(a, (hipStream_t)hip_stream);
}
