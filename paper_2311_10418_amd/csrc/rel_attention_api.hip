// C-ABI entry points and dispatch of attention with a relative position bias.
#include "rel_attention.hpp"
#include <algorithm>
#include <cmath>

constexpr int kRelReach = 1024, kRelBuckets = 1024, kRelLongest = 1 << 28;

// Work-groups that share the keys of a head, for sequences of at most 64 queries in a tensor of at most 64 rows for each of them (the shares go to scratch
// by row of that tensor, whose lengths the scratch's size does not know): from 129 keys on, 64 at least each, at most one for a lane of the wavefront that joins them;
// matrix-core kernels as many as make two for every compute unit at head size 64, one at 128; general ones three.
// Tokens on a cache, 16 heads, us, 1 / 2 / 3 / 4 to a compute unit: bf16, heads of 64, 16 sequences of 1 019 keys, one query  - / 19.0 / 17.6 / 20.9, of 16 384  - / 206 / 213 / 266,
// one of 32 768  - / 32 / 36 / 43; heads of 128, 25.5 / 29.2 / 30.1 / 31.2, 431 / 390 / 435 / 387, 49 / 52 / 57 / 62; fp32, four queries, 1 019 keys: heads of 64  - / 41 / 36 / 44, of 128
// 106 / 65 / 56 / 69.  (With a join that took shares beyond 16 one by one: at one of 32 768 it is 29 now, not 32.)
static constexpr int kSplitQueries = 64, kSplitMost = 64;
static int most_splits(bool general, int n_heads, int head_dim, int q_total_rows, int max_k_len, int n_seq) {
    const long long items = (long long)n_seq * n_heads;
    if (q_total_rows > (long long)kSplitQueries * n_seq || max_k_len < 129) return 1;
    const long long groups = (general ? 3 : head_dim <= 64 ? 2 : 1) * kRelUnits;
    return (int)std::max(1LL, std::min({groups / items, (long long)kSplitMost, ((long long)max_k_len + 63) / 64}));
}
// The kernel for single queries: its work-groups take rel_few_keys keys at a time, and four of them to a compute unit wait for memory together.
static int few_splits(int32_t dtype, int n_heads, int head_dim, int q_total_rows, int max_q_len, int max_k_len, int n_seq) {
    if (q_total_rows > (long long)kSplitQueries * n_seq) return 1;
    const long long items = (long long)n_seq * n_heads * max_q_len, keys = rel_few_keys(dtype, head_dim);
    return (int)std::max(1LL, std::min({4LL * kRelUnits / items, (long long)kSplitMost, ((long long)max_k_len + keys - 1) / keys}));
}

// The matrix-core kernels where blocks of 128 rows are few: work-groups that may share a block (the scratch has room for as many), four blocks of 64 of the other side each at least,
// 56 MiB of sums at most.
static constexpr int kShareGroups = 3 * kRelUnits;
static constexpr long long kShareBytes = 56LL << 20;
static long long share_groups(int n_heads, int q_total_rows, int k_total_rows, int n_seq) {
    return ((long long)std::max(q_total_rows, k_total_rows) / 128 + n_seq) * n_heads;
}
static int most_back_splits(int n_heads, int head_dim, int q_total_rows, int k_total_rows, int longest, int n_seq) {
    const long long bytes = 4 * (q_total_rows + 2LL * k_total_rows) * n_heads * head_dim;
    return (int)std::max(1LL, std::min({kShareGroups / share_groups(n_heads, q_total_rows, k_total_rows, n_seq), (long long)kRelShares, (long long)longest / 256, kShareBytes / bytes}));
}
// Forward with more than 64 queries, bf16: as many shares of the keys as an estimate prefers by a tenth: a work-group takes 4 us and `step` for each block of 64 keys, each more on a compute unit 0.45
// of one alone; under a causal mask half as long on average; the shares are written, read and joined.
// Measured, us, with 1 / 2 / 3 / 4 / most shares (sequences x length, heads of size, c: causal; *: chosen): 1 x 1 565, 4 of 128 c 33 / 26 / *23 / 23 / 24; 1 x 8 192, 2 of 64 c 109 / 67 / 50 / 43 / *40; 1 x 4 096,
// 8 of 128 c 80 / *65; 1 x 1 024, 4 of 128 24 / 20 / 19 / *18; 4 x 600, 9 of 128 *21 / 30; 2 x 1 181, 16 of 64 c *22 / 29; 1 x 2 048, 16 of 128 c *44 / 43; 1 x 512, 4 of 64 *12.7 / 11.7.
static int most_fwd_splits(int n_heads, int head_dim, int q_total_rows, int max_k_len, int n_seq) {
    const long long bytes = 4LL * q_total_rows * n_heads * (head_dim + 4);
    return (int)std::max(1LL, std::min({kShareGroups / share_groups(n_heads, q_total_rows, 0, n_seq), (long long)kRelShares, (long long)max_k_len / 256, kShareBytes / bytes}));
}
static int fwd_splits(const RelAttnArgs& a) {
    const int most = most_fwd_splits(a.n_heads, a.head_dim, a.q_total_rows, a.max_k_len, a.n_seq), steps = (a.max_k_len + 63) / 64;
    const double groups = (double)share_groups(a.n_heads, a.q_total_rows, 0, a.n_seq), step = a.head_dim == 64 ? 0.85 : 1.15;
    const double part_us = 2.0 * 4 * a.q_total_rows * a.n_heads * (a.head_dim + 4) / 4.5e6;
    double alone = 0, least = 0;
    int best = 1;
    for (int s = 1; s <= most; ++s) {
        const double chain = step * ((steps + s - 1) / s) + 4, each = groups * s / kRelUnits;
        double cost = (0.55 + 0.45 * std::max(1.0, std::ceil(each))) * chain;
        if (a.mask) cost = std::max(chain, (0.55 + 0.45 * std::max(1.0, each)) * (4 + 0.5 * step * steps / s));
        if (s == 1) alone = least = cost;
        else if (cost += 4 + s * part_us; cost < least && cost < 0.9 * alone) least = cost, best = s;
    }
    return best;
}
// As many as an estimate of dQ and dK/dV together prefers by a tenth: a work-group takes `fixed` us and `step` for each block of 64 of the other side; one to a compute unit at head size
// 128, at 64 two in 1.6 times the time of one; under a causal mask chains are half as long on average.  Shares are joined in a launch of their own (rel_back_join_kernel).
// Measured, us, with 1 / 2 / 3 / 4 / most shares (sequences x length, heads of size, c: causal; *: chosen): 1 x 1 565, 4 of 128 c 97 / 72 / 61 / 57 / 56 (five: *54); 1 x 1 972, 3 of 64 c 80 / 54 / 45 /
// 41 / 40 (five: *39); 3 x 1 193, 5 of 128 c 83 / *79 / 88 / 95; 2 x 1 181, 16 of 64 c *62 / 66; 1 x 1 024, 16 of 128 *72 / 69 / 88; 4 x 600, 9 of 128 *58 / 86; 1 x 8 192, 2 of 64 c 286 / 163 / 126 / *109 / 103; 1 x 4 096,
// 8 of 128 c *224 / 177 / 175 (beyond 56 MiB); 1 x 512, 4 of 64 31 / *26; 1 x 2 048, 16 of 128 c *124 / 118 / 116.
static int back_splits(const RelAttnArgs& a) {
    const int longest = std::max(a.max_q_len, a.max_k_len), most = most_back_splits(a.n_heads, a.head_dim, a.q_total_rows, a.k_total_rows, longest, a.n_seq);
    const double groups = (double)share_groups(a.n_heads, a.q_total_rows, a.k_total_rows, a.n_seq), step = a.head_dim == 64 ? 2.2 : 3.05, fixed = a.head_dim == 64 ? 14 : 20;
    const double pair = a.head_dim == 64 ? 1.6 : 2, part_us = 4 * ((double)a.q_total_rows + 2.0 * a.k_total_rows) * a.n_heads * a.head_dim / 4.5e6;
    const int steps = (longest + 63) / 64;
    double alone = 0, least = 0;
    int best = 1;
    for (int s = 1; s <= most; ++s) {
        const double chain = step * ((steps + s - 1) / s) + fixed, each = groups * s / kRelUnits;              // work-groups to a compute unit
        double cost;
        if (a.mask) {
            cost = std::max(chain, each * pair / 2 * (fixed + 0.5 * step * steps / s));
        } else {
            const int rounds = (int)std::ceil(each);
            cost = (rounds / 2 * pair + rounds % 2) * chain;
        }
        if (s == 1) alone = least = cost;
        else if (cost += 4 + s * part_us; cost < least && cost < 0.9 * alone) least = cost, best = s;
    }
    return best;
}

// Scratch: the work lists of the matrix-core kernels; what the dQ kernels hand to the dK/dV kernels, 32 bytes for each query of a head (the general ones use 4 of
// them); the slots of dbias, for each share of each block of 64 queries (of 32 where the general kernels have at most 512 work-groups of 64); what shares of a block leave.  A forward call has the parts of
// split keys in the place of the last two.
static size_t lists_size(int q_total_rows, int k_total_rows, int n_seq) { return attn_scratch_bytes(0, 0, q_total_rows, k_total_rows, n_seq); }
static size_t slots_size(int n_heads, int q_total_rows, int n_seq, int reach, int shares) {
    const size_t blocks = std::max(((size_t)q_total_rows / 64 + n_seq) * n_heads * shares, (size_t)4 * kRelUnits);
    return (blocks * (2 * reach + 1) * 4 + 15) & ~(size_t)15;
}
static size_t rel_scratch_bytes(int n_heads, int head_dim, int reach, int q_total_rows, int k_total_rows, int n_seq) {
    const size_t entries = (size_t)n_heads * q_total_rows;
    const int shares = most_back_splits(n_heads, head_dim, q_total_rows, k_total_rows, std::max(q_total_rows, k_total_rows), n_seq);
    const size_t parts = shares > 1 ? (size_t)shares * ((size_t)q_total_rows + 2 * (size_t)k_total_rows) * n_heads * head_dim * 4 : 0;
    const size_t backward = entries * 32 + slots_size(n_heads, q_total_rows, n_seq, reach, shares) + parts;
    const int splits = std::max({most_splits(true, n_heads, head_dim, q_total_rows, k_total_rows, n_seq), most_fwd_splits(n_heads, head_dim, q_total_rows, k_total_rows, n_seq),
                                 few_splits(DS_DTYPE_F32, n_heads, head_dim, q_total_rows, 1, k_total_rows, n_seq)});    // (never fewer than the others)
    const size_t forward = splits > 1 ? entries * splits * (head_dim + 4) * 4 : 0;
    return lists_size(q_total_rows, k_total_rows, n_seq) + std::max(backward, forward);
}

static bool four_at_once(const void* p, size_t size) { return !p || (uintptr_t)p % (4 * size) == 0; }

static ds_status check(RelAttnArgs& a) {
    if (a.n_seq <= 0 || a.n_heads <= 0 || a.head_dim <= 0 || a.head_dim > 128 || a.head_dim % 8) return DS_EINVAL;
    if (a.dtype != DS_DTYPE_F32 && a.dtype != DS_DTYPE_BF16) return DS_EINVAL;
    if (a.mask != 0 && a.mask != 1) return DS_EINVAL;
    if (!a.q_row || !a.q_len || !a.k_row || !a.k_len || !a.q || !a.k || !a.v || !a.bias || !a.bucket || !a.o || !a.lse) return DS_EINVAL;
    if (a.reach < 1 || a.reach > kRelReach || a.n_buckets < 1 || a.n_buckets > kRelBuckets) return DS_EINVAL;
    if (!(a.scale > 0.f) || std::isinf(a.scale * 1.4426950408889634f)) return DS_EINVAL;        // (the kernels multiply scores by this; infinite, it makes NaN of a score of 0)
    if (a.max_q_len <= 0 || a.max_k_len <= 0 || a.q_total_rows <= 0 || a.k_total_rows <= 0) return DS_EINVAL;
    if (a.n_seq > 65534 || a.n_heads > 65535) return DS_EINVAL;
    const long long wide = (long long)a.n_heads * a.head_dim;
    if (a.ldq < wide || a.ldk < wide || a.ldv < wide || a.ldo < wide) return DS_EINVAL;
    if (!a.scratch || (uintptr_t)a.scratch % 16 ||
        a.scratch_bytes < rel_scratch_bytes(a.n_heads, a.head_dim, a.reach, a.q_total_rows, a.k_total_rows, a.n_seq)) return DS_EINVAL;
    a.max_q_len = std::min(a.max_q_len, a.q_total_rows);
    a.max_k_len = std::min(a.max_k_len, a.k_total_rows);
    if (std::max(a.max_q_len, a.max_k_len) > kRelLongest) return DS_EINVAL;
    const size_t size = dtype_size(a.dtype);
    for (const void* p : {a.q, a.k, a.v, (const void*)a.o, a.d_o, (const void*)a.dq, (const void*)a.dk, (const void*)a.dv, a.bias})
        if ((uintptr_t)p % size) return DS_EINVAL;
    a.vec = four_at_once(a.q, size) && four_at_once(a.k, size) && four_at_once(a.v, size) && four_at_once(a.o, size) && four_at_once(a.d_o, size) &&
            four_at_once(a.dq, size) && four_at_once(a.dk, size) && four_at_once(a.dv, size) && a.ldq % 4 == 0 && a.ldk % 4 == 0 && a.ldv % 4 == 0 && a.ldo % 4 == 0;
    char* after_lists = (char*)a.scratch + lists_size(a.q_total_rows, a.k_total_rows, a.n_seq);
    const size_t entries = (size_t)a.n_heads * a.q_total_rows;
    a.k_splits = a.b_splits = 1;
    a.aug = after_lists;
    a.d = (float*)after_lists;
    a.slots = (float*)(after_lists + entries * 32);
    a.split_part = (float*)after_lists;
    a.n_items = (const int32_t*)a.scratch;              // (valid memory also where no list is made)
    return DS_OK;
}

// Blocks of 128 rows that each of the sequences may have, if a grid of all of them is at most a quarter larger than one that goes by a list (and has no more than
// there are slots for); otherwise 0.
static int blocks_without_list(int max_len, int total_rows, int n_seq) {
    const long long blocks = ((long long)max_len + 127) / 128, all = blocks * n_seq;
    return all <= (long long)total_rows / 64 + n_seq && 4 * all <= 5 * ((long long)total_rows / 128 + n_seq) ? (int)blocks : 0;
}

// How a call goes to the kernels: fp32 arithmetic or bf16 matrix cores; work-groups that share a head's keys (forward); bf16: whether there is no work list; the
// kernel for few queries instead (forward); work-groups that share a block (backward)
struct RelChoice { int32_t general, k_splits, direct, few, b_splits; };
static RelChoice choose(RelAttnArgs& a, bool backward, bool force_generic) {
    RelChoice c = {1, 1, 0, 0, 1};
    if (!backward && !force_generic && rel_few_supported(a) && !rel_mfma_supported(a)) {
        c.few = 1;
        c.k_splits = a.k_splits = few_splits(a.dtype, a.n_heads, a.head_dim, a.q_total_rows, a.max_q_len, a.max_k_len, a.n_seq);
        return c;
    }
    c.general = force_generic || !rel_mfma_supported(a);
    if (!backward && a.max_q_len <= kSplitQueries) c.k_splits = most_splits(c.general, a.n_heads, a.head_dim, a.q_total_rows, a.max_k_len, a.n_seq);
    if (!c.general && !backward && a.max_q_len > kSplitQueries) c.k_splits = fwd_splits(a);
    a.k_splits = c.k_splits;
    if (!c.general) c.direct = blocks_without_list(a.max_q_len, a.q_total_rows, a.n_seq);
    if (c.direct && backward) {
        a.direct_k = blocks_without_list(a.max_k_len, a.k_total_rows, a.n_seq);
        if (a.direct_k == 0) c.direct = 0;
    }
    a.direct = c.direct;
    if (!c.general && backward) {
        c.b_splits = a.b_splits = back_splits(a);
        a.part_q = a.slots + slots_size(a.n_heads, a.q_total_rows, a.n_seq, a.reach, a.b_splits) / 4;
        a.part_k = a.part_q + (size_t)a.b_splits * a.q_total_rows * a.n_heads * a.head_dim;
    }
    return c;
}

// For tests: what `choose` says of a call whose tensors have the least strides and are aligned: the members of RelChoice, then blocks of keys without a list (backward)
// columns of a work-group of the general dQ and dK/dV kernels, work-groups that share a block (backward); `backward`: bit 0, bit 1: causal.  Not part of the C ABI's header.
extern "C" void ds_rel_attention_choice(int32_t dtype, int32_t n_seq, int32_t n_heads, int32_t head_dim, int32_t max_q_len, int32_t max_k_len, int32_t q_total_rows,
                                        int32_t k_total_rows, int32_t backward, int32_t force_generic, int32_t* out) {
    RelAttnArgs a = {};
    a.dtype = dtype; a.n_seq = n_seq; a.n_heads = n_heads; a.head_dim = head_dim; a.scale = 1.0f;
    a.max_q_len = std::min(max_q_len, q_total_rows); a.max_k_len = std::min(max_k_len, k_total_rows);
    a.q_total_rows = q_total_rows; a.k_total_rows = k_total_rows;
    a.ldq = a.ldk = a.ldv = a.ldo = (long long)n_heads * head_dim;
    a.reach = 1;
    a.mask = backward >> 1 & 1;
    const RelChoice c = choose(a, backward & 1, force_generic != 0);
    for (const int32_t v : {c.general, c.k_splits, c.direct, c.few, (backward & 1) && c.direct ? a.direct_k : 0, rel_general_columns(a, a.max_q_len), rel_general_columns(a, a.max_k_len), c.b_splits}) *out++ = v;
}

extern "C" int64_t ds_rel_attention_scratch_bytes(int32_t n_heads, int32_t head_dim, int32_t reach, int32_t q_total_rows, int32_t k_total_rows, int32_t n_seq) {
    if (n_heads <= 0 || head_dim <= 0 || head_dim > 128 || reach <= 0 || reach > kRelReach || q_total_rows <= 0 || k_total_rows <= 0 || n_seq <= 0) return 0;
    return (int64_t)rel_scratch_bytes(n_heads, head_dim, reach, q_total_rows, k_total_rows, n_seq);
}

extern "C" ds_status ds_rel_attention_fwd(int32_t dtype, int32_t n_seq, int32_t n_heads, int32_t head_dim, int32_t mask, const int32_t* q_row,
                                          const int32_t* q_len, const int32_t* k_row, const int32_t* k_len, const int32_t* q_pos, int32_t max_q_len,
                                          int32_t max_k_len, const void* q, int32_t ldq, const void* k, int32_t ldk, const void* v, int32_t ldv, float scale,
                                          const void* bias, int32_t n_buckets, const int32_t* bucket, int32_t reach, void* o, int32_t ldo, float* lse,
                                          int32_t q_total_rows, int32_t k_total_rows, void* scratch, int64_t scratch_bytes, int32_t force_generic,
                                          void* hip_stream) {
    RelAttnArgs a = {};
    a.dtype = dtype; a.n_seq = n_seq; a.n_heads = n_heads; a.head_dim = head_dim; a.mask = mask;
    a.q_row = q_row; a.q_len = q_len; a.k_row = k_row; a.k_len = k_len; a.q_pos = q_pos;
    a.max_q_len = max_q_len; a.max_k_len = max_k_len;
    a.q = q; a.k = k; a.v = v; a.ldq = ldq; a.ldk = ldk; a.ldv = ldv;
    a.scale = scale; a.bias = bias; a.n_buckets = n_buckets; a.bucket = bucket; a.reach = reach;
    a.o = o; a.ldo = ldo; a.lse = lse; a.lse_stride = q_total_rows;
    a.q_total_rows = q_total_rows; a.k_total_rows = k_total_rows;
    a.scratch = scratch; a.scratch_bytes = scratch_bytes < 0 ? 0 : (size_t)scratch_bytes;
    const ds_status r = check(a);
    if (r != DS_OK) return r;
    const RelChoice c = choose(a, false, force_generic != 0);
    if (c.few) return rel_fwd_few(a, (hipStream_t)hip_stream);
    return c.general ? rel_fwd_general(a, (hipStream_t)hip_stream) : rel_fwd_mfma(a, (hipStream_t)hip_stream);
}

extern "C" ds_status ds_rel_attention_bwd(int32_t dtype, int32_t n_seq, int32_t n_heads, int32_t head_dim, int32_t mask, const int32_t* q_row,
                                          const int32_t* q_len, const int32_t* k_row, const int32_t* k_len, const int32_t* q_pos, int32_t max_q_len,
                                          int32_t max_k_len, const void* q, int32_t ldq, const void* k, int32_t ldk, const void* v, int32_t ldv, float scale,
                                          const void* bias, int32_t n_buckets, const int32_t* bucket, int32_t reach, const void* o, const void* d_o,
                                          int32_t ldo, const float* lse, void* dq, void* dk, void* dv, float* dbias, int32_t accumulate,
                                          int32_t q_total_rows, int32_t k_total_rows, void* scratch, int64_t scratch_bytes, int32_t force_generic,
                                          void* hip_stream) {
    RelAttnArgs a = {};
    a.dtype = dtype; a.n_seq = n_seq; a.n_heads = n_heads; a.head_dim = head_dim; a.mask = mask;
    a.q_row = q_row; a.q_len = q_len; a.k_row = k_row; a.k_len = k_len; a.q_pos = q_pos;
    a.max_q_len = max_q_len; a.max_k_len = max_k_len;
    a.q = q; a.k = k; a.v = v; a.ldq = ldq; a.ldk = ldk; a.ldv = ldv;
    a.scale = scale; a.bias = bias; a.n_buckets = n_buckets; a.bucket = bucket; a.reach = reach;
    a.o = const_cast<void*>(o); a.d_o = d_o; a.ldo = ldo; a.lse = const_cast<float*>(lse); a.lse_stride = q_total_rows;
    a.dq = dq; a.dk = dk; a.dv = dv; a.dbias = dbias; a.accumulate = accumulate;
    a.q_total_rows = q_total_rows; a.k_total_rows = k_total_rows;
    a.scratch = scratch; a.scratch_bytes = scratch_bytes < 0 ? 0 : (size_t)scratch_bytes;
    const ds_status r = check(a);
    if (r != DS_OK) return r;
    if (!d_o || !dq || !dk || !dv || !dbias || (accumulate != 0 && accumulate != 1)) return DS_EINVAL;
    return choose(a, true, force_generic != 0).general ? rel_bwd_general(a, (hipStream_t)hip_stream) : rel_bwd_mfma(a, (hipStream_t)hip_stream);
}

// The bucket of distance n >= 0 among `half`: itself up to half of them, then by logarithm.  log(n / exact) / log(far / exact) is rarely a whole number of
// steps but by design (n = far, and powers between): what lies within 2^-40 of one is taken to be one.
static int bucket_of(int n, int half, int far) {
    const int exact = half / 2;
    if (n < exact) return n;
    if (n >= far || exact < 1) return half - 1;
    const long double steps = logl((long double)n / exact) / logl((long double)far / exact) * (half - exact);
    return std::min(half - 1, exact + (int)floorl(steps + 0x1p-40L));
}
extern "C" ds_status ds_rel_buckets(int32_t n_buckets, int32_t max_distance, int32_t bidirectional, int32_t* bucket) {
    if (!bucket || (bidirectional != 0 && bidirectional != 1) || n_buckets > kRelBuckets || max_distance > kRelReach) return DS_EINVAL;
    const int half = bidirectional ? n_buckets / 2 : n_buckets;
    if (half < 2 || (bidirectional && n_buckets % 2) || max_distance <= half / 2) return DS_EINVAL;
    for (int d = -max_distance; d <= max_distance; ++d)
        bucket[max_distance + d] = d <= 0 ? bucket_of(-d, half, max_distance) : bidirectional ? half + bucket_of(d, half, max_distance) : 0;
    return DS_OK;
}
