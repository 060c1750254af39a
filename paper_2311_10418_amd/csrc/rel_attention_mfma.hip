// bf16 attention with a relative position bias on the CDNA4 matrix cores (v_mfma_f32_32x32x16_bf16), heads of 64 or 128, forward and backward.  Register layout,
// memory, scheduling are those of attention_mfma.hip, which explains them; here is what the bias adds.
//
// Forward and dQ: a wavefront's block of scores covers 95 (63) distances.  Where all lie beyond reach the bias is one number and rides in the FMA that scales the
// scores: no instruction more.  Near blocks read the table of the head in LDS, whose entries stand by distance, so that the 16 rows of a lane are 16 constant
// offsets from one address (ds_read2_b32 of neighbours), and scale their scores in that step instead of the later one.
// dbias: dS is there in fp32, before it is rounded for the product, in the dQ kernel.  Blocks beyond reach add it up in a register, near ones along their
// diagonals: two additions an element with a shift of lanes in them (row_shl, row_shr), two values a lane and block into an array by distance in LDS, private to
// the lane half and the wavefront.  (16 ds_add_f32 a block instead: 160 cycles each, and the dQ kernel took 370 us instead of 77 for 31 sequences of 366 to 523,
// 16 heads of 64.)  Work-groups leave their sums in a slot; work-groups in front of the dK/dV grid add the slots up.
// dK/dV: the loop over the blocks of queries is cut by distance, so that steps stay straight code: steps with the table and steps with one number.
//
// What bounds them: forward and dQ at head size 64 the issue of a SIMD, which vector instructions (exponential, FMA, maximum and packing of every score) share with the matrix pipe's; the
// others, with one or two wavefronts to a SIMD, that and waits for fragments and transfers.  Measured, us (TFLOP/s of the products that they do; share of the compute units' busy cycles
// with the matrix pipe / with the vector ALU busy / with any instruction issued): 31 sequences of 366 to 523, 16 heads of 64, bidirectional, forward 55 (450; 26 / 63 / 95 %), dQ 76 (490; 28 / 58 / 93),
// dK/dV 91 (545; 35 / 36 / 63); 8 of 1 638 to 2 048, 16 heads of 128, causal, 160 (685; 42 / 54 / 80), 226 (725; 42 / 41 / 65), 332 (660; 38 / 28 / 44).  A fifth of a launch (heads of 128, dK/dV: an
// eighth) compute units have no work: its start and its last round.  Forward and dK/dV take as long as ordinary attention within 4 %: what the bias adds is the table's reads at near blocks and,
// in dQ, the diagonal sums.
// Roundings to bf16: probabilities and dS as operands of the second products, which the matrix instructions take in bf16 only (at most 2^-8 of each; softmax statistics, sums and dbias stay in
// fp32).  Error against 64 bits, relative, 0.0019 - 0.0021 forward and 0.0024 backward, where outputs rounded once from fp32 have 0.0016 - 0.0017.
// Registers: dK/dV at head size 64 without a mask has all 256 and spills 4 or 5 more; at 128 it keeps 192 to 240 in accumulation registers, 64 of which move over in every step.
//
// Few blocks of rows: work-groups share a block, each with some of the other side, and leave fp32 sums in the scratch (forward k_splits, backward b_splits and SHARED).
// Few queries over long keys (k_splits > 1): the keys of a head are dealt out to work-groups, see RelPart.  Where the grid of all blocks that a sequence
// may have is hardly larger than the list's (direct), there is none: its launch takes 5 us.
#include "rel_attention.hpp"
#include "attention_tiles.hpp"
#include <algorithm>
#include <initializer_list>
#include <type_traits>

namespace {

constexpr int kTablePad = 94;                           // distances that a near block (64 x 32 pairs) may reach beyond `reach`
constexpr int kAllLds = 160 * 1024;
__host__ __device__ constexpr int table_floats(int reach) { return (2 * (reach + kTablePad) + 1 + 3) & ~3; }
__device__ __forceinline__ float uniform(float v) { return __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, v))); }
// The table of a head, in three parts, so that its two trips to memory (the buckets, then their biases) go beside those that a work-group begins with anyway (its
// item, then its tables).  The last entries of a long reach are made in the end.
struct TableFill {
    int bucket[2];
    float bias[2];
    static __device__ __forceinline__ int entries(const RelAttnArgs& a) { return 2 * (a.reach + kTablePad) + 1; }
    __device__ __forceinline__ void buckets(const RelAttnArgs& a) {
#pragma unroll
        for (int i = 0; i < 2; ++i) bucket[i] = a.bucket[min(max((int)threadIdx.x + 256 * i - kTablePad, 0), 2 * a.reach)];
    }
    __device__ __forceinline__ void biases(const RelAttnArgs& a, int h) {
#pragma unroll
        for (int i = 0; i < 2; ++i) bias[i] = kLog2e * (float)((const bf16_t*)a.bias)[(size_t)min(max(bucket[i], 0), a.n_buckets - 1) * a.n_heads + h];
    }
    __device__ __forceinline__ void store(const RelAttnArgs& a, int h, float* table) const {
#pragma unroll
        for (int i = 0; i < 2; ++i)
            if ((int)threadIdx.x + 256 * i < entries(a)) table[threadIdx.x + 256 * i] = bias[i];
        for (int i = threadIdx.x + 512; i < entries(a); i += 256) table[i] = rel_bias(a, h, i - kTablePad);
    }
};
// a float as the sum of three bf16 values, exactly (the difference from the first has at most 16 bits, that from the second at most 8), as a row of eight
__device__ __forceinline__ uint4 three_parts(float v) {
    const uint32_t two = split_hi_lo(v);
    const float rest = (v - __builtin_bit_cast(float, two << 16)) - __builtin_bit_cast(float, two & 0xffff0000u);
    return make_uint4(two, (uint32_t)__builtin_bit_cast(unsigned short, (bf16_t)rest), 0u, 0u);
}
template <int HD> __device__ __forceinline__ void store_cols_f32(const f32x16_t (&acc)[HD / 32], float* __restrict__ out_row, int g) {
#pragma unroll
    for (int dt = 0; dt < HD / 32; ++dt)
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4)
            *reinterpret_cast<f32x4_t*>(out_row + dt * 32 + 8 * q4 + 4 * g) = f32x4_t{acc[dt][4 * q4], acc[dt][4 * q4 + 1], acc[dt][4 * q4 + 2], acc[dt][4 * q4 + 3]};
}

// Item of a grid without a list: `blocks` blocks of 128 rows to each sequence, whether it has them or not.  Sequences last to first (a plan lists them by ascending
// length), and under a causal mask their last queries first.
__device__ __forceinline__ int2 direct_item(const RelAttnArgs& a, int item, int blocks, bool last_first) {
    const int n = item / blocks, b = item - n * blocks;
    return make_int2(a.n_seq - 1 - n, last_first ? blocks - 1 - b : b);
}

// Items of the dK/dV kernel, as WorkDraw, in a grid whose first a.first_group work-groups do something else
struct RelDraw {
    int32_t* ctr;
    int total, xcd, k, groups;
    bool fixed;                                         // a work-group for every item: nothing is drawn (and no list kernel has cleared the counters)
    __device__ __forceinline__ RelDraw(const RelAttnArgs& a) {
        const int me = (int)blockIdx.x - a.first_group;
        ctr = const_cast<int32_t*>(a.n_items) + kCtrHeader;
        groups = a.groups;
        fixed = a.direct != 0;
        total = (a.direct ? a.n_seq * a.direct_k : a.n_items[1]) * a.b_splits * a.n_heads;
        xcd = me & 7;
        k = me >> 3;
    }
    __device__ __forceinline__ int index() const { return 8 * k + xcd; }
    __device__ __forceinline__ bool valid() const { return index() < total; }
    __device__ __forceinline__ int take() const {       // thread 0 draws; the other threads' result is meaningless
        int next = 1 << 26;
        if (threadIdx.x == 0 && !fixed) next = (groups >> 3) + __hip_atomic_fetch_add(ctr + xcd, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        return next;
    }
    __device__ __forceinline__ void advance(int next) { k = next; }
    __device__ __forceinline__ void finish() const {
        if (threadIdx.x != 0 || fixed) return;
        if (__hip_atomic_fetch_add(ctr + 8, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == groups - 1) {
#pragma unroll
            for (int i = 0; i < 9; ++i) ctr[i] = 0;
        }
    }
};

__host__ __device__ constexpr bool dkv_persistent(int hd) { return hd == 128; }

// ------------------------------------------------------------------------------------ forward
template <int HD, bool CAUSAL>
__global__ __launch_bounds__(256, HD == 64 ? 3 : 2) void rel_fwd_mfma_kernel(RelAttnArgs a) {
    extern __shared__ __attribute__((aligned(16))) char smem[];
    constexpr int TILE = 64 * HD * 2;                  // bytes of one K tile == one V tile
    constexpr int AHEAD_K = HD == 64 ? 2 : FWD_AHEAD, AHEAD_V = HD == 64 ? 2 : PV_AHEAD;
    const uint32_t lds0 = lds_address(smem);
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 31, g = lane >> 5;
    TableFill fill;
    fill.buckets(a);
    int item = blockIdx.x / a.n_heads;
    const int h = blockIdx.x - item * a.n_heads, split = a.k_splits > 1 ? item % a.k_splits : 0;
    if (a.k_splits > 1) item /= a.k_splits;
    int2 it;
    if (a.direct) {
        it = direct_item(a, item, a.direct, CAUSAL);
    } else {
        it = a.items_q[item];                           // (within the list's capacity; read beside its length, not behind it)
        if (item >= a.n_items[0]) return;
    }
    const int s = __builtin_amdgcn_readfirstlane(it.x), q0 = __builtin_amdgcn_readfirstlane(it.y) * 128;
    const int ql = __builtin_amdgcn_readfirstlane(a.q_len[s]), pos0 = __builtin_amdgcn_readfirstlane(rel_position(a, s));
    if (q0 >= ql) return;
    fill.biases(a, h);
    int kl = rel_keys(a, __builtin_amdgcn_readfirstlane(a.k_len[s]), ql, pos0), kfirst = 0;
    if (a.k_splits > 1) {                               // keys kfirst .. kfirst + kl - 1 of those that this block sees: whole tiles, as evenly as they go
        if (CAUSAL) kl = min(kl, max(0, pos0 + min(q0 + 128, ql)));
        const long long run = ((long long)kl + 64LL * a.k_splits - 1) / (64LL * a.k_splits) * 64;
        kfirst = (int)min(run * split, (long long)kl);
        kl = (int)min(run, (long long)kl - kfirst);
    }
    const int pos = pos0 - kfirst;                      // positions are counted from the first key of this work-group
    const long long qrow0 = a.q_row[s];
    const bf16_t* Q = (const bf16_t*)a.q + qrow0 * a.ldq + h * HD;
    const bf16_t* K = (const bf16_t*)a.k + ((long long)a.k_row[s] + kfirst) * a.ldk + h * HD;
    const bf16_t* V = (const bf16_t*)a.v + ((long long)a.k_row[s] + kfirst) * a.ldv + h * HD;
    const int qw0 = q0 + wave * 32;
    const int qi = qw0 + col;
    const int qi_c = qi < ql ? qi : ql - 1;

    bf16x8_t qf[HD / 16];
#pragma unroll
    for (int ks = 0; ks < HD / 16; ++ks)
        qf[ks] = *reinterpret_cast<const bf16x8_t*>(Q + (long long)qi_c * a.ldq + ks * 16 + g * 8);

    BufferTileLoader<HD> ldK, ldV;
    ldK.setup(K, a.ldk, kl, wave, lane);
    ldV.setup(V, a.ldv, kl, wave, lane);
    TrOffsets<HD> tro;
    tro.init(lane);
    const int rbase = col * (HD * 2);
    const int rsw = swz<HD>(col);

    f32x16_t oacc[HD / 32];
#pragma unroll
    for (int dt = 0; dt < HD / 32; ++dt)
#pragma unroll
        for (int e = 0; e < 16; ++e) oacc[dt][e] = 0.f;
    float m = -INFINITY, lsum = 0.f;                   // running max (in the exp2 domain) and sum
    const float c = a.scale * kLog2e;

    const int pw0 = pos + qw0, pi = pos + qi;           // positions of this wavefront's first and of this lane's query
    const int kv_end = CAUSAL ? min(kl, max(0, pos + min(q0 + 128, ql))) : kl;
    const int wave_last = CAUSAL ? min(kl - 1, pw0 + 31) : kl - 1;     // last key this wavefront can see
    const int nb = (kv_end + 63) / 64;
    if (nb > 0) {                                       // (a sequence without keys: zero output, nothing to fetch)
        ldK.issue(lds0, 0);
        ldV.issue(lds0 + TILE, 0);
    }
    float* table = reinterpret_cast<float*>(smem + 4 * TILE);
    fill.store(a, h, table);
    __syncthreads();
    const float flat_behind = uniform(table[0]), flat_front = uniform(table[2 * (a.reach + kTablePad)]);
    for (int b = 0; b < nb; ++b) {
        const int kv0 = b * 64;
        char* sK = smem + (b & 1) * (2 * TILE);
        char* sV = sK + TILE;
        wait_tiles_and_sync();                          // block b has landed; the other stage is free
        // The transfers of block b+1.  A wavefront cannot issue anything else while a transfer of its own passes the
        // address stage of the texture path (measured with timestamps: one burst of 8 transfers with an M0 each held
        // a wavefront for about 600 cycles of a 4400-cycle step; grouped under one M0 per tile, 250), so a wavefront
        // that computes in this step hands out the two groups between the MFMAs of its first product (after the last
        // block: the last tiles again, into the free stage); wavefronts without work issue them at once.
        const int kv_next = min(kv0 + 64, (nb - 1) * 64);
        const bool active = !(kv0 > wave_last || qw0 >= ql);
        const uint32_t nK_lds = lds0 + ((b + 1) & 1) * (2 * TILE);
        if (!active) {
            ldK.issue(nK_lds, kv_next);
            ldV.issue(nK_lds + TILE, kv_next);
            continue;
        }

        f32x16_t sacc[2];
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int e = 0; e < 16; ++e) sacc[kt][e] = 0.f;
        // first product, S^T = K Q^T: fragment reads AHEAD_K MFMAs in front of their use, the order pinned by fences
        // (see the dK/dV kernel)
        {
            constexpr int NF = 2 * (HD / 16);
            bf16x8_t fk[NF];
            auto read_k = [&](int i) {
                const int ks = i >> 1, kt = i & 1;
                fk[i] = *reinterpret_cast<const bf16x8_t*>(sK + kt * (32 * HD * 2) + rbase + (((ks * 2 + g) ^ rsw) << 4));
            };
#pragma unroll
            for (int i = 0; i < AHEAD_K; ++i) read_k(i);
#pragma unroll
            for (int i = 0; i < NF; ++i) {
                if (i + AHEAD_K < NF) read_k(i + AHEAD_K);
                __builtin_amdgcn_sched_barrier(kFence);
                sacc[i & 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fk[i], qf[i >> 1], sacc[i & 1], 0, 0, 0);
                __builtin_amdgcn_sched_barrier(kFence);
                if (i == NF / 4 - 1) {                  // the next K tile after a quarter of the product ...
                    ldK.issue(nK_lds, kv_next);
                    __builtin_amdgcn_sched_barrier(0);
                }
                if (i == 3 * NF / 4 - 1) {              // ... the next V tile after three quarters
                    ldV.issue(nK_lds + TILE, kv_next);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        }
        // the bias: near blocks get theirs from the table, and their scores are in the exp2 domain from here on; the rest has one number
        const int first = kv0 - pw0 - 31;               // the block's distances: first .. first + 94
        float cc = c, flat = first >= a.reach ? flat_front : flat_behind;
        if (first + 94 > -a.reach && first < a.reach) {
            int lane_at = lane;                         // (opaque: a real branch, as the mask's below, and nothing of it kept in registers)
            asm volatile("" : "+v"(lane_at));
            const int at = kv0 - pw0 + a.reach + kTablePad - (lane_at & 31) + 4 * (lane_at >> 5);
            const float* near = table + at;
#pragma unroll
            for (int i = 0; i < 8; ++i) {               // (four at a time: registers)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int kt = i >> 2, e = (i & 3) * 4 + j;
                    sacc[kt][e] = __builtin_fmaf(sacc[kt][e], c, near[kt * 32 + 8 * (e >> 2) + (e & 3)]);
                }
                if (HD == 64) __builtin_amdgcn_sched_barrier(0);
            }
            cc = 1.f;
            flat = 0.f;
        }
        // the first V^T fragments of the second product are fetched now and land during the softmax
        constexpr int NV = 4 * (HD / 32);
        bf16x8_t fv[NV];
        auto read_v = [&](int i) { fv[i] = read_tr<HD>(sV, tro, i / (HD / 32), i % (HD / 32)); };
#pragma unroll
        for (int i = 0; i < AHEAD_V; ++i) read_v(i);
        __builtin_amdgcn_sched_barrier(kFence);
        const bool need_mask = (kv0 + 64 > kl) || (CAUSAL && kv0 + 63 > pw0);
        if (need_mask) {
            // the volatile statement keeps the whole mask computation inside a real branch: hoisted or if-converted,
            // its ~130 compare / select instructions would run on every step, not just on the diagonal and the tail
            int kbase = kv0;
            asm volatile("" : "+s"(kbase));
            const int last = (CAUSAL ? min(kl - 1, pi) : kl - 1) - kbase - 4 * g;      // last visible row, as this lane counts them
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (kt * 32 + 8 * (e >> 2) + (e & 3) > last) sacc[kt][e] = -INFINITY;
        }
        float mx = -INFINITY;
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int e = 0; e < 16; e += 2) mx = max3f(mx, sacc[kt][e], sacc[kt][e + 1]);
        const float m_new = max3f(m, __builtin_fmaf(mx, cc, flat), __builtin_fmaf(__shfl_xor(mx, 32, 64), cc, flat));
        const float m_use = m_new == -INFINITY ? 0.f : m_new, shift = flat - m_use;        // (nothing seen so far: probabilities of 0)
        float rs = 0.f;
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(sacc[kt][e], cc, shift));
                sacc[kt][e] = p;
                rs += p;
            }
        const float alpha = __builtin_amdgcn_exp2f(m - m_use);
        lsum = lsum * alpha + rs;
        if (__builtin_amdgcn_ballot_w64(m_new > m) != 0) {      // some column's max moved: rescale the accumulator
#pragma unroll
            for (int dt = 0; dt < HD / 32; ++dt)
#pragma unroll
                for (int e = 0; e < 16; ++e) oacc[dt][e] *= alpha;
        }
        m = m_new;
        // second product, O^T += V^T P^T: transpose reads AHEAD_V MFMAs in front of their use
        bf16x8_t pf;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (i + AHEAD_V < NV) read_v(i + AHEAD_V);
            if (i % (HD / 32) == 0) pf = frag_from_acc(sacc[(i / (HD / 32)) >> 1], (i / (HD / 32)) & 1);
            __builtin_amdgcn_sched_barrier(kFence);
            oacc[i % (HD / 32)] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fv[i], pf, oacc[i % (HD / 32)], 0, 0, 0);
            __builtin_amdgcn_sched_barrier(kFence);
        }
    }
    __builtin_amdgcn_s_waitcnt(0x0F70);                 // no transfer may still be writing LDS when the work-group ends
    lsum += __shfl_xor(lsum, 32, 64);
    if (qi < ql && a.k_splits > 1) {
        const RelPart to = rel_part(a, h, qrow0 + qi, split);
        if (g == 0) to.stat[0] = m, to.stat[1] = lsum;
        store_cols_f32<HD>(oacc, to.o, g);
    } else if (qi < ql) {
        const long long row = qrow0 + qi;
        store_cols<HD>(oacc, lsum > 0.f ? 1.0f / lsum : 0.f, (bf16_t*)a.o + row * a.ldo + h * HD, g);
        if (g == 0) a.lse[(size_t)h * a.lse_stride + row] = (m + __builtin_amdgcn_logf(lsum)) * kLn2;
    }
}

// ------------------------------------------------------------------------------------ backward: dQ (and delta)
template <int HD, bool CAUSAL, bool SHARED>
__global__ __launch_bounds__(256, 2) void rel_bwd_dq_mfma_kernel(RelAttnArgs a) {
    extern __shared__ __attribute__((aligned(16))) char smem[];
    constexpr int TILE = 64 * HD * 2;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 31, g = lane >> 5;
    TableFill fill;
    fill.buckets(a);
    const int place = blockIdx.x / a.n_heads, h = blockIdx.x - place * a.n_heads;
    const int item = SHARED ? place / a.b_splits : place, share = SHARED ? place - item * a.b_splits : 0;
    int2 it;
    if (a.direct) {
        it = direct_item(a, item, a.direct, CAUSAL);
    } else {
        if (item >= a.n_items[0]) return;
        it = a.items_q[item];
    }
    const int s = __builtin_amdgcn_readfirstlane(it.x), q0 = __builtin_amdgcn_readfirstlane(it.y) * 128;
    const int ql = __builtin_amdgcn_readfirstlane(a.q_len[s]);
    int pos = __builtin_amdgcn_readfirstlane(rel_position(a, s)), kfirst = 0;
    const int wide = table_floats(a.reach);
    float* table = reinterpret_cast<float*>(smem + 4 * TILE);
    float* slot = a.slots + ((size_t)place * a.n_heads + h) * (2 * a.reach + 1);
    if (q0 >= ql) {                                     // (a sequence without queries, where there is no list)
        for (int i = tid; i <= 2 * a.reach; i += 256) slot[i] = 0.f;
        return;
    }
    fill.biases(a, h);
    int kl = rel_keys(a, __builtin_amdgcn_readfirstlane(a.k_len[s]), ql, pos);
    if constexpr (SHARED) {                             // keys kfirst .. kfirst + kl - 1 of those that this block sees: whole tiles, as evenly as they go
        const int seen = CAUSAL ? min(kl, max(0, pos + min(q0 + 128, ql))) : kl;
        const long long run = ((long long)seen + 64LL * a.b_splits - 1) / (64LL * a.b_splits) * 64;
        kfirst = (int)min(run * share, (long long)seen);
        kl = (int)min(run, (long long)seen - kfirst);
        pos -= kfirst;                                  // positions are counted from the first key of this work-group
    }
    const long long qrow0 = a.q_row[s];
    const bf16_t* Q = (const bf16_t*)a.q + qrow0 * a.ldq + h * HD;
    const bf16_t* dO = (const bf16_t*)a.d_o + qrow0 * a.ldo + h * HD;
    const bf16_t* O = (const bf16_t*)a.o + qrow0 * a.ldo + h * HD;
    const bf16_t* K = (const bf16_t*)a.k + ((long long)a.k_row[s] + kfirst) * a.ldk + h * HD;
    const bf16_t* V = (const bf16_t*)a.v + ((long long)a.k_row[s] + kfirst) * a.ldv + h * HD;
    const int qw0 = q0 + wave * 32;
    const int qi = qw0 + col;
    const int qi_c = qi < ql ? qi : ql - 1;

    const int pw0 = pos + qw0, pi = pos + qi;           // positions of this wavefront's first and of this lane's query
    const uint32_t lds0 = lds_address(smem);
    TileLoader<HD> ldK, ldV;
    ldK.setup(K, a.ldk, kl, wave, lane);
    ldV.setup(V, a.ldv, kl, wave, lane);
    const int kv_end = CAUSAL ? min(kl, max(0, pos + min(q0 + 128, ql))) : kl;
    if (kv_end > 0) {
        ldK.issue(lds0, 0);
        ldV.issue(lds0 + TILE, 0);
    }

    bf16x8_t qf[HD / 16], dof[HD / 16];
    float delta = 0.f;                                  // rowsum(dO * O) of this lane's query, this head
#pragma unroll
    for (int ks = 0; ks < HD / 16; ++ks) {
        qf[ks] = *reinterpret_cast<const bf16x8_t*>(Q + (long long)qi_c * a.ldq + ks * 16 + g * 8);
        dof[ks] = *reinterpret_cast<const bf16x8_t*>(dO + (long long)qi_c * a.ldo + ks * 16 + g * 8);
        const bf16x8_t of = *reinterpret_cast<const bf16x8_t*>(O + (long long)qi_c * a.ldo + ks * 16 + g * 8);
#pragma unroll
        for (int j = 0; j < 8; ++j) delta = __builtin_fmaf((float)of[j], (float)dof[ks][j], delta);
    }
    delta += __shfl_xor(delta, 32, 64);
    const float lse_q = a.lse[(size_t)h * a.lse_stride + qrow0 + qi_c];
    if (g == 0 && qi < ql && share == 0) {
        // for the dK/dV kernel: lse/scale and delta as the sums of three bf16 values, which it appends to its contractions
        const size_t at = (size_t)h * a.lse_stride + qrow0 + qi;
        reinterpret_cast<uint4*>(a.aug_lse)[at] = three_parts(lse_q == -INFINITY ? 1e30f : lse_q * (1.0f / a.scale));
        reinterpret_cast<uint4*>(a.aug_delta)[at] = three_parts(delta);
    }
    const float lse2 = qi < ql ? rel_lse2(lse_q) : INFINITY;         // (a lane past the last query repeats it, with probabilities of 0)
    const float c = a.scale * kLog2e;

    TrOffsets<HD> tro;
    tro.init(lane);
    const int rbase = col * (HD * 2);
    const int rsw = swz<HD>(col);

    f32x16_t gacc[HD / 32];
#pragma unroll
    for (int dt = 0; dt < HD / 32; ++dt)
#pragma unroll
        for (int e = 0; e < 16; ++e) gacc[dt][e] = 0.f;

    fill.store(a, h, table);
    for (int i = tid; i < 8 * wide; i += 256) table[wide + i] = 0.f;
    __syncthreads();
    // sums of dS by distance: two arrays for each wavefront, since the distances of its lane halves, rows 4 apart, overlap
    float* const sums = table + wide * (1 + 2 * wave + g);
    const float flat_behind = uniform(table[0]), flat_front = uniform(table[2 * (a.reach + kTablePad)]);
    float beyond_behind = 0.f, beyond_front = 0.f, carry = 0.f;
    float* to = sums;                                   // (where `carry` belongs: 32 on)
    const int wave_last = CAUSAL ? min(kl - 1, pw0 + 31) : kl - 1;
    const int nb = (kv_end + 63) / 64;
    for (int b = 0; b < nb; ++b) {
        const int kv0 = b * 64;
        char* sK = smem + (b & 1) * (2 * TILE);
        char* sV = sK + TILE;
        wait_tiles_and_sync();
        if (b + 1 < nb) {
            const uint32_t n = lds0 + ((b + 1) & 1) * (2 * TILE);
            ldK.issue(n, kv0 + 64);
            ldV.issue(n + TILE, kv0 + 64);
        }
        if (kv0 > wave_last || qw0 >= ql) continue;
        const bool need_mask = (kv0 + 64 > kl) || (CAUSAL && kv0 + 63 > pw0);
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) {
            if (kv0 + kt * 32 > wave_last) continue;                    // the half beyond the last key this wavefront sees
            f32x16_t sacc, pacc;
#pragma unroll
            for (int e = 0; e < 16; ++e) { sacc[e] = 0.f; pacc[e] = 0.f; }
            {
                constexpr int NF = HD / 16;
                bf16x8_t fk[NF], fv[NF];
                auto read_kv = [&](int ks) {
                    const int o = kt * (32 * HD * 2) + rbase + (((ks * 2 + g) ^ rsw) << 4);
                    fk[ks] = *reinterpret_cast<const bf16x8_t*>(sK + o);
                    fv[ks] = *reinterpret_cast<const bf16x8_t*>(sV + o);
                };
#pragma unroll
                for (int ks = 0; ks < DQ_AHEAD; ++ks) read_kv(ks);
#pragma unroll
                for (int ks = 0; ks < NF; ++ks) {
                    if (ks + DQ_AHEAD < NF) read_kv(ks + DQ_AHEAD);
                    __builtin_amdgcn_sched_barrier(kFence);
                    sacc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fk[ks], qf[ks], sacc, 0, 0, 0);
                    pacc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fv[ks], dof[ks], pacc, 0, 0, 0);
                    __builtin_amdgcn_sched_barrier(kFence);
                }
            }
            const int first = kv0 + kt * 32 - pw0 - 31; // the half's distances: first .. first + 62
            const bool near = first + 62 > -a.reach && first < a.reach;
            int at = kv0 + kt * 32 - pi + 4 * g + a.reach + kTablePad;
            if (near) {
                asm volatile("" : "+v"(at));
                const float* from = table + at;
#pragma unroll
                for (int e = 0; e < 16; ++e) sacc[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(sacc[e], c, from[8 * (e >> 2) + (e & 3)] - lse2));   // P^T
            } else {
                const float shift = (first >= a.reach ? flat_front : flat_behind) - lse2;
#pragma unroll
                for (int e = 0; e < 16; ++e) sacc[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(sacc[e], c, shift));
            }
            if (need_mask) {
                // one real branch around the whole mask (see the forward kernel): tested per element, it would cut
                // the chain of exponentials into sixteen basic blocks
                int kbase = kv0 + kt * 32;
                asm volatile("" : "+s"(kbase));
                const int last = (CAUSAL ? min(kl - 1, pi) : kl - 1) - kbase - 4 * g;  // last visible row, as this lane counts them
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (8 * (e >> 2) + (e & 3) > last) sacc[e] = 0.f;
            }
#pragma unroll
            for (int e = 0; e < 16; ++e) sacc[e] *= pacc[e] - delta;          // dS^T
            if (near) {
                // rows 8 (e / 4) + e % 4 (+ 4 g) of columns 16 (lane / 16 % 2) + lane % 16: three sums a lane, of distances 16 apart.  The third is the first of the
                // half behind, 32 keys on, and goes there in a register.
                float sum[3] = {carry, 0.f, 0.f};
                add_diagonals<0>(sacc[0], sum[0], sum[1]);
                add_diagonals<1>(sacc[1], sum[0], sum[1]);
                add_diagonals<2>(sacc[2], sum[0], sum[1]);
                add_diagonals<3>(sacc[3], sum[0], sum[1]);
                add_diagonals<8>(sacc[4], sum[0], sum[1]);
                add_diagonals<9>(sacc[5], sum[0], sum[1]);
                add_diagonals<10>(sacc[6], sum[0], sum[1]);
                add_diagonals<11>(sacc[7], sum[0], sum[1]);
                add_diagonals<0>(sacc[8], sum[1], sum[2]);
                add_diagonals<1>(sacc[9], sum[1], sum[2]);
                add_diagonals<2>(sacc[10], sum[1], sum[2]);
                add_diagonals<3>(sacc[11], sum[1], sum[2]);
                add_diagonals<8>(sacc[12], sum[1], sum[2]);
                add_diagonals<9>(sacc[13], sum[1], sum[2]);
                add_diagonals<10>(sacc[14], sum[1], sum[2]);
                add_diagonals<11>(sacc[15], sum[1], sum[2]);
                to = sums + (kv0 + kt * 32 - pw0 + 4 * g - (lane & 31) + a.reach + kTablePad);
                wave_lds_sync();                                            // (one lane's second place is another's first)
                to[0] += sum[0];
                wave_lds_sync();
                to[16] += sum[1];
                wave_lds_sync();
                carry = sum[2];
            } else {
                float x[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = sacc[e] + sacc[e + 8];
                const float add = ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
                if (first >= a.reach) beyond_front += add;
                else beyond_behind += add;
            }
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const bf16x8_t dsf = frag_from_acc(sacc, u);
#pragma unroll
                for (int dt = 0; dt < HD / 32; ++dt) {
                    const bf16x8_t kt_f = read_tr<HD>(sK, tro, 2 * kt + u, dt);
                    gacc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kt_f, dsf, gacc[dt], 0, 0, 0);
                }
            }
        }
    }
    if (qi < ql) {
        if constexpr (SHARED) store_cols_f32<HD>(gacc, a.part_q + ((size_t)share * a.q_total_rows + qrow0 + qi) * ((size_t)a.n_heads * HD) + h * HD, g);
        else store_cols<HD>(gacc, a.scale, (bf16_t*)a.dq + (qrow0 + qi) * a.ldq + h * HD, g);
    }
    to[32] += carry;
    beyond_behind = wave_sum(beyond_behind);
    beyond_front = wave_sum(beyond_front);
    if (lane == 0) {
        lds_add(sums, beyond_behind);
        lds_add(sums + 2 * (a.reach + kTablePad), beyond_front);
    }
    // the block's slot: what the wavefronts have, in a fixed order; distances beyond reach with those at it
    __syncthreads();
    for (int i = tid; i <= 2 * (a.reach + kTablePad); i += 256) {
        float sum = 0.f;
#pragma unroll
        for (int w = 0; w < 8; ++w) sum += table[wide * (1 + w) + i];
        const int d = i - kTablePad;
        if (d > 0 && d < 2 * a.reach) slot[d] = sum;
        else table[i] = sum;
    }
    __syncthreads();
    if (wave < 2) {
        const float* from = table + wave * (2 * a.reach + kTablePad);
        float sum = 0.f;
        for (int i = lane; i <= kTablePad; i += 64) sum += from[i];
        sum = wave_sum(sum);
        if (lane == 0) slot[wave * 2 * a.reach] = sum;
    }
}

// ------------------------------------------------------------------------------------ backward: dK, dV
// LDS, a ring of four stages of: Q tile, dO tile ([64][HD]) and the two statistics tiles ([64 rows][8] bf16:
// three parts and five zeros of lse/scale and of delta, as the dQ kernel left them).  Three blocks are in flight while one is
// consumed: with one wavefront per SIMD (about 370 registers) nothing else hides the latency of the transfers.
//
// Persistent work-groups at head size 128 (PS) where work goes by a list: as many as fit on the chip, each drawing its next item (key block, head) while it works on
// the current one, and requesting that item's first three query blocks and its K / V fragments BEFORE it stores the current results.  With a work-group per item
// nothing hides what lies between two items (the end of one work-group, the start of the next, dependent table reads, the first tiles); measured with ordinary attention,
// 65 536 tokens of mean length 385: 1015 -> 962 us.  Not at head size 64, where two work-groups share a CU and the dispatcher's replacement is quicker than a draw
// (there, one-step items 47 us, 59 with draws).  Without a list lengths are much the same, and a work-group takes one item.
template <int HD, bool CAUSAL, bool SHARED>
__global__ __launch_bounds__(256, HD == 64 ? 2 : 1) void rel_bwd_dkv_mfma_kernel(RelAttnArgs a) {
    extern __shared__ __attribute__((aligned(16))) char smem[];
    constexpr int TILE = 64 * HD * 2;
    constexpr int STAGE = 2 * TILE + 2048;
    constexpr int NS = 4;                               // ring of stages: three blocks in flight while one is consumed
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 31, g = lane >> 5;
    const uint32_t lds0 = lds_address(smem);
    // the next draw, in two words used in turn: an item may have no step (a sequence without queries, keys beyond the last
    // query of a causal one) and then no other barrier than the one behind the write, so the word written for an item must
    // not be the one that a slower wavefront may still be reading for the item before
    volatile int* s_next = reinterpret_cast<volatile int*>(smem + NS * STAGE);
    int turn = 0;
    char* s_zero = smem + NS * STAGE + 64;              // 32 rows of zeros, see phase_d
    TileLoader<HD> ldQ, ldO;
    ldQ.setup(nullptr, a.ldq, 0, wave, lane);
    ldO.setup(nullptr, a.ldo, 0, wave, lane);
    constexpr bool PS = dkv_persistent(HD);
    RelDraw draw(a);
    float* table = reinterpret_cast<float*>(smem + NS * STAGE + 64 + 64 * HD);
    if ((int)blockIdx.x < a.first_group) {              // work-groups in front: one for each head sums up dbias
        if ((int)blockIdx.x < a.n_heads) sum_dbias<256>(a, blockIdx.x, (a.direct ? a.n_seq * a.direct : a.n_items[0]) * a.b_splits, reinterpret_cast<float*>(smem));
        return;
    }
    int kw0, ki, kl, ql, h, q_begin, nb, pos, share = 0, table_head = -1;
    int k0;
    long long krow0;
    const char* aug_src;
    bf16x8_t kf[HD / 16], vf[HD / 16];
    // block blk -> stage blk % 4: Q tile, dO tile, and (wavefronts 0 and 1) the two statistics tiles, all by direct
    // transfers; indices past the last block are clamped (redundant transfers into a free stage keep the count of
    // outstanding transfers the same at every step)
    auto issue_block = [&](int blk) {
        const uint32_t n = lds0 + (blk & (NS - 1)) * STAGE;
        const int bc = blk < nb ? blk : nb - 1;
        const int q0 = q_begin + bc * 64;
        ldQ.issue(n, q0);
        ldO.issue(n + TILE, q0);
        if (wave < 2) {
            int r = q0 + lane;
            r = r < ql ? r : ql - 1;
            lds_dma16_at(aug_src + (size_t)r * 16, n + 2 * TILE + wave * 1024);
        }
    };
    TableFill fill;
    // take up the item `draw` stands at: its tables, the first three blocks, the K / V fragments
    auto begin_item = [&] {
        fill.buckets(a);
        int item = draw.index() / a.n_heads;
        h = draw.index() - item * a.n_heads;
        if constexpr (SHARED) {
            share = item % a.b_splits;
            item /= a.b_splits;
        }
        const int2 it = a.direct ? direct_item(a, item, a.direct_k, false) : a.items_k[item];
        const int s = __builtin_amdgcn_readfirstlane(it.x);
        k0 = __builtin_amdgcn_readfirstlane(it.y) * 128;
        pos = __builtin_amdgcn_readfirstlane(rel_position(a, s));
        ql = __builtin_amdgcn_readfirstlane(a.q_len[s]);
        kl = __builtin_amdgcn_readfirstlane(a.k_len[s]);
        fill.biases(a, h);
        const long long qrow0 = __builtin_amdgcn_readfirstlane(a.q_row[s]);
        krow0 = __builtin_amdgcn_readfirstlane(a.k_row[s]);
        kw0 = k0 + wave * 32;
        ki = kw0 + col;
        q_begin = CAUSAL ? max(0, k0 - pos) : 0;
        nb = k0 < kl ? max(0, (ql - q_begin + 63) / 64) : 0;                  // (none: keys beyond the last query of a causal sequence)
        if constexpr (SHARED) {                         // this work-group's blocks of queries: ql is the end of the last of them
            const int run = (nb + a.b_splits - 1) / a.b_splits, first = min(run * share, nb);
            nb = min(run, nb - first);
            q_begin += 64 * first;
            ql = min(ql, q_begin + 64 * nb);
        }
        ldQ.base = reinterpret_cast<const char*>((const bf16_t*)a.q + qrow0 * a.ldq + h * HD);
        ldO.base = reinterpret_cast<const char*>((const bf16_t*)a.d_o + qrow0 * a.ldo + h * HD);
        ldQ.n_valid = ldO.n_valid = ql;
        aug_src = reinterpret_cast<const char*>(wave == 0 ? a.aug_lse : a.aug_delta) + ((size_t)h * a.lse_stride + qrow0) * 16;
        if (nb > 0) {
            issue_block(0);
            issue_block(1);
            issue_block(2);
        }
        if (k0 >= kl) return;                           // (a sequence without keys, where there is no list)
        const int ki_c = ki < kl ? ki : kl - 1;
        const bf16_t* K = (const bf16_t*)a.k + (krow0 + ki_c) * a.ldk + h * HD;
        const bf16_t* V = (const bf16_t*)a.v + (krow0 + ki_c) * a.ldv + h * HD;
#pragma unroll
        for (int ks = 0; ks < HD / 16; ++ks) {
            kf[ks] = *reinterpret_cast<const bf16x8_t*>(K + ks * 16 + g * 8);
            vf[ks] = *reinterpret_cast<const bf16x8_t*>(V + ks * 16 + g * 8);
        }
    };
    if (!draw.valid()) {
        if (PS) draw.finish();
        return;
    }
    begin_item();
    for (int i = tid; i < 64 * HD / 16; i += 256) reinterpret_cast<uint4*>(s_zero)[i] = make_uint4(0u, 0u, 0u, 0u);
    bf16x8_t neg_ones;                                  // contraction slots 0 to 2 (lane half 0) pick the three parts
#pragma unroll
    for (int j = 0; j < 8; ++j) neg_ones[j] = (bf16_t)((g == 0 && j < 3) ? -1.0f : 0.0f);
    const float c = a.scale * kLog2e;

    TrOffsets<HD> tro;
    tro.init(lane);
    const int rbase = col * (HD * 2);
    const int rsw = swz<HD>(col);

    f32x16_t dkacc[HD / 32], dvacc[HD / 32];
    for (;;) {
#pragma unroll
    for (int dt = 0; dt < HD / 32; ++dt)
#pragma unroll
        for (int e = 0; e < 16; ++e) { dkacc[dt][e] = 0.f; dvacc[dt][e] = 0.f; }

    int next = 0;
    if (PS) next = draw.take();                         // (needed after the loop)
    if (h != table_head) {                              // (nobody reads the old one: a barrier ended the item before)
        fill.store(a, h, table);
        __syncthreads();
        table_head = h;
    }
    const float flat_behind = uniform(table[0]), flat_front = uniform(table[2 * (a.reach + kTablePad)]);
    // the K / V fragments (ordinary loads) and the stores of the item before are complete before the loop: left to the
    // compiler, its waits for them would sit inside the loop as "nothing outstanding", which would also drain the
    // transfers in flight.  So are the zeros of s_zero, in front of the first step's barrier.
    __builtin_amdgcn_s_waitcnt(0x0070);
    // One step = one 64-query block, straight code: any branch inside it, even one that is never taken, splits the live
    // ranges of the 128 accumulator registers and costs hundreds of register copies per step.  The step exists with the
    // mask as selects and without, with biases from the table and with one number, and the loop is cut where these change.
    const bool wave_has_keys = kw0 < kl;
    auto step = [&](int b, auto masked_t, auto near_t, float flat) {
        constexpr bool MASKED = decltype(masked_t)::value, NEAR = decltype(near_t)::value;
        const int q0 = q_begin + b * 64;
        char* sQ = smem + (b & (NS - 1)) * STAGE;
        char* sdO = sQ + TILE;
        char* s_lse = sdO + TILE;
        char* s_delta = s_lse + 1024;
        // block b has landed for this wavefront (the two newest blocks may still be in flight), then for everybody;
        // the stage read in the previous step is free
        if (wave < 2) __builtin_amdgcn_s_waitcnt(vmcnt_imm(2 * (2 * (HD / 32) + 1)));
        else __builtin_amdgcn_s_waitcnt(vmcnt_imm(2 * (2 * (HD / 32))));
        __builtin_amdgcn_s_barrier();
        issue_block(b + 3);
        if (!wave_has_keys) return;
        if (MASKED && CAUSAL && pos + q0 + 63 < kw0) return;
        // queries of the block that see this lane's key, as this lane counts its rows: first .. first + visible - 1
        const int first = (CAUSAL ? max(ki - pos - q0, 0) : 0) - 4 * g;
        const unsigned visible = (unsigned)max(ql - q0 - 4 * g - first, 0);
        // The two 32-query halves software-pipelined.  The exp / product work of half 0 sits between
        // the MFMAs of half 1's first products, that of half 1 between the MFMAs of half 0's second products, so
        // that the one wavefront of this SIMD keeps the matrix pipe and the vector ALU busy at the same time.
        constexpr int NA = HD / 16 + 1, AHEAD = 3, ND = 2 * (HD / 32), AHEAD_D = 2;
        f32x16_t sa[2], pa[2];
        // the table's entry of this lane's key and the block's first query; a block beyond reach reads entries that are all alike
        const float* from = table;
        if constexpr (NEAR) from += min(max(kw0 - pos - q0 - 63, -a.reach - kTablePad), a.reach) + 63 + col - 4 * g + a.reach + kTablePad;
        float ahead[2];                                 // biases of the next two elements
        auto read_bias = [&](int qt, int e) {
            if constexpr (NEAR) {
#pragma unroll
                for (int i = 0; i < 2; ++i) ahead[i] = from[-(qt * 32 + 8 * (e >> 2) + (e & 3) + i)];
            }
        };
        bf16x8_t fq[NA], fo[NA], td[ND], tq[ND], pf[2], dsf[2];
        auto read_a = [&](int qt, int i) {
            if (i < HD / 16) {
                const int o = qt * (32 * HD * 2) + rbase + (((i * 2 + g) ^ rsw) << 4);
                fq[i] = *reinterpret_cast<const bf16x8_t*>(sQ + o);
                fo[i] = *reinterpret_cast<const bf16x8_t*>(sdO + o);
            } else {
                fq[i] = *reinterpret_cast<const bf16x8_t*>(s_lse + (qt * 32 + col) * 16);
                fo[i] = *reinterpret_cast<const bf16x8_t*>(s_delta + (qt * 32 + col) * 16);
            }
        };
        auto softmax2 = [&](int qt, int e0) {         // two elements of half qt: P and dS in place
#pragma unroll
            for (int e = e0; e < e0 + 2; ++e) {
                const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(sa[qt][e], c, NEAR ? ahead[e - e0] : flat));
                const bool out = MASKED && (unsigned)(qt * 32 + 8 * (e >> 2) + (e & 3) - first) >= visible;
                sa[qt][e] = out ? 0.f : p;
                pa[qt][e] = out ? 0.f : p * pa[qt][e];
            }
            if (e0 < 14) read_bias(qt, e0 + 2);
        };
        auto phase_a = [&](int qt, bool with_prev) {
#pragma unroll
            for (int e = 0; e < 16; ++e) { sa[qt][e] = 0.f; pa[qt][e] = 0.f; }
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) read_a(qt, i);
#pragma unroll
            for (int i = 0; i < NA; ++i) {
                if (i + AHEAD < NA) read_a(qt, i + AHEAD);
                __builtin_amdgcn_sched_barrier(kFence);
                sa[qt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fq[i], i < HD / 16 ? kf[i < HD / 16 ? i : 0] : neg_ones, sa[qt], 0, 0, 0);
                pa[qt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fo[i], i < HD / 16 ? vf[i < HD / 16 ? i : 0] : neg_ones, pa[qt], 0, 0, 0);
                __builtin_amdgcn_sched_barrier(kFence);
                if (with_prev && i == 0) read_bias(qt ^ 1, 0);
                if (with_prev && i < NA - 1) {          // 16 / (NA - 1) elements of the other half per slice
#pragma unroll
                    for (int e = i * (16 / (NA - 1)); e < (i + 1) * (16 / (NA - 1)); e += 2) softmax2(qt ^ 1, e);
                }
            }
        };
        auto phase_d = [&](int qt, bool with_next) {
#pragma unroll
            for (int u = 0; u < 2; ++u) { pf[u] = frag_from_acc(sa[qt], u); dsf[u] = frag_from_acc(pa[qt], u); }
            // a half that no key of this wavefront sees: zeros instead of its rows, which may hold infinities (0 x Inf is NaN)
            const bool hidden = MASKED && (qt ? q0 + 32 >= ql : CAUSAL && pos + q0 + 31 < kw0);
            const char* rO = hidden ? s_zero - qt * (32 * HD * 2) : sdO;
            const char* rQ = hidden ? s_zero - qt * (32 * HD * 2) : sQ;
            auto read_d = [&](int j) {
                td[j] = read_tr<HD>(rO, tro, 2 * qt + j / (HD / 32), j % (HD / 32));
                tq[j] = read_tr<HD>(rQ, tro, 2 * qt + j / (HD / 32), j % (HD / 32));
            };
#pragma unroll
            for (int j = 0; j < AHEAD_D; ++j) read_d(j);
#pragma unroll
            for (int j = 0; j < ND; ++j) {
                if (j + AHEAD_D < ND) read_d(j + AHEAD_D);
                __builtin_amdgcn_sched_barrier(kFence);
                dvacc[j % (HD / 32)] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(td[j], pf[j / (HD / 32)], dvacc[j % (HD / 32)], 0, 0, 0);
                dkacc[j % (HD / 32)] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(tq[j], dsf[j / (HD / 32)], dkacc[j % (HD / 32)], 0, 0, 0);
                __builtin_amdgcn_sched_barrier(kFence);
                if (with_next && j == 0) read_bias(qt ^ 1, 0);
                if (with_next) {
#pragma unroll
                    for (int e = j * (16 / ND); e < (j + 1) * (16 / ND); e += 2) softmax2(qt ^ 1, e);
                }
            }
        };
        phase_a(0, false);
        phase_a(1, true);          // + exp / products of half 0
        phase_d(0, true);          // + exp / products of half 1
        phase_d(1, false);
    };
    // Blocks in order of their queries: (causal) those that not all keys of the work-group are seen by, then by the bias of this wavefront's pairs: beyond
    // reach in front (unmasked only), near, beyond reach behind; the ragged last one.  Every wavefront goes through as many steps.
    const int n_diag = CAUSAL ? min(nb, max(0, (k0 + 127 - pos - q_begin + 63) / 64)) : 0;
    const int n_full = min(nb, max(n_diag, (ql - q_begin) / 64));            // blocks b < n_full have all their 64 rows (nb = 0: no keys here)
    const int before = kw0 - pos - q_begin;             // distance of this wavefront's first key and the first query: block b has before - 64 b - 63 .. before - 64 b + 31
    const int n_front = CAUSAL ? 0 : min(n_full, max(0, (before - 63 - a.reach + 64) >> 6));                        // blocks with before - 64 b - 63 >= reach
    const int n_near = min(n_full, max(0, (before + 31 + a.reach + 63) >> 6));                                      // ... and before - 64 b + 31 > -reach
    const std::true_type yes;
    const std::false_type no;
    int b = 0;
    if constexpr (CAUSAL) {
        for (; b < n_diag; ++b) step(b, yes, yes, 0.f);
    } else {
        for (; b < n_front; ++b) step(b, no, no, flat_front);
    }
    for (; b < n_near; ++b) step(b, no, yes, 0.f);
    for (; b < n_full; ++b) step(b, no, no, flat_behind);
    for (; b < nb; ++b) step(b, yes, yes, 0.f);
    __builtin_amdgcn_s_waitcnt(0x0F70);                 // no transfer may still be writing LDS ...
    const bool store = ki < kl;
    bf16_t* dk = (bf16_t*)a.dk + (krow0 + ki) * a.ldk + h * HD;
    bf16_t* dv = (bf16_t*)a.dv + (krow0 + ki) * a.ldv + h * HD;
    float* part = SHARED ? a.part_k + ((size_t)share * a.k_total_rows + krow0 + ki) * (2 * (size_t)a.n_heads * HD) + h * HD : nullptr;
    bool more = false;
    if constexpr (PS) {
        if (tid == 0) s_next[turn] = next;
        __builtin_amdgcn_s_waitcnt(0xC07F);             // lgkmcnt(0)
        __builtin_amdgcn_s_barrier();                   // ... and nobody is reading it any more
        draw.advance(__builtin_amdgcn_readfirstlane(s_next[turn]));
        turn ^= 1;
        more = draw.valid();
        if (more) begin_item();
    }
    if (store) {
        if constexpr (SHARED) {
            store_cols_f32<HD>(dkacc, part, g);
            store_cols_f32<HD>(dvacc, part + (size_t)a.n_heads * HD, g);
        } else {
            store_cols<HD>(dkacc, a.scale, dk, g);
            store_cols<HD>(dvacc, 1.0f, dv, g);
        }
    }
    if (!more) break;
    }   // for (;;): the next item
    if (PS) draw.finish();
}

// Forward of many queries: what at most kRelShares work-groups that shared a block found, four features to a thread (rel_join is for few queries: a wavefront for each head of each)
template <int HD> __global__ __launch_bounds__(256) void rel_rows_join_kernel(RelAttnArgs a) {
    const int s = blockIdx.y, per = a.n_heads * (HD / 4), n = a.k_splits;
    const long long row0 = a.q_row[s], all = (long long)a.q_len[s] * per;
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < all; i += (long long)gridDim.x * 256) {
        const long long row = row0 + i / per;
        const int at = (int)(i % per), h = at / (HD / 4), d = at % (HD / 4) * 4;
        const RelPart p = rel_part(a, h, row, 0);
        f32x4_t v[kRelShares];
        float2 st[kRelShares];
#pragma unroll
        for (int k = 0; k < kRelShares; ++k)
            if (k < n) {
                st[k] = *reinterpret_cast<const float2*>(p.stat + k * (HD + 4));
                v[k] = *reinterpret_cast<const f32x4_t*>(p.o + k * (HD + 4) + d);
            }
        float top = -INFINITY, sum = 0.f;
#pragma unroll
        for (int k = 0; k < kRelShares; ++k)
            if (k < n && st[k].y != 0.f) top = fmaxf(top, st[k].x);
        f32x4_t o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < kRelShares; ++k)
            if (k < n) {                                // (a share without keys has sum 0, and its maximum does not count)
                const float w = st[k].y == 0.f ? 0.f : __builtin_amdgcn_exp2f(st[k].x - top);
                sum = __builtin_fmaf(w, st[k].y, sum);
                o += w * v[k];
            }
        const float r = sum == 0.f ? 0.f : 1.0f / sum;
        bf16x4_t x;
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = (bf16_t)(o[e] * r);
        *reinterpret_cast<bf16x4_t*>((bf16_t*)a.o + row * a.ldo + h * HD + d) = x;
        if (d == 0) a.lse[(size_t)h * a.lse_stride + row] = (top + __builtin_amdgcn_logf(sum)) * kLn2;
    }
}
template <int HD> ds_status rows_join(const RelAttnArgs& a, hipStream_t st) {
    const long long pieces = (long long)a.max_q_len * a.n_heads * (HD / 4);
    hipLaunchKernelGGL(rel_rows_join_kernel<HD>, dim3((unsigned)std::min((pieces + 255) / 256, 2048LL), a.n_seq), dim3(256), 0, st, a);
    DS_LAUNCH_CHECK();
    return DS_OK;
}

// Backward: what the work-groups that shared a block found, in their order; blockIdx.z 0: dQ, 1: dK and dV, four features to a thread
template <int HD> __global__ __launch_bounds__(256) void rel_back_join_kernel(RelAttnArgs a) {
    const int s = blockIdx.y;
    const bool keys = blockIdx.z != 0;
    const long long row0 = keys ? a.k_row[s] : a.q_row[s], total = keys ? a.k_total_rows : a.q_total_rows;
    const int wide = a.n_heads * HD, per = (keys ? 2 : 1) * wide / 4;
    const long long n = (long long)(keys ? a.k_len[s] : a.q_len[s]) * per;
    const float* from = keys ? a.part_k : a.part_q;
    const size_t step = (size_t)total * per * 4;
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < n; i += (long long)gridDim.x * 256) {
        const long long row = row0 + i / per;
        const int c = (int)(i % per) * 4;
        const float* p = from + (size_t)row * per * 4 + c;
        f32x4_t sum = *reinterpret_cast<const f32x4_t*>(p);
#pragma unroll 4
        for (int k = 1; k < a.b_splits; ++k) sum += *reinterpret_cast<const f32x4_t*>(p + k * step);
        const bool value = keys && c >= wide;
        bf16_t* to = !keys ? (bf16_t*)a.dq + row * a.ldq + c : value ? (bf16_t*)a.dv + row * a.ldv + (c - wide) : (bf16_t*)a.dk + row * a.ldk + c;
        bf16x4_t x;
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = (bf16_t)(value ? sum[e] : sum[e] * a.scale);
        *reinterpret_cast<bf16x4_t*>(to) = x;
    }
}

template <int HD, bool CAUSAL>
ds_status fwd_launch(const RelAttnArgs& a, hipStream_t st) {
    static std::atomic<uint64_t> allowed{0};
    auto kern = rel_fwd_mfma_kernel<HD, CAUSAL>;
    const int smem = 4 * (64 * HD * 2) + table_floats(a.reach) * 4;
    ds_status r = allow_dynamic_lds(kern, kAllLds, allowed);
    if (r != DS_OK) return r;
    hipLaunchKernelGGL(kern, dim3((unsigned)(a.direct ? a.n_seq * a.direct : a.max_items_q) * a.k_splits * a.n_heads), dim3(256), smem, st, a);
    DS_LAUNCH_CHECK();
    return DS_OK;
}

template <int HD, bool CAUSAL, bool SHARED>
ds_status bwd_launch(const RelAttnArgs& a, hipStream_t st) {
    static std::atomic<uint64_t> allowed_q{0}, allowed_kv{0};
    auto kq = rel_bwd_dq_mfma_kernel<HD, CAUSAL, SHARED>;
    auto kkv = rel_bwd_dkv_mfma_kernel<HD, CAUSAL, SHARED>;
    const int smem_q = 4 * (64 * HD * 2) + 9 * table_floats(a.reach) * 4;
    const int smem_kv = 4 * (2 * (64 * HD * 2) + 2048) + 64 + 64 * HD + table_floats(a.reach) * 4;      // stages, draws, zeros, table
    ds_status r = allow_dynamic_lds(kq, kAllLds, allowed_q);
    if (r != DS_OK) return r;
    r = allow_dynamic_lds(kkv, kAllLds, allowed_kv);
    if (r != DS_OK) return r;
    hipLaunchKernelGGL(kq, dim3((unsigned)(a.direct ? a.n_seq * a.direct : a.max_items_q) * a.b_splits * a.n_heads), dim3(256), smem_q, st, a);
    DS_LAUNCH_CHECK();
    const unsigned items_kv = (unsigned)(a.direct ? a.n_seq * a.direct_k : a.max_items_k) * a.b_splits * a.n_heads;
    RelAttnArgs b = a;
    b.first_group = (a.n_heads + 7) / 8 * 8;            // (the rest keeps its XCDs)
    b.groups = dkv_persistent(HD) && !a.direct ? (int32_t)persistent_grid(items_kv) : (int32_t)items_kv;
    hipLaunchKernelGGL(kkv, dim3((unsigned)b.first_group + b.groups), dim3(256), smem_kv, st, b);
    DS_LAUNCH_CHECK();
    if constexpr (SHARED) {
        const long long pieces = std::max((long long)a.max_q_len, 2LL * a.max_k_len) * a.n_heads * (HD / 4);
        hipLaunchKernelGGL(rel_back_join_kernel<HD>, dim3((unsigned)std::min((pieces + 255) / 256, 2048LL), a.n_seq, 2), dim3(256), 0, st, a);
        DS_LAUNCH_CHECK();
    }
    return DS_OK;
}
}  // namespace

bool rel_mfma_supported(const RelAttnArgs& a) {
    if (a.dtype != DS_DTYPE_BF16 || (a.head_dim != 64 && a.head_dim != 128)) return false;
    const long long ld_max = 1LL << 23;                 // 64 rows of a tile stay within a 31-bit byte offset
    for (const long long ld : {a.ldq, a.ldk, a.ldv, a.ldo})
        if (ld % 8 || ld >= ld_max) return false;
    for (const void* p : {a.q, a.k, a.v, (const void*)a.o, a.d_o, (const void*)a.dq, (const void*)a.dk, (const void*)a.dv})
        if ((uintptr_t)p & 15) return false;
    if (a.d_o && !(a.scale >= 0x1p-20f && a.scale <= 0x1p20f)) return false;        // (log-sum-exps reach the dK/dV kernel divided by it)
    // work-items of a launch: 32 bits
    const long long items = (long long)std::max(a.q_total_rows, a.k_total_rows) / 128 + (long long)a.n_seq * 2;
    return items * a.n_heads + a.n_heads + 8 < 1LL << 23;       // (shares only where work-groups are few)
}

static ds_status prepare(RelAttnArgs& a, bool backward, hipStream_t st) {
    a.aug_lse = a.aug;
    a.aug_delta = a.aug + (size_t)a.n_heads * a.q_total_rows * 16;
    if (a.direct) return DS_OK;
    return attn_prepare_lists(a, backward, st);
}

ds_status rel_fwd_mfma(const RelAttnArgs& a0, hipStream_t st) {
    RelAttnArgs a = a0;
    ds_status r = prepare(a, false, st);
    if (r != DS_OK) return r;
    if (a.head_dim == 128) r = a.mask ? fwd_launch<128, true>(a, st) : fwd_launch<128, false>(a, st);
    else r = a.mask ? fwd_launch<64, true>(a, st) : fwd_launch<64, false>(a, st);
    if (r != DS_OK || a.k_splits == 1) return r;
    if (a.max_q_len <= 64 || a.k_splits > kRelShares) return rel_join(a, st);
    return a.head_dim == 128 ? rows_join<128>(a, st) : rows_join<64>(a, st);
}

ds_status rel_bwd_mfma(const RelAttnArgs& a0, hipStream_t st) {
    RelAttnArgs a = a0;
    const ds_status r = prepare(a, true, st);
    if (r != DS_OK) return r;
    auto by_shares = [&](auto hd, auto causal) {
        return a.b_splits > 1 ? bwd_launch<decltype(hd)::value, decltype(causal)::value, true>(a, st) : bwd_launch<decltype(hd)::value, decltype(causal)::value, false>(a, st);
    };
    auto by_mask = [&](auto hd) { return a.mask ? by_shares(hd, std::true_type{}) : by_shares(hd, std::false_type{}); };
    return a.head_dim == 128 ? by_mask(std::integral_constant<int, 128>{}) : by_mask(std::integral_constant<int, 64>{});
}
