// Differential attention in bf16 on the matrix cores (v_mfma_f32_32x32x16_bf16), head size 64 or 128 (maps of 32 or 64), causal or
// unmasked, forward and backward.  Register layout, tiles, transpose reads and work lists are those of attention_mfma.hip: a wavefront
// owns 32 columns (queries in forward and dQ, keys in dK/dV) and computes transposed score tiles, one set of accumulator registers
// being the B operand of the next product as it stands.
//
// What two maps change.  The products that make scores contract over half a head each, so that both maps' scores cost what one map's
// of the whole head do; dP = dO V^T is common to both, and so is dV (one product with P_1 - lambda P_2); dQ and dK of a map are half a
// head wide.  Backward therefore takes the matrix instructions of ordinary attention, with twice the exponentials.  Forward cannot form
// P_1 - lambda P_2 before both sums are known, so it keeps two accumulators and multiplies every fragment of V^T by both maps'
// probabilities (6 instead of 4 products of a head's width; a first pass over the scores for the sums would cost the same).
//
// Probabilities, their difference and dS are rounded to bf16 as they become operands (the matrix instructions take nothing wider at this rate), which is at
// most 2^-8 of one, as for the results themselves; scores, statistics (in the dK/dV kernel as exact sums of bf16 values), sums, dP, D and dlambda are fp32.
// D_1 and D_2 come from O and O_2 as stored.  Against 64 bits a result is 0.0024 to 0.0031 of its size off, where rounding it alone is 0.0017.
//
// Bound by issue: at two wavefronts per SIMD the matrix pipe (37 % of the cycles forward) and the vector instructions (43 %) add up, as an MFMA hides
// about four vector instructions and a softmax of two maps has ten beside each.  Measured with 16 heads of 128, 8 sequences of 1 639 to 2 048 tokens,
// causal: forward 204 us (525 TFLOP/s, counting four head sizes of operations a pair), dQ 240, dK/dV 332; 16 heads of 64, 31 sequences of 366 to 523,
// unmasked: dQ 77, dK/dV 91.  One map of the whole head (attention_mfma.hip) takes 152 to 179 us forward and 504 to 538 backward on the first of them.
#include "diff_attention_tiles.hpp"
#include <cfloat>
#include <type_traits>

namespace {

constexpr float kSlack = 8.0f;                          // see diff_fwd_mfma_kernel
constexpr float kLowest = -FLT_MAX;                     // a maximum of nothing: finite, so that a step in which a query sees no key adds nothing, and below no score

// ------------------------------------------------------------------------------------ forward
// A tile of 64 keys goes in two steps of 32, so that both maps' scores (32 registers) and both accumulators (128 at head size 128) leave room
// for two wavefronts per SIMD, whose vector work and matrix instructions then overlap.
template <int HD, bool CAUSAL, int KS>
__global__ __launch_bounds__(256, HD == 64 && KS == 1 ? 3 : 2) void diff_fwd_mfma_kernel(DiffAttnArgs a) {
    extern __shared__ __attribute__((aligned(16))) char smem[];
    constexpr int TILE = 64 * HD * 2, NS = HD / 16, ND = HD / 32, AHEAD = 2, AHEAD_V = 1;
    constexpr int RING = KeySplit<KS>::RING;
    const uint32_t lds0 = lds_address(smem);
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 31, g = lane >> 5;
    int s, h, q0 = 0, split = 0;
    if constexpr (KS == 1) {
        const int item = blockIdx.x / a.n_heads;
        const int2 it = block_of(a, a.items_q, item);
        if (item >= block_count(a, 0)) return;
        if (a.direct && a.q_len[it.x] == 0) return;     // (in no list)
        s = it.x;
        q0 = it.y * 128;
        h = blockIdx.x - item * a.n_heads;
    } else {                                            // one block of queries in a sequence: no list
        split = blockIdx.x;
        h = blockIdx.y;
        s = blockIdx.z;
        if (a.q_len[s] == 0) return;
    }
    const int ql = a.q_len[s];
    const KeyRange range = KS == 1 ? KeyRange{0, a.k_len[s]} : split_keys(a, a.k_len[s], split);
    const int kl = range.count;
    const long long krow0 = (long long)a.k_row[s] + range.first;
    const long long qrow0 = a.q_row[s];
    const bf16_t* Q = (const bf16_t*)a.q + qrow0 * a.ldq + h * HD;
    const bf16_t* K = (const bf16_t*)a.k + krow0 * a.ldk + h * HD;
    const bf16_t* V = (const bf16_t*)a.v + krow0 * a.ldv + h * HD;
    KeySplit<KS> ks;
    ks.init(wave);
    const int qw0 = q0 + ks.group * 32;
    const int qi = qw0 + col;
    const int qi_c = qi < ql ? qi : ql - 1;

    bf16x8_t qf[NS];
#pragma unroll
    for (int i = 0; i < NS; ++i) qf[i] = *reinterpret_cast<const bf16x8_t*>(Q + (long long)qi_c * a.ldq + i * 16 + g * 8);

    PieceLoader<HD> ldK, ldV;
    ldK.setup(K, a.ldk, kl, wave, lane);
    ldV.setup(V, a.ldv, kl, wave, lane);
    FragOffsets<HD> at;
    at.init(lane);

    f32x16_t o[2][ND];
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int dt = 0; dt < ND; ++dt)
#pragma unroll
            for (int e = 0; e < 16; ++e) o[m][dt][e] = 0.f;
    float top[2] = {kLowest, kLowest}, l[2] = {0.f, 0.f};              // running maxima (in the exp2 domain) and sums
    const float c = a.scale * kLog2e;

    const int kv_end = CAUSAL ? min(kl, q0 + 128) : kl;
    const int wave_last = CAUSAL ? min(kl - 1, qw0 + 31) : kl - 1;     // last key this wavefront can see
    const int nb = (kv_end + 63) / 64;
    auto fetch = [&](int b) {                           // (of a block past the last one every row is past the end)
        const uint32_t n = lds0 + (b % RING) * (2 * TILE);
        ldK.issue(n, b * 64);
        ldV.issue(n + TILE, b * 64);
    };
    if (nb > 0)                                         // (a sequence without keys: zero output, nothing to fetch)
#pragma unroll
        for (int b = 0; b < RING - 1; ++b) fetch(b);
    // scores -> probabilities of map m in place.  The running maximum is raised, and what was summed so far rescaled, only where a score exceeds it
    // by more than kSlack: probabilities are then at most 2^kSlack times what they are relative to the true maximum, which costs no digits, and a
    // lane needs nothing of the lane that holds the other half of its column.
    auto soften = [&](f32x16_t& p, int m) {
        float x = -INFINITY;
#pragma unroll
        for (int e = 0; e < 16; e += 2) x = max3f(x, p[e], p[e + 1]);
        x *= c;
        if (__builtin_amdgcn_ballot_w64(x > top[m] + kSlack) != 0) {
            const float up = max3f(top[m], x, __shfl_xor(x, 32, 64));
            const float alpha = __builtin_amdgcn_exp2f(top[m] - up);
            l[m] *= alpha;
            top[m] = up;
#pragma unroll
            for (int dt = 0; dt < ND; ++dt)
#pragma unroll
                for (int e = 0; e < 16; ++e) o[m][dt][e] *= alpha;
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            p[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(p[e], c, -top[m]));
            l[m] += p[e];
        }
    };
    for (int b = 0; b < nb; ++b) {
        const int kv0 = b * 64;
        const char* sK = smem + (b % RING) * (2 * TILE);
        ring_wait<RING, 2 * (HD / 32)>();               // block b has landed; the stage of the block before is free
        if (RING > 2 || b + 1 < nb) fetch(b + RING - 1);
        if (kv0 > wave_last || qw0 >= ql) continue;
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) {
            if (kv0 + kt * 32 > wave_last || !ks.mine(2 * b + kt)) continue;      // the half beyond the last key this wavefront sees
            const char* tK = sK + kt * (32 * HD * 2);
            const char* tV = tK + TILE;
            f32x16_t p[2];
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int e = 0; e < 16; ++e) p[m][e] = 0.f;
            bf16x8_t fk[NS], fv[2 * ND];
            auto read_k = [&](int i) { fk[i] = at.row(tK, i); };
            auto read_v = [&](int i) { fv[i] = at.turned(tV + (i / ND) * (16 * HD * 2), i % ND); };
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) read_k(i);
#pragma unroll
            for (int i = 0; i < NS; ++i) {
                if (i + AHEAD < NS) read_k(i + AHEAD);
                __builtin_amdgcn_sched_barrier(kFence);
                p[i >= NS / 2] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fk[i], qf[i], p[i >= NS / 2], 0, 0, 0);
                __builtin_amdgcn_sched_barrier(kFence);
            }
            if (kv0 + kt * 32 + 32 > kl || (CAUSAL && kv0 + kt * 32 + 31 > qw0)) {
                int kbase = kv0 + kt * 32;              // (one real branch around the whole mask: see attention_mfma.hip)
                asm volatile("" : "+s"(kbase));
                const int last = (CAUSAL ? min(kl - 1, qi) : kl - 1) - kbase - 4 * g;      // last visible row, as this lane counts them
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (8 * (e >> 2) + (e & 3) > last) { p[0][e] = -INFINITY; p[1][e] = -INFINITY; }
            }
            soften(p[0], 0);
            soften(p[1], 1);
#pragma unroll
            for (int i = 0; i < AHEAD_V; ++i) read_v(i);
            bf16x8_t f1, f2;
#pragma unroll
            for (int i = 0; i < 2 * ND; ++i) {
                if (i + AHEAD_V < 2 * ND) read_v(i + AHEAD_V);
                if (i % ND == 0) { f1 = frag_from_acc(p[0], i / ND); f2 = frag_from_acc(p[1], i / ND); }
                __builtin_amdgcn_sched_barrier(kFence);
                o[0][i % ND] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fv[i], f1, o[0][i % ND], 0, 0, 0);
                o[1][i % ND] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fv[i], f2, o[1][i % ND], 0, 0, 0);
                __builtin_amdgcn_sched_barrier(kFence);
            }
        }
    }
    if constexpr (KS > 1) {
        __builtin_amdgcn_s_waitcnt(0x0F70);             // no transfer may still be writing LDS
        constexpr int N = 2 * ND * 16 + 4;
        join_splits<KS, N>(smem, ks, lane,
            [&](float* p) {
#pragma unroll
                for (int m = 0; m < 2; ++m) {
                    p[(2 * m) * 64] = top[m];
                    p[(2 * m + 1) * 64] = l[m];
#pragma unroll
                    for (int i = 0; i < ND * 16; ++i) p[(4 + m * ND * 16 + i) * 64] = o[m][i / 16][i % 16];
                }
            },
            [&](const float* p) {
#pragma unroll
                for (int m = 0; m < 2; ++m) {
                    const float other = p[(2 * m) * 64], up = fmaxf(top[m], other);
                    const float mine = __builtin_amdgcn_exp2f(top[m] - up), theirs = __builtin_amdgcn_exp2f(other - up);
                    l[m] = l[m] * mine + p[(2 * m + 1) * 64] * theirs;
                    top[m] = up;
#pragma unroll
                    for (int i = 0; i < ND * 16; ++i) o[m][i / 16][i % 16] = o[m][i / 16][i % 16] * mine + p[(4 + m * ND * 16 + i) * 64] * theirs;
                }
            });
        if (ks.split != 0) return;
    }
#pragma unroll
    for (int m = 0; m < 2; ++m) l[m] += __shfl_xor(l[m], 32, 64);
    if (qw0 >= ql) return;
    const long long row = qrow0 + qi;
    if (KS > 1 && a.k_splits > 1) {
        if (qi >= ql) return;
        const SplitPart to = split_part(a, h, row, split);
        if (g == 0) *reinterpret_cast<float4*>(to.stat) = make_float4(top[0], l[0], top[1], l[1]);
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int i = 0; i < ND * 4; ++i) {
                const f32x16_t& f = o[m][i / 4];
                const int e = 4 * (i % 4);
                *reinterpret_cast<float4*>(to.o[m] + 8 * i + 4 * g) = make_float4(f[e], f[e + 1], f[e + 2], f[e + 3]);
            }
        return;
    }
    const float r1 = l[0] > 0.f ? 1.0f / l[0] : 0.f, r2 = l[1] > 0.f ? 1.0f / l[1] : 0.f, lam = a.lambda[h];
#pragma unroll
    for (int dt = 0; dt < ND; ++dt)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            o[1][dt][e] *= r2;
            o[0][dt][e] = o[0][dt][e] * r1 - lam * o[1][dt][e];
        }
    store_cols16<HD>(o[0], 1.0f, 1.0f, (bf16_t*)a.o + row * a.ldo + h * HD, g, qi < ql);
    if (a.o2) store_cols16<HD>(o[1], 1.0f, 1.0f, (bf16_t*)a.o2 + row * a.ldo + h * HD, g, qi < ql);
    if (g == 0 && qi < ql) {
        a.lse[(size_t)(2 * h) * a.lse_stride + row] = (top[0] + __builtin_amdgcn_logf(l[0])) * kLn2;
        a.lse[(size_t)(2 * h + 1) * a.lse_stride + row] = (top[1] + __builtin_amdgcn_logf(l[1])) * kLn2;
    }
}

template <int HD, bool CAUSAL, int KS>
ds_status fwd_launch(const DiffAttnArgs& a, hipStream_t st) {
    static bool attr = false;
    auto kern = diff_fwd_mfma_kernel<HD, CAUSAL, KS>;
    const int smem = KeySplit<KS>::RING * 2 * (64 * HD * 2);
    const ds_status r = set_smem(kern, smem, attr);
    if (r != DS_OK) return r;
    const dim3 grid = KS == 1 ? dim3((unsigned)(a.direct ? a.n_seq : a.max_items_q) * a.n_heads) : dim3(a.k_splits, a.n_heads, a.n_seq);
    hipLaunchKernelGGL(kern, grid, dim3(256), smem, st, a);
    DS_LAUNCH_CHECK();
    return KS > 1 && a.k_splits > 1 ? diff_join(a, st) : DS_OK;
}

}  // namespace

// what the matrix-core kernels ask beside a scratch that is large enough: 16-byte accesses, 64 rows of a tile within a 31-bit byte offset
bool diff_mfma_supported(const DiffAttnArgs& a) {
    if (a.dtype != DS_DTYPE_BF16 || (a.head_dim != 64 && a.head_dim != 128)) return false;
    const long long ld_max = 1LL << 23;
    for (const long long ld : {a.ldq, a.ldk, a.ldv, a.ldo})
        if (ld % 8 || ld >= ld_max) return false;
    for (const void* p : {a.q, a.k, a.v, (const void*)a.o, (const void*)a.o2, a.d_o, (const void*)a.dq, (const void*)a.dk, (const void*)a.dv})
        if ((uintptr_t)p & 15) return false;
    // the grids: one work-group per (block of 128 rows, head), and at most eight for a head beside them; fewer than 2^32 threads
    const long long most = 0xffffffffLL / 256;
    return ((long long)a.q_total_rows / 128 + a.n_seq + 8) * a.n_heads <= most && ((long long)a.k_total_rows / 128 + a.n_seq + 8) * a.n_heads <= most;
}

int diff_mfma_sharing(const DiffAttnArgs& a) { return sharing(a); }
bool diff_mfma_direct(const DiffAttnArgs& a, bool backward) {
    return one_block_each(a, a.max_q_len, a.max_k_len) && (!backward || one_block_each(a, a.max_k_len, a.max_q_len));
}

ds_status diff_fwd_mfma(const DiffAttnArgs& a0, hipStream_t st) {
    return diff_by_kind(a0, [&](auto hd, auto causal, auto split) {
        DiffAttnArgs a = a0;
        a.direct = diff_mfma_direct(a, false);
        const ds_status r = split == 1 && !a.direct ? attn_prepare_lists(a, false, st) : DS_OK;
        return r != DS_OK ? r : fwd_launch<decltype(hd)::value, decltype(causal)::value, decltype(split)::value>(a, st);
    });
}
