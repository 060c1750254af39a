// The backward pass of diff_attention_fwd.hip, which says how two maps share the products.
//
// Split into a dQ kernel and a dK/dV kernel, so that every result has one owner: no atomics, the same result every time.
#include "diff_attention_tiles.hpp"
#include <type_traits>

namespace {

// A float as the sum of three bf16 values, exactly: the difference from the first has at most 16 bits, that from the second at most 8.
struct BfParts {
    bf16_t p[3];
    __device__ __forceinline__ explicit BfParts(float v) {
#pragma unroll
        for (int i = 0; i < 3; ++i) {
            p[i] = (bf16_t)v;
            v -= (float)p[i];
        }
    }
    __device__ __forceinline__ static uint32_t bits(bf16_t b) { return __builtin_bit_cast(unsigned short, b); }
    __device__ __forceinline__ uint32_t half(int g) const { return g ? bits(p[2]) : bits(p[0]) | bits(p[1]) << 16; }
};
constexpr int kStatTile = 64 * 32;                      // bytes

// ------------------------------------------------------------------------------------ backward: dQ (and the statistics, the parts of dlambda)
// For the dK/dV kernel a query leaves one entry of sixteen bf16 values: lse_1 / scale, lse_2 / scale, D_1 and D_2 - D_1, each as the sum of three, which
// together have all 24 bits of it: {first, second} of the four in the first half, {third, 0} of the four in the second (see BfParts).
template <int HD, bool CAUSAL, int KS>
__global__ __launch_bounds__(256, 2) void diff_bwd_dq_mfma_kernel(DiffAttnArgs a) {
    extern __shared__ __attribute__((aligned(16))) char smem[];
    constexpr int TILE = 64 * HD * 2, NS = HD / 16, ND = HD / 32, AHEAD = 2;
    constexpr int RING = KeySplit<KS>::RING;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 31, g = lane >> 5;
    const int item = blockIdx.x / a.n_heads, h = blockIdx.x - item * a.n_heads;
    if (item >= block_count(a, 0)) return;
    const int2 it = block_of(a, a.items_q, item);
    const int s = it.x, q0 = it.y * 128;
    const int ql = a.q_len[s], kl = a.k_len[s];
    if (ql == 0) return;                                // (in no list)
    const long long qrow0 = a.q_row[s];
    const bf16_t* Q = (const bf16_t*)a.q + qrow0 * a.ldq + h * HD;
    const bf16_t* dO = (const bf16_t*)a.d_o + qrow0 * a.ldo + h * HD;
    const bf16_t* O = (const bf16_t*)a.o + qrow0 * a.ldo + h * HD;
    const bf16_t* O2 = (const bf16_t*)a.o2 + qrow0 * a.ldo + h * HD;
    const bf16_t* K = (const bf16_t*)a.k + (long long)a.k_row[s] * a.ldk + h * HD;
    const bf16_t* V = (const bf16_t*)a.v + (long long)a.k_row[s] * a.ldv + h * HD;
    KeySplit<KS> ks;
    ks.init(wave);
    const int qw0 = q0 + ks.group * 32;
    const int qi = qw0 + col;
    const int qi_c = qi < ql ? qi : ql - 1;

    const uint32_t lds0 = lds_address(smem);
    PieceLoader<HD> ldK, ldV;
    ldK.setup(K, a.ldk, kl, wave, lane);
    ldV.setup(V, a.ldv, kl, wave, lane);
    const int kv_end = CAUSAL ? min(kl, q0 + 128) : kl;
    const int wave_last = CAUSAL ? min(kl - 1, qw0 + 31) : kl - 1;
    const int nb = (kv_end + 63) / 64;
    auto fetch = [&](int b) {                           // (of a block past the last one every row is past the end)
        const uint32_t n = lds0 + (b % RING) * (2 * TILE);
        ldK.issue(n, b * 64);
        ldV.issue(n + TILE, b * 64);
    };
    if (nb > 0)
#pragma unroll
        for (int b = 0; b < RING - 1; ++b) fetch(b);

    const float lam = a.lambda[h];
    bf16x8_t qf[NS], dof[NS];
    float d1 = 0.f, d2 = 0.f;
#pragma unroll
    for (int i = 0; i < NS; ++i) {
        qf[i] = *reinterpret_cast<const bf16x8_t*>(Q + (long long)qi_c * a.ldq + i * 16 + g * 8);
        dof[i] = *reinterpret_cast<const bf16x8_t*>(dO + (long long)qi_c * a.ldo + i * 16 + g * 8);
        const bf16x8_t of = *reinterpret_cast<const bf16x8_t*>(O + (long long)qi_c * a.ldo + i * 16 + g * 8);
        const bf16x8_t of2 = *reinterpret_cast<const bf16x8_t*>(O2 + (long long)qi_c * a.ldo + i * 16 + g * 8);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            d1 = __builtin_fmaf((float)of[j], (float)dof[i][j], d1);
            d2 = __builtin_fmaf((float)of2[j], (float)dof[i][j], d2);
        }
    }
    d2 += __shfl_xor(d2, 32, 64);
    d1 += __shfl_xor(d1, 32, 64);
    d1 += lam * d2;
    const float lse1 = a.lse[(size_t)(2 * h) * a.lse_stride + qrow0 + qi_c], lse2 = a.lse[(size_t)(2 * h + 1) * a.lse_stride + qrow0 + qi_c];
    if (qi < ql && ks.split == 0)                       // lane half g writes half g
        reinterpret_cast<uint4*>(a.aug)[2 * ((size_t)h * a.q_total_rows + qrow0 + qi) + g] =
            make_uint4(BfParts(lse1 * (1.0f / a.scale)).half(g), BfParts(lse2 * (1.0f / a.scale)).half(g), BfParts(d1).half(g), BfParts(d2 - d1).half(g));
    const float e1 = lse1 * kLog2e, e2 = lse2 * kLog2e;
    const float c = a.scale * kLog2e;

    FragOffsets<HD> at;
    at.init(lane);

    f32x16_t gacc[ND];
#pragma unroll
    for (int dt = 0; dt < ND; ++dt)
#pragma unroll
        for (int e = 0; e < 16; ++e) gacc[dt][e] = 0.f;
    float lam_sum = 0.f;

    for (int b = 0; b < nb; ++b) {
        const int kv0 = b * 64;
        const char* sK = smem + (b % RING) * (2 * TILE);
        ring_wait<RING, 2 * (HD / 32)>();               // block b has landed; the stage of the block before is free
        if (RING > 2 || b + 1 < nb) fetch(b + RING - 1);
        if (kv0 > wave_last || qw0 >= ql) continue;
        const bool need_mask = (kv0 + 64 > kl) || (CAUSAL && kv0 + 63 > qw0);
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) {
            if (kv0 + kt * 32 > wave_last || !ks.mine(2 * b + kt)) continue;      // the half beyond the last key this wavefront sees
            f32x16_t p1, p2, gr;
#pragma unroll
            for (int e = 0; e < 16; ++e) { p1[e] = 0.f; p2[e] = 0.f; gr[e] = 0.f; }
            const char* tK = sK + kt * (32 * HD * 2);
            bf16x8_t fk[NS], fv[NS];
            auto read_kv = [&](int i) {
                fk[i] = at.row(tK, i);
                fv[i] = at.row(tK + TILE, i);
            };
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) read_kv(i);
#pragma unroll
            for (int i = 0; i < NS; ++i) {
                if (i + AHEAD < NS) read_kv(i + AHEAD);
                __builtin_amdgcn_sched_barrier(kFence);
                if (i < NS / 2) p1 = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fk[i], qf[i], p1, 0, 0, 0);
                else p2 = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fk[i], qf[i], p2, 0, 0, 0);
                gr = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fv[i], dof[i], gr, 0, 0, 0);
                __builtin_amdgcn_sched_barrier(kFence);
            }
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                p1[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(p1[e], c, -e1));
                p2[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(p2[e], c, -e2));
            }
            if (need_mask) {
                int kbase = kv0 + kt * 32;
                asm volatile("" : "+s"(kbase));
                const int last = (CAUSAL ? min(kl - 1, qi) : kl - 1) - kbase - 4 * g;  // last visible row, as this lane counts them
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (8 * (e >> 2) + (e & 3) > last) { p1[e] = 0.f; p2[e] = 0.f; gr[e] = 0.f; }
            }
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                lam_sum = __builtin_fmaf(p2[e], gr[e], lam_sum);
                p1[e] *= gr[e] - d1;                                  // dS_1^T
                p2[e] *= gr[e] - d2;                                  // dS_2^T / -lambda
            }
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const bf16x8_t f1 = frag_from_acc(p1, u), f2 = frag_from_acc(p2, u);
#pragma unroll
                for (int dt = 0; dt < ND; ++dt) {
                    const bf16x8_t kt_f = at.turned(tK + u * (16 * HD * 2), dt);
                    gacc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kt_f, dt < ND / 2 ? f1 : f2, gacc[dt], 0, 0, 0);
                }
            }
        }
    }
    if constexpr (KS > 1) {
        __builtin_amdgcn_s_waitcnt(0x0F70);             // no transfer may still be writing LDS
        join_splits<KS, ND * 16 + 1>(smem, ks, lane,
            [&](float* p) {
                p[0] = lam_sum;
#pragma unroll
                for (int i = 0; i < ND * 16; ++i) p[(1 + i) * 64] = gacc[i / 16][i % 16];
            },
            [&](const float* p) {
                lam_sum += p[0];
#pragma unroll
                for (int i = 0; i < ND * 16; ++i) gacc[i / 16][i % 16] += p[(1 + i) * 64];
            });
        if (ks.split != 0) return;
    }
    lam_sum = wave_sum(qi < ql ? lam_sum : 0.f);
    if (lane == 0 && qw0 < ql) a.lam_part[(size_t)h * a.q_total_rows + qrow0 + qw0] = lam_sum;
    if (qw0 >= ql) return;
    store_cols16<HD>(gacc, a.scale, -lam * a.scale, (bf16_t*)a.dq + (qrow0 + qi) * a.ldq + h * HD, g, qi < ql);
}

// ------------------------------------------------------------------------------------ backward: dK, dV
// A ring of four stages of Q tile, dO tile ([64][HD]) and statistics tile ([64 queries][16] bf16, see above), three blocks in flight.  One matrix
// instruction with the statistics as its A operand and -1 in the slots of a value subtracts it, with all its bits: score_i - lse_i / scale and, from the
// one dP, dP - D_1 and dP - D_2.  At head size 128 work-groups are persistent, one to a compute unit (see attention_mfma.hip).
template <int HD, bool CAUSAL>
__global__ __launch_bounds__(256, HD == 64 ? 2 : 1) void diff_bwd_dkv_mfma_kernel(DiffAttnArgs a) {
    extern __shared__ __attribute__((aligned(16))) char smem[];
    constexpr int TILE = 64 * HD * 2;
    constexpr int STAGE = 2 * TILE + kStatTile;
    constexpr int NS = 4;
    constexpr bool PS = HD == 128;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 31, g = lane >> 5;
    const uint32_t lds0 = lds_address(smem);
    volatile int* s_next = reinterpret_cast<volatile int*>(smem + NS * STAGE);      // two words used in turn (an item without steps has one barrier only)
    int turn = 0;
    char* s_zero = smem + NS * STAGE + 64;              // 32 rows of zeros
    PieceLoader<HD> ldQ, ldO;
    ldQ.setup(nullptr, a.ldq, 0, wave, lane);
    ldO.setup(nullptr, a.ldo, 0, wave, lane);
    const int first = (a.n_heads + 7) / 8 * 8;          // the first work-groups sum up dlambda
    if ((int)blockIdx.x < first) {
        if ((int)blockIdx.x < a.n_heads) sum_dlambda<32, 256>(a, blockIdx.x, reinterpret_cast<float*>(smem));
        return;
    }
    LateDraw draw(a, 1, first);
    int kw0, ki, kl, ql, h, q_begin, nb;
    long long krow0;
    const char* aug_src;
    float lam;
    bf16x8_t kf[HD / 16], vf[HD / 16];
    // block blk -> stage blk % 4 by direct transfers (the statistics by wavefronts 0 and 1).  Queries past the last one are zeros in
    // all three: P is 1 there, and multiplies zeros (dV), and dS is 1 (0 - 0): no mask
    auto issue_block = [&](int blk) {
        const uint32_t n = lds0 + (blk & (NS - 1)) * STAGE;
        const int q0 = q_begin + blk * 64;
        ldQ.issue(n, q0);
        ldO.issue(n + TILE, q0);
        if (wave < 2) lds_dma16_buffer(make_raw_buffer(aug_src + (long long)q0 * 32, (uint32_t)max(0, min(64, ql - q0)) * 32), (uint32_t)(wave * 64 + lane) * 16, n + 2 * TILE + wave * 1024);
    };
    auto begin_item = [&] {
        const int item = draw.index() / a.n_heads;
        h = draw.index() - item * a.n_heads;
        const int2 it = block_of(a, a.items_k, item);
        const int s = __builtin_amdgcn_readfirstlane(it.x), k0 = __builtin_amdgcn_readfirstlane(it.y) * 128;
        ql = __builtin_amdgcn_readfirstlane(a.q_len[s]);
        kl = __builtin_amdgcn_readfirstlane(a.k_len[s]);
        const long long qrow0 = __builtin_amdgcn_readfirstlane(a.q_row[s]);
        krow0 = __builtin_amdgcn_readfirstlane(a.k_row[s]);
        lam = a.lambda[h];
        kw0 = k0 + wave * 32;
        ki = kw0 + col;
        q_begin = CAUSAL ? k0 : 0;
        nb = (ql - q_begin + 63) / 64;                  // (none: keys beyond the last query of a causal sequence)
        ldQ.base = reinterpret_cast<const char*>((const bf16_t*)a.q + qrow0 * a.ldq + h * HD);
        ldO.base = reinterpret_cast<const char*>((const bf16_t*)a.d_o + qrow0 * a.ldo + h * HD);
        ldQ.n_valid = ldO.n_valid = ql;
        aug_src = a.aug + ((size_t)h * a.q_total_rows + qrow0) * 32;
        if (nb > 0) {
            issue_block(0);
            issue_block(1);
            issue_block(2);
        }
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
    if (a.direct && a.k_len[a.n_seq - 1 - draw.index() / a.n_heads] == 0) return;        // (in no list)
    begin_item();
    for (int i = tid; i < 64 * HD / 16; i += 256) reinterpret_cast<uint4*>(s_zero)[i] = make_uint4(0u, 0u, 0u, 0u);
    bf16x8_t minus;                                     // -1 in the contraction slots 0, 1 (lane half 0) and 8, 9 (lane half 1), where a statistic's parts are put
#pragma unroll
    for (int j = 0; j < 8; ++j) minus[j] = (bf16_t)(j < 2 ? -1.0f : 0.0f);
    const float c = a.scale * kLog2e;

    FragOffsets<HD> at;
    at.init(lane);

    f32x16_t dkacc[HD / 32], dvacc[HD / 32];
    for (;;) {
#pragma unroll
    for (int dt = 0; dt < HD / 32; ++dt)
#pragma unroll
        for (int e = 0; e < 16; ++e) { dkacc[dt][e] = 0.f; dvacc[dt][e] = 0.f; }

    int next = 0;
    if (PS) next = draw.take();                         // (needed after the loop)
    // ordinary loads and stores are complete before the loop (left to the compiler its waits would sit inside it), and so are the zeros of s_zero
    __builtin_amdgcn_s_waitcnt(0x0070);
    const bool wave_has_keys = kw0 < kl;
    // one step = one 64-query block, straight code, with the mask as selects or without (see attention_mfma.hip)
    auto step = [&](int b, auto masked_t) {
        constexpr bool MASKED = decltype(masked_t)::value;
        const int q0 = q_begin + b * 64;
        const char* sQ = smem + (b & (NS - 1)) * STAGE;
        const char* sdO = sQ + TILE;
        const char* s_stat = sdO + TILE;
        // block b has landed for this wavefront (the two newest may still be in flight), then for everybody; the stage read before is free
        if (wave < 2) __builtin_amdgcn_s_waitcnt(vmcnt_imm(2 * (2 * (HD / 32) + 1)));
        else __builtin_amdgcn_s_waitcnt(vmcnt_imm(2 * (2 * (HD / 32))));
        __builtin_amdgcn_s_barrier();
        issue_block(b + 3);
        if (!wave_has_keys) return;
        if (MASKED && q0 + 63 < kw0) return;
        const int first = ki - q0 - 4 * g;             // the first query of the block that sees this lane's key, as this lane counts its rows
        // two 32-query halves: the exponentials of half 0 between the first products of half 1, those of half 1 between the second products of half 0
        // (without the freedom to move vector instructions across, the register allocation of the causal kernel at head size 128 copies fewer
        // accumulators: 407 us against 452 at 8 sequences of up to 2048, 16 heads; the unmasked one is better with it, 8.6 against 9.5 us per 32 keys)
        constexpr int FENCE = HD == 128 && !CAUSAL ? kFence : 0;
        constexpr int NA = HD / 16, AHEAD = 2, ND = 2 * (HD / 32), AHEAD_D = 2;
        f32x16_t sa[2], sb[2], ga[2];
        u32x4_t fs[2];
        bf16x8_t fq[NA], fo[NA], td[ND], tq[ND], pf[2][2], f1[2][2], f2[2][2];
        auto less = [&](f32x16_t x, uint32_t parts) {   // x minus a statistic of its rows
            const u32x4_t f = {parts, 0u, 0u, 0u};
            return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, f), minus, x, 0, 0, 0);
        };
        auto read_a = [&](int qt, int i) {
            fq[i] = at.row(sQ + qt * (32 * HD * 2), i);
            fo[i] = at.row(sdO + qt * (32 * HD * 2), i);
        };
        auto hidden = [&](int qt, int e) { return MASKED && qt * 32 + 8 * (e >> 2) + (e & 3) < first; };
        // scores and dP of half qt to operands, in 32 pieces: P_1 and dS_1 first (16), then P_2, the difference and dS_2
        auto soften = [&](int qt, int i) {
            const int e = i & 15;
            if (i < 16) {
                sa[qt][e] = __builtin_amdgcn_exp2f(sa[qt][e] * c);
                const float d = hidden(qt, e) ? 0.f : sa[qt][e] * ga[qt][e];
                f1[qt][e >> 3][e & 7] = (bf16_t)d;
            } else {
                const float p2 = __builtin_amdgcn_exp2f(sb[qt][e] * c);
                pf[qt][e >> 3][e & 7] = (bf16_t)(hidden(qt, e) ? 0.f : __builtin_fmaf(-lam, p2, sa[qt][e]));
                f2[qt][e >> 3][e & 7] = (bf16_t)(hidden(qt, e) ? 0.f : p2 * ga[qt][e]);      // dS_2 / -lambda
            }
            if (i == 15) ga[qt] = less(ga[qt], fs[qt][3]);       // dP - D_2: the fourth value is D_2 - D_1
        };
        auto phase_a = [&](int qt, bool with_prev) {
#pragma unroll
            for (int e = 0; e < 16; ++e) { sa[qt][e] = 0.f; sb[qt][e] = 0.f; ga[qt][e] = 0.f; }
            fs[qt] = *reinterpret_cast<const u32x4_t*>(s_stat + (qt * 32 + col) * 32 + g * 16);
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) read_a(qt, i);
#pragma unroll
            for (int i = 0; i < NA; ++i) {
                if (i + AHEAD < NA) read_a(qt, i + AHEAD);
                __builtin_amdgcn_sched_barrier(FENCE);
                if (i < NA / 2) sa[qt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fq[i], kf[i], sa[qt], 0, 0, 0);
                else sb[qt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fq[i], kf[i], sb[qt], 0, 0, 0);
                ga[qt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fo[i], vf[i], ga[qt], 0, 0, 0);
                __builtin_amdgcn_sched_barrier(FENCE);
                if (with_prev) {
#pragma unroll
                    for (int e = i * (32 / NA); e < (i + 1) * (32 / NA); ++e) soften(qt ^ 1, e);
                }
            }
            sa[qt] = less(sa[qt], fs[qt][0]);
            sb[qt] = less(sb[qt], fs[qt][1]);
            ga[qt] = less(ga[qt], fs[qt][2]);
        };
        auto phase_d = [&](int qt, bool with_next) {
            // a half that no key of this wavefront sees: zeros instead of its rows, which may hold infinities (0 x Inf is NaN)
            const bool none = MASKED && q0 + 32 * qt + 31 < kw0;
            const char* rO = none ? s_zero : sdO + qt * (32 * HD * 2);
            const char* rQ = none ? s_zero : sQ + qt * (32 * HD * 2);
            auto read_d = [&](int j) {
                td[j] = at.turned(rO + (j / (HD / 32)) * (16 * HD * 2), j % (HD / 32));
                tq[j] = at.turned(rQ + (j / (HD / 32)) * (16 * HD * 2), j % (HD / 32));
            };
#pragma unroll
            for (int j = 0; j < AHEAD_D; ++j) read_d(j);
#pragma unroll
            for (int j = 0; j < ND; ++j) {
                if (j + AHEAD_D < ND) read_d(j + AHEAD_D);
                __builtin_amdgcn_sched_barrier(FENCE);
                const int dt = j % (HD / 32), u = j / (HD / 32);
                dvacc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(td[j], pf[qt][u], dvacc[dt], 0, 0, 0);
                dkacc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(tq[j], dt < HD / 64 ? f1[qt][u] : f2[qt][u], dkacc[dt], 0, 0, 0);
                __builtin_amdgcn_sched_barrier(FENCE);
                if (with_next) {
#pragma unroll
                    for (int e = j * (32 / ND); e < (j + 1) * (32 / ND); ++e) soften(qt ^ 1, e);
                }
            }
        };
        phase_a(0, false);
        phase_a(1, true);
        phase_d(0, true);
        phase_d(1, false);
    };
    const int n_diag = CAUSAL ? min(2, nb) : 0;         // causal: queries k0 .. k0+127 meet this block's own keys
    int b = 0;
    if constexpr (CAUSAL)
        for (; b < n_diag; ++b) step(b, std::true_type{});
    for (; b < nb; ++b) step(b, std::false_type{});
    __builtin_amdgcn_s_waitcnt(0x0F70);                 // no transfer may still be writing LDS ...
    const bool store = ki < kl;
    const float lam_of_item = lam;                      // (begin_item moves on)
    bf16_t* dk = (bf16_t*)a.dk + (krow0 + ki) * a.ldk + h * HD;
    bf16_t* dv = (bf16_t*)a.dv + (krow0 + ki) * a.ldv + h * HD;
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
    if (wave_has_keys) {
        store_cols16<HD>(dkacc, a.scale, -lam_of_item * a.scale, dk, g, store);
        store_cols16<HD>(dvacc, 1.0f, 1.0f, dv, g, store);
    }
    if (!more) break;
    }   // for (;;): the next item
    if (PS) draw.finish();
}

template <int HD, bool CAUSAL, int KS>
ds_status bwd_launch(const DiffAttnArgs& a, hipStream_t st) {
    static bool attr_q = false, attr_kv = false;
    auto kq = diff_bwd_dq_mfma_kernel<HD, CAUSAL, KS>;
    auto kkv = diff_bwd_dkv_mfma_kernel<HD, CAUSAL>;
    const int smem_q = KeySplit<KS>::RING * 2 * (64 * HD * 2);
    const int smem_kv = 4 * (2 * (64 * HD * 2) + kStatTile) + 64 + 64 * HD; // stages, draws, zeros
    ds_status r = set_smem(kq, smem_q, attr_q);
    if (r != DS_OK) return r;
    r = set_smem(kkv, smem_kv, attr_kv);
    if (r != DS_OK) return r;
    hipLaunchKernelGGL(kq, dim3((unsigned)(a.direct ? a.n_seq : a.max_items_q) * a.n_heads), dim3(256), smem_q, st, a);
    DS_LAUNCH_CHECK();
    const unsigned items_kv = (unsigned)(a.direct ? a.n_seq : a.max_items_k) * a.n_heads, for_dlambda = (a.n_heads + 7) / 8 * 8;
    hipLaunchKernelGGL(kkv, dim3((HD == 128 && !a.direct ? persistent_grid(items_kv) : items_kv) + for_dlambda), dim3(256), smem_kv, st, a);
    DS_LAUNCH_CHECK();
    return DS_OK;
}

}  // namespace

ds_status diff_bwd_mfma(const DiffAttnArgs& a0, hipStream_t st) {
    DiffAttnArgs a = a0;
    a.direct = diff_mfma_direct(a, true);
    const ds_status r = a.direct ? DS_OK : attn_prepare_lists(a, true, st);
    if (r != DS_OK) return r;
    return diff_by_kind(a, [&](auto hd, auto causal, auto split) { return bwd_launch<decltype(hd)::value, decltype(causal)::value, decltype(split)::value>(a, st); });
}
