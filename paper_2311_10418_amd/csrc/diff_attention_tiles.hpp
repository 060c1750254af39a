// What the matrix-core kernels of differential attention share beside attention_tiles.hpp.
#pragma once
#include "attention_tiles.hpp"
#include "diff_attention.hpp"
#include <type_traits>

namespace {

// Transfers of 64-row tiles, 1 KB (4 rows of 128 columns or 8 of 64) at a time, HD / 32 per wavefront and tile, through a raw buffer that ends
// at the last valid row: rows past it arrive as zeros.  The swizzled chunk of a lane in transfer i is that of transfer 0 with i
// (HD = 128) or 2 i flipped in, so that one register per tensor and one for the chunk make every offset.
template <int HD> struct PieceLoader {
    static constexpr int PW = HD / 32, ROWS = 512 / HD;               // transfers, rows per transfer
    const char* base;
    int ld2, n_valid;
    uint32_t row0, chunk0, lds_off;
    __device__ __forceinline__ void setup(const bf16_t* base_, long long ld_, int n_valid_, int wave, int lane) {
        base = (const char*)base_; ld2 = (int)ld_ * 2; n_valid = n_valid_; lds_off = wave * (PW * 1024);
        const int u = wave * PW * 64 + lane;
        row0 = (uint32_t)(TileLoader<HD>::row_of(u) * ld2);
        chunk0 = (uint32_t)TileLoader<HD>::chunk_of(u) * 16;
    }
    // rows r0 .. r0+63 -> the tile at LDS address lds_tile, one transfer or all
    __device__ __forceinline__ i32x4_t rows(int r0) const { return make_raw_buffer(base + (long long)r0 * ld2, (uint32_t)max(0, min(64, n_valid - r0)) * (uint32_t)ld2); }
    __device__ __forceinline__ void piece(i32x4_t buf, int i, uint32_t lds_tile) const {
        lds_dma16_buffer(buf, row0 + (uint32_t)(i * ROWS * ld2) + (chunk0 ^ (uint32_t)(i * (HD == 128 ? 16 : 32))), lds_tile + lds_off + i * 1024);
    }
    __device__ __forceinline__ void issue(uint32_t lds_tile, int r0) const {
        const i32x4_t buf = rows(r0);
#pragma unroll
        for (int i = 0; i < PW; ++i) piece(buf, i, lds_tile);
    }
};

// This lane's offset in a tile for the fragments of the first product, and for transpose reads; the k-th 16 features or the dt-th 32 features are
// the same with k << 5 or dt << 6 flipped in: three registers instead of one per fragment.
template <int HD> struct FragOffsets {
    uint32_t rows, lo, hi;
    __device__ __forceinline__ void init(int lane) {
        const int col = lane & 31, g = lane >> 5;
        rows = (uint32_t)(col * (HD * 2) + ((g ^ swz<HD>(col)) << 4));
        TrOffsets<HD> t;
        t.init(lane);
        lo = t.lo[0];
        hi = t.hi[0];
    }
    // features 16 k .. of the 32 rows at t
    __device__ __forceinline__ bf16x8_t row(const char* t, int k) const { return *reinterpret_cast<const bf16x8_t*>(t + (rows ^ (uint32_t)(k << 5))); }
    // features 32 dt .. of the 16 rows at t, turned
    __device__ __forceinline__ bf16x8_t turned(const char* t, int dt) const {
        const s16x4_t a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_ptr)(t + (lo ^ (uint32_t)(dt << 6))));
        const s16x4_t b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_ptr)(t + (hi ^ (uint32_t)(dt << 6))));
        const s16x8_t v = __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
        return __builtin_bit_cast(bf16x8_t, v);
    }
};

// The block of 128 rows that belongs to a place in a launch, longest sequences first (a plan lists them by ascending length), and their number.
__device__ __forceinline__ int2 block_of(const DiffAttnArgs& a, const int2* list, int item) { return a.direct ? make_int2(a.n_seq - 1 - item, 0) : list[item]; }
__device__ __forceinline__ int block_count(const DiffAttnArgs& a, int list) { return a.direct ? a.n_seq : a.n_items[list]; }
// No list where every sequence has one block and the order does not matter much: one work-group for a compute unit at most, or (head size 64, whose dK/dV
// kernel is not persistent) all of them short and not too many.  Launch and kernel of the list take 3 to 4 us.  With -> without, forward / backward, us, 16
// heads of 64: 16 sequences of 96 tokens 10.1 -> 7.0 / 20.0 -> 16.8, 64 of 128 23.1 -> 19.7 / 61.2 -> 58.7, 256 of 32 25.5 -> 21.6 / 86.9 -> 83.1; but 256 of
// 128 85 -> 90 / 238 -> 242.
inline bool one_block_each(const DiffAttnArgs& a, int max_len, int other_len) {
    const long long items = (long long)a.n_seq * a.n_heads, units = kDiffUnits;
    return max_len <= 128 && (items <= units || (a.head_dim == 64 && other_len <= 128 && items * max_len <= 1024 * units));
}

// WorkDraw for a launch whose first work-groups (a multiple of 8) do something else.  Without a list every work-group has one item and draws no other.
struct LateDraw : WorkDraw {
    int groups;
    bool once;
    __device__ __forceinline__ LateDraw(const DiffAttnArgs& a, int list, int first) : WorkDraw(a, list), groups((int)gridDim.x - first), once(a.direct) {
        k = ((int)blockIdx.x - first) >> 3;
        total = block_count(a, list) * a.n_heads;
    }
    __device__ __forceinline__ int take() const {
        if (once) return 0x7fffff00 >> 3;               // past every item
        int next = 0;
        if (threadIdx.x == 0) next = (groups >> 3) + __hip_atomic_fetch_add(ctr + xcd, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        return next;
    }
    __device__ __forceinline__ void finish() const {
        if (threadIdx.x != 0 || once) return;
        if (__hip_atomic_fetch_add(ctr + 8, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == groups - 1) {
#pragma unroll
            for (int i = 0; i < 9; ++i) ctr[i] = 0;
        }
    }
};

// Short queries (at most 64 or 32 in every sequence) of few sequences and heads: a work-group's four wavefronts hold two or one blocks of 32
// queries, and KS = 2 or 4 of them share one, each taking every KS-th step of 32 keys; what they have is joined through LDS in the end.  Tiles then
// come in a ring of four, three blocks of keys in flight: with few queries nothing else hides the transfers.  diff_by_kind has the rule.
template <int KS> struct KeySplit {
    static constexpr int RING = KS > 1 ? 4 : 2, GROUPS = 4 / KS;       // stages; blocks of 32 queries
    int split, group;
    __device__ __forceinline__ void init(int wave) {
        group = wave % GROUPS;
        split = wave / GROUPS;
    }
    __device__ __forceinline__ bool mine(int step) const { return KS == 1 || step % KS == split; }
};
// Waits until block b of a ring has landed for everybody, `transfers` per wavefront and block; the stage before is free then.
template <int RING, int TRANSFERS> __device__ __forceinline__ void ring_wait() {
    if constexpr (RING == 2) __builtin_amdgcn_s_waitcnt(0x0F70);
    else __builtin_amdgcn_s_waitcnt(vmcnt_imm((RING - 2) * TRANSFERS));
    __builtin_amdgcn_s_barrier();
}
// The wavefronts of splits KS / 2 .. write N registers per lane each, those of the lower half read and `join` them, then a quarter and so on.
// lds: two wavefronts write at a time at most: 2 x N x 256 bytes.  Every wavefront of the work-group calls it.
template <int KS, int N, class Put, class Join>
__device__ __forceinline__ void join_splits(char* lds, const KeySplit<KS>& ks, int lane, Put put, Join join) {
    constexpr int GROUPS = 4 / KS;
#pragma unroll
    for (int half = KS / 2; half >= 1; half /= 2) {
        __syncthreads();                                // what the memory held before has been read
        float* p = reinterpret_cast<float*>(lds) + (size_t)((ks.split % half) * GROUPS + ks.group) * N * 64 + lane;
        if (ks.split >= half && ks.split < 2 * half) put(p);
        __syncthreads();
        if (ks.split < half) join(p);
    }
}

// Stores a transposed [HD x 32] accumulator block times mul (first half of the features) or mul2 (second half): lane column = row `row` of the output.
// A lane holds 4 of every 8 features, the lane 32 further on the other 4: they swap, so that each has 8 of every 16 and the stores are 16 bytes wide.
// Every lane of the wavefront takes part; `on` says whether this lane's row is stored.
template <int HD>
__device__ __forceinline__ void store_cols16(const f32x16_t (&acc)[HD / 32], float mul, float mul2, bf16_t* __restrict__ row, int g, bool on) {
#pragma unroll
    for (int dt = 0; dt < HD / 32; ++dt)
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            uint32_t x[2][2];                           // [8-feature group][two packed pairs]
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                bf16x4_t v;
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] = (bf16_t)(acc[dt][8 * q + 4 * i + j] * (dt < HD / 64 ? mul : mul2));
                __builtin_memcpy(x[i], &v, 8);
            }
            const auto a = __builtin_amdgcn_permlane32_swap(x[0][0], x[1][0], false, false);
            const auto b = __builtin_amdgcn_permlane32_swap(x[0][1], x[1][1], false, false);
            if (on) *reinterpret_cast<uint4*>(row + dt * 32 + q * 16 + g * 8) = make_uint4(a[0], b[0], a[1], b[1]);
        }
}

// f(head size, causal, wavefronts that share a block of queries) with the template arguments of a call
//
// Sharing (KeySplit) pays where there is about one work-group for a compute unit or less, and costs where others would hide the transfers anyway:
// its ring takes twice the LDS.  It pays from about 320 keys on, which a causal sequence of 64 does not have.  One wavefront to a block of queries ->
// sharing, forward, 16 heads of 64 / of 128, us a call (keys not split, with a list on both sides):
//     1 sequence,   1 query,   4096 keys:  79 ->  55 / 108 ->  83      16 sequences, 33 queries, 1019 keys:  28 -> 26 / 37 -> 37
//     4 sequences,  1 query,   2048 keys:  44 ->  36 /  59 ->  50      16 sequences, 20 queries, 1019 keys:  26 -> 26 / 35 -> 38
//    64 sequences, 33 queries,  500 keys:  36 ->  38 /  61 ->  82     200 sequences, 20 queries,  300 keys:  52 -> 78 / 122 -> 208
// and without a list on either, keys split where there are enough: 1 sequence, 1 query, 256 keys 7.8 -> 8.0 / 10.2 -> 11.5, 300 keys 9.3 -> 9.7 / 12.0 -> 12.4,
// 512 keys 12 -> 9.5 / 16 -> 12.2
inline int sharing(const DiffAttnArgs& a) {
    const bool few = (long long)a.n_seq * a.n_heads * a.head_dim <= 64LL * kDiffUnits;
    if (a.mask || !few || a.max_k_len <= 320 || a.max_q_len > 64) return 1;
    return a.max_q_len <= 32 ? 4 : 2;
}
template <class F> ds_status diff_by_kind(const DiffAttnArgs& a, F f) {
    auto by_mask = [&](auto hd) {
        if (a.mask) return f(hd, std::true_type{}, std::integral_constant<int, 1>{});
        const int ks = sharing(a);
        if (ks == 1) return f(hd, std::false_type{}, std::integral_constant<int, 1>{});
        if (ks == 4) return f(hd, std::false_type{}, std::integral_constant<int, 4>{});
        return f(hd, std::false_type{}, std::integral_constant<int, 2>{});
    };
    return a.head_dim == 128 ? by_mask(std::integral_constant<int, 128>{}) : by_mask(std::integral_constant<int, 64>{});
}

}  // namespace
