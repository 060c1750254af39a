// What the bf16 matrix-core attention kernels share: tiles of 64 token rows in LDS (loaders, swizzle, transpose reads), fragments out of
// accumulators, and the work items of persistent work-groups.  attention_mfma.hip says how they are used.
#pragma once
#include "attention.hpp"
#include "gemm.hpp"

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
// sched_barrier mask: vector ALU, scalar ALU and transcendental instructions may cross, LDS accesses and MFMAs may not
constexpr int kFence = 0x2 | 0x4 | 0x400;
// how many fragment reads (forward) / pairs of reads (dQ) run in front of the MFMAs that use them
constexpr int FWD_AHEAD = 4, PV_AHEAD = 4, DQ_AHEAD = 2;

typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef short s16x8_t __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) s16x4_t* lds_s16x4_ptr;

// LDS swizzle: the 16-byte chunk index of a row is XORed with swz(row).  Row-wise fragment reads
// (16 lanes = 16 consecutive rows, same chunk) need the 16 rows in 16 different 16-byte units of a
// 256-byte window; transpose reads (32 lanes = 4 consecutive rows x 64 bytes) need the 4 rows in 4
// different 64-byte units.  Both hold for these bijections of the low row bits.
template <int HD> __device__ __forceinline__ int swz(int row) {
    return HD == 128 ? (((row & 3) << 2) | ((row >> 2) & 3)) : ((((row >> 1) & 1) << 2) | ((row >> 2) & 3));
}
template <int HD> __device__ __forceinline__ int off_rows(int row, int chunk) {      // [row][HD] tile, 16-byte chunk
    return row * (HD * 2) + ((chunk ^ swz<HD>(row)) << 4);
}

// max of three through v_max3_f32 directly: fmaxf() makes the compiler canonicalise every operand first (one extra
// multiply per score), which the hardware instruction does not need
__device__ __forceinline__ float max3f(float a, float b, float c) {
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}

// {hi, lo} bf16 pair with hi + lo = v to ~2^-17 relative, packed into one dword
__device__ __forceinline__ uint32_t split_hi_lo(float v) {
    const bf16_t hi = (bf16_t)v;
    const bf16_t lo = (bf16_t)(v - (float)hi);
    return (uint32_t)__builtin_bit_cast(unsigned short, hi) | ((uint32_t)__builtin_bit_cast(unsigned short, lo) << 16);
}

// accumulator registers 8u..8u+7 of a 32x32 tile -> one bf16 B fragment
__device__ __forceinline__ bf16x8_t frag_from_acc(const f32x16_t& a, int u) {
    bf16x8_t f;
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = (bf16_t)a[8 * u + j];
    return f;
}

// Per-lane byte offsets of the transposed A fragments of a token-major tile: fragment (t, dt) lists,
// for feature dt*32 + lane%32, the tokens 16t + 4g + {0..3} (low read) and 16t + 8 + 4g + {0..3} (high read).
template <int HD> struct TrOffsets {
    int lo[HD / 32], hi[HD / 32];
    __device__ __forceinline__ void init(int lane) {
        const int i = lane & 15, halfd = (lane >> 4) & 1, g = lane >> 5;
        const int r_lo = 4 * g + (i >> 2), r_hi = r_lo + 8;
        const int c2 = halfd * 2 + ((i >> 1) & 1), byte = (i & 1) * 8;
#pragma unroll
        for (int dt = 0; dt < HD / 32; ++dt) {
            lo[dt] = off_rows<HD>(r_lo, dt * 4 + c2) + byte;
            hi[dt] = off_rows<HD>(r_hi, dt * 4 + c2) + byte;
        }
    }
};
template <int HD>
__device__ __forceinline__ bf16x8_t read_tr(const char* tile, const TrOffsets<HD>& o, int t, int dt) {
    const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_ptr)(tile + t * (16 * HD * 2) + o.lo[dt]));
    const s16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_ptr)(tile + t * (16 * HD * 2) + o.hi[dt]));
    const s16x8_t v = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    return __builtin_bit_cast(bf16x8_t, v);
}

// Direct-to-LDS loader of 64-row tiles of one row-major tensor: each wavefront issues HD/32 transfers of
// 64 x 16 bytes per tile.  A transfer is addressed as a wavefront-uniform base (tensor + first row of the tile,
// scalar arithmetic) plus a 32-bit byte offset per lane; the offsets of a tile whose 64 rows all exist are fixed
// for the whole kernel, so stepping along the sequence costs no vector instruction.  Only the ragged last tile
// recomputes them (rows past the end are clamped to the last valid row; the consumers mask the duplicates).
template <int HD> struct TileLoader {
    static constexpr int PW = HD / 32;
    const char* base;
    long long ld2;                                      // row stride in bytes (64 rows of it fit in 31 bits)
    int n_valid, wave, lane;
    uint32_t off_full[PW];
    uint32_t off_group[PW];                             // the same offsets as lds_dma16_group wants them
    __device__ __forceinline__ static int row_of(int u) { return HD == 128 ? (u >> 4) : (u >> 3); }
    __device__ __forceinline__ static int chunk_of(int u) {
        return (HD == 128 ? (u & 15) : (u & 7)) ^ swz<HD>(row_of(u));
    }
    __device__ __forceinline__ void setup(const bf16_t* base_, long long ld_, int n_valid_, int wave_, int lane_) {
        base = (const char*)base_; ld2 = ld_ * 2; n_valid = n_valid_; wave = wave_; lane = lane_;
#pragma unroll
        for (int i = 0; i < PW; ++i) {
            const int u = (wave * PW + i) * 64 + lane;
            off_full[i] = (uint32_t)(row_of(u) * (int)ld2 + chunk_of(u) * 16);
            off_group[i] = dma_lane_offset<PW>(off_full[i], i);
        }
    }
    // rows r0 .. r0+63 -> the tile at LDS address lds_tile; 0 <= r0 < n_valid.  A tile whose 64 rows all exist goes as
    // one group of PW transfers under a single M0 with the fixed offsets; the ragged last tile clamps its rows.
    __device__ __forceinline__ void issue(uint32_t lds_tile, int r0) const {
        const char* b = base + (long long)r0 * ld2;
        if (r0 + 64 <= n_valid) {
            lds_dma16_group<PW>(dma_group_base<PW>(b), off_group, lds_tile + wave * (PW * 1024));
        } else {
            const int last = n_valid - 1 - r0;
            uint32_t off[PW];
#pragma unroll
            for (int i = 0; i < PW; ++i) {
                const int u = (wave * PW + i) * 64 + lane;
                const int rr = min(row_of(u), last);
                off[i] = dma_lane_offset<PW>((uint32_t)(rr * (int)ld2 + chunk_of(u) * 16), i);
            }
            lds_dma16_group<PW>(dma_group_base<PW>(b), off, lds_tile + wave * (PW * 1024));
        }
    }
};

// Loader of 64-row tiles through a raw buffer whose length ends at the last valid row: rows past the end arrive as zeros,
// so that every tile, ragged or not, is fetched by the same instructions with the same per-lane offsets.
template <int HD> struct BufferTileLoader {
    static constexpr int PW = HD / 32;
    const char* base;
    long long ld2;
    int n_valid, wave;
    uint32_t off[PW];
    __device__ __forceinline__ void setup(const bf16_t* base_, long long ld_, int n_valid_, int wave_, int lane) {
        base = (const char*)base_; ld2 = ld_ * 2; n_valid = n_valid_; wave = wave_;
#pragma unroll
        for (int i = 0; i < PW; ++i) {
            const int u = (wave * PW + i) * 64 + lane;
            off[i] = dma_lane_offset<PW>((uint32_t)(TileLoader<HD>::row_of(u) * (int)ld2 + TileLoader<HD>::chunk_of(u) * 16), i);
        }
    }
    // rows r0 .. r0+63 -> the tile at LDS address lds_tile; 0 <= r0 < n_valid
    __device__ __forceinline__ void issue(uint32_t lds_tile, int r0) const {
        const uint32_t bytes = (uint32_t)min(64, n_valid - r0) * (uint32_t)ld2;
        const i32x4_t buf = make_raw_buffer(base + (long long)r0 * ld2 - 1024 * (PW - 1), bytes + 1024u * (PW - 1));
        lds_dma16_buffer_group<PW>(buf, off, lds_tile + wave * (PW * 1024));
    }
};

// this wavefront's direct loads have landed, then everybody's; the stage read in the previous step is free
__device__ __forceinline__ void wait_tiles_and_sync() {
    __builtin_amdgcn_s_waitcnt(0x0F70);     // vmcnt(0)
    __builtin_amdgcn_s_barrier();
}

// store a transposed [HD x 32] accumulator block: lane column = row `row` of the output, 4 consecutive d per group
template <int HD>
__device__ __forceinline__ void store_cols(const f32x16_t (&acc)[HD / 32], float mul, bf16_t* __restrict__ out_row, int g) {
#pragma unroll
    for (int dt = 0; dt < HD / 32; ++dt)
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4) {
            bf16x4_t v;
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = (bf16_t)(acc[dt][4 * q4 + j] * mul);
            *reinterpret_cast<bf16x4_t*>(out_row + dt * 32 + 8 * q4 + 4 * g) = v;
        }
}

// the scratch starts with the two list lengths; from this int on, 16 for the draw counters (see lists_bytes)
constexpr int kCtrHeader = 16;

// Items of a persistent kernel.  The (item, head) pairs of the list, heads fastest, are dealt to the XCDs in turn as a plain
// grid would be, so that the blocks of one (sequence, head) stay on one XCD; a work-group starts with pair
// blockIdx.x and draws further ones of its XCD from a counter.  Counters: 8 per-XCD draws and the number of finished
// work-groups, in the scratch header (the list kernel clears them, the last work-group of a launch leaves them cleared;
// calls that share a scratch do not overlap).  The grid is a multiple of 8.
struct WorkDraw {
    int32_t* ctr;
    int total, xcd, k;
    __device__ __forceinline__ WorkDraw(const AttnArgs& a, int list) {       // list: 0 the query side, 1 the key side
        ctr = const_cast<int32_t*>(a.n_items) + kCtrHeader;
        total = a.n_items[list] * a.n_heads;
        xcd = blockIdx.x & 7;
        k = blockIdx.x >> 3;
    }
    __device__ __forceinline__ int index() const { return 8 * k + xcd; }
    __device__ __forceinline__ bool valid() const { return index() < total; }
    // thread 0 draws; the other threads' result is meaningless
    __device__ __forceinline__ int take() const {
        int next = 0;
        if (threadIdx.x == 0)
            next = ((int)gridDim.x >> 3) + __hip_atomic_fetch_add(ctr + xcd, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        return next;
    }
    __device__ __forceinline__ void advance(int next) { k = next; }
    __device__ __forceinline__ void finish() const {
        if (threadIdx.x != 0) return;
        if (__hip_atomic_fetch_add(ctr + 8, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (int)gridDim.x - 1) {
#pragma unroll
            for (int i = 0; i < 9; ++i) ctr[i] = 0;
        }
    }
};

template <class Kern>
ds_status set_smem(Kern kern, int bytes, bool& done) {
    if (!done) {
        DS_HIP_CHECK(hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, bytes));
        done = true;
    }
    return DS_OK;
}

// work-groups of a persistent kernel, one to a compute unit: no more than there are items, a multiple of 8
unsigned persistent_grid(unsigned items) {
    const unsigned n_cu = (unsigned)gemm_cu_count(), n = items < n_cu ? items : n_cu;
    return (n + 7) / 8 * 8;
}

}  // namespace
