// Pieces that the attention kernels share (gfx950, wave64): tiles of bf16 rows in the LDS, the two ways a fragment is read from
// them, and where a workgroup's rows lie among packed sequences.
//
// Every product of these kernels is v_mfma_f32_32x32x16_bf16 with a streamed tile as A (from the LDS) and the wavefront's own 32
// rows as B (in registers).  In the result lane l has column l % 32, i.e. one of the own rows, and of the 32 A rows those with
// 8 b + 4 (l / 32) + r (b, r < 4): what belongs to one own row lies in one lane and its partner l ^ 32, so row statistics need one
// exchange.  That result, rounded to bf16, is also the B fragment of the next product, whose K extent is the streamed rows: lane half h
// has its 8 values of a K16 step as rows 16 s + 4 h + {0..3} and 16 s + 8 + 4 h + {0..3}, and the A fragment is read in the same
// order (a sum does not care), so no value changes lanes in between.
#pragma once
#include "common.h"

namespace attention {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) s16x4* lds_s16x4_t;

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

__device__ __forceinline__ f32x16 mfma32(bf16x8 a, bf16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }

// A tile of rows of HD bf16 in the LDS (HD = 64 or 128; shorter heads are padded with zeros).  16-byte chunk c of row r lies at chunk
// c ^ swizzle(r) of its row.  A 128-bit read serves together the 16 lanes that share lane bit 5 and the parity of lane bits 2 to 4, a
// 64-bit one 32 lanes; 256 bytes hold the banks once.  Read by rows (lane = row), 16 such rows have 16 different positions; read
// transposed, the 4 rows x 64 bytes of a half-wavefront fall on 4 different quarters of the banks.
template <int HD>
struct Tile {
    static constexpr int kRowBytes = 2 * HD, kChunks = HD / 8;
    __device__ static __forceinline__ int swizzle(int r) {
        if constexpr (HD == 128) return ((r & 3) << 2) | ((r >> 2) & 3);
        else return ((r & 2) << 1) | ((r >> 2) & 3);     // odd rows lie 128 bytes on by themselves
    }
    __device__ static __forceinline__ int at(int r, int c) { return r * kRowBytes + ((c ^ swizzle(r)) << 4); }
    // A fragment for a product over the head: row `row`, K16 step s
    __device__ static __forceinline__ bf16x8 by_row(const unsigned char* tile, int row, int s, int half) {
        return *reinterpret_cast<const bf16x8*>(tile + at(row, 2 * s + half));
    }
    // A fragment for a product over the tile's rows 16 s .. 16 s + 15, head elements 32 d .. 32 d + 31: the transposing read gives lane j
    // of a block of 16 the four rows' values of head element j, lane 4 e + q holding the address of row e, elements 4 q .. 4 q + 3
    __device__ static __forceinline__ bf16x8 by_column(const unsigned char* tile, int s, int d, int lane) {
        const int row = 16 * s + 4 * (lane >> 5) + ((lane >> 2) & 3);
        const int chunk = 4 * d + 2 * ((lane >> 4) & 1) + ((lane >> 1) & 1), within = (lane & 1) * 8;
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t)(tile + at(row, chunk) + within));
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t)(tile + at(row + 8, chunk) + within));
        typedef short s16x8 __attribute__((ext_vector_type(8)));
        const s16x8 v = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        return __builtin_bit_cast(bf16x8, v);
    }
};

// ROWS rows on their way from memory to the LDS through registers: rows past `valid` and head elements past hd become zeros,
// whatever lies there (another sequence's rows, or nothing that may be read).
template <int HD, int ROWS, int THREADS>
struct Staged {
    static constexpr int kPer = ROWS * Tile<HD>::kChunks / THREADS;
    static_assert(kPer * THREADS == ROWS * Tile<HD>::kChunks, "whole rounds");
    u32x4 x[kPer];
    __device__ __forceinline__ void load(const uint16_t* base, int64_t stride, int valid, int hd) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int id = threadIdx.x + i * THREADS, row = id / Tile<HD>::kChunks, c = id % Tile<HD>::kChunks;
            u32x4 v = {0, 0, 0, 0};
            if (row < valid && c * 8 < hd) v = *reinterpret_cast<const u32x4*>(base + row * stride + c * 8);
            x[i] = v;
        }
    }
    __device__ __forceinline__ void store(unsigned char* tile) const {
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int id = threadIdx.x + i * THREADS;
            *reinterpret_cast<u32x4*>(tile + Tile<HD>::at(id / Tile<HD>::kChunks, id % Tile<HD>::kChunks)) = x[i];
        }
    }
};

// B fragments of the wavefront's own 32 rows (lane = row), zeros past `valid` and hd.
template <int HD>
__device__ __forceinline__ void load_own(bf16x8 (&f)[HD / 16], const uint16_t* base, int64_t stride, int valid, int hd, int lane) {
    const int row = lane & 31;
#pragma unroll
    for (int s = 0; s < HD / 16; ++s) {
        const int e = 16 * s + 8 * (lane >> 5);
        u32x4 v = {0, 0, 0, 0};
        if (row < valid && e < hd) v = *reinterpret_cast<const u32x4*>(base + row * stride + e);
        f[s] = __builtin_bit_cast(bf16x8, v);
    }
}

// Own rows' results: lane l has elements 32 d + 8 b + 4 (l / 32) + r of row l % 32.
template <int HD>
__device__ __forceinline__ void store_own(const f32x16 (&acc)[HD / 32], float factor, uint16_t* base, int64_t stride, int valid, int hd, int lane) {
    const int row = lane & 31;
    if (row >= valid) return;
#pragma unroll
    for (int d = 0; d < HD / 32; ++d)
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            const int e = 32 * d + 8 * b + 4 * (lane >> 5);
            if (e < hd) {
                typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
                const f32x4 v = {acc[d][4 * b] * factor, acc[d][4 * b + 1] * factor, acc[d][4 * b + 2] * factor, acc[d][4 * b + 3] * factor};
                *reinterpret_cast<bf16x4*>(base + row * stride + e) = __builtin_convertvector(v, bf16x4);
            }
        }
}

// 16 rows' worth of a 32 x 32 result (registers 8 s .. 8 s + 7) as the B fragment of K16 step s.
__device__ __forceinline__ bf16x8 as_fragment(const f32x16& x, int s) {
    typedef float f32x8 __attribute__((ext_vector_type(8)));
    f32x8 v;
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = x[8 * s + j];
    return __builtin_convertvector(v, bf16x8);
}

__device__ __forceinline__ float half_max(float v) {     // over lane and lane ^ 32
    const wave_pair32 p = wave_pair_u32<32>(__float_as_uint(v));
    return fmaxf(__uint_as_float(p.a), __uint_as_float(p.b));
}
__device__ __forceinline__ float half_sum(float v) {
    const wave_pair32 p = wave_pair_u32<32>(__float_as_uint(v));
    return __uint_as_float(p.a) + __uint_as_float(p.b);
}

// Packed sequences: offsets clamped into [0, T].  Segment 0 is what lies before the first sequence, segments 1 .. n are the
// sequences, n + 1 what lies behind the last.  Segment s begins at bound(s).
struct Packed {
    const int64_t* cu;
    int64_t T;
    int n;
    __device__ __forceinline__ int64_t bound(int s) const {
        if (s <= 0) return 0;
        if (s > n + 1) return T;
        const int64_t c = cu[s - 1];
        return c < 0 ? 0 : c < T ? c : T;
    }
};

// Tiles of `rows` rows, none across two segments: segment s has the tiles from bound(s) / rows + s on, which leaves it at least as
// many as it needs whatever the lengths, and at most one spare.  So the grid is T / rows + n + 2 without a look at the offsets, and a workgroup finds
// its segment by a search that 64 lanes do together (two rounds for 4,096 sequences).  Offsets out of order give empty or misplaced tiles, all
// within [0, T).
template <unsigned ROWS, class Bound>
__device__ __forceinline__ bool find_tile(const Bound& bound, int segments, int64_t tile, int lane, int& segment, int64_t& first, int64_t& end) {
    const auto start_of = [&](int s) { return static_cast<int64_t>(static_cast<uint64_t>(bound(s)) / ROWS) + s; };
    int lo = 0, count = segments;
    while (count > 1) {
        const int step = (count + 63) >> 6, at = lane * step;
        const bool before = at < count && start_of(lo + at) <= tile;
        const uint64_t votes = __ballot(before);
        const int k = votes == ~0ull ? 63 : __builtin_ctzll(~votes) - 1;
        const int skip = (k < 0 ? 0 : k) * step;
        lo += skip;
        count = count - skip < step ? count - skip : step;
    }
    segment = __builtin_amdgcn_readfirstlane(lo);
    const int64_t start = start_of(segment);
    end = bound(segment + 1);
    first = bound(segment) + (tile - start) * ROWS;
    return tile >= start && first < end;
}
template <unsigned ROWS>
__device__ __forceinline__ bool find_tile(const Packed& p, int64_t tile, int lane, int& segment, int64_t& first, int64_t& end) {
    return find_tile<ROWS>([&](int s) { return p.bound(s); }, p.n + 2, tile, lane, segment, first, end);
}
inline int64_t tile_bound(int64_t T, int n, int rows) { return T / rows + n + 2; }

}  // namespace attention
