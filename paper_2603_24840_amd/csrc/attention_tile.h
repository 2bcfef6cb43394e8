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
typedef const __attribute__((address_space(3))) bf16x8* lds_bf16x8_t;
typedef const __attribute__((address_space(3))) f32x4* lds_f32x4_t;

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
    // Fragments are read at `base` (an LDS address; what a lane adds to a tile's, plus the tile's, a multiple of 256) with the K16 step or the block of
    // 32 head elements exclusive-ored in and everything else as the instruction's own offset: one address register each for the two ways.
    // By row: A fragment for a product over the head, lane = row, K16 step s.
    __device__ static __forceinline__ unsigned row_base(int lane) {
        const int row = lane & 31;
        return row * kRowBytes + (((lane >> 5) ^ swizzle(row)) << 4);
    }
    __device__ static __forceinline__ bf16x8 by_row(unsigned base, int s, int offset) {
        return *(lds_bf16x8_t)static_cast<uintptr_t>((base ^ (s << 5)) + offset);
    }
    // By column: A fragment for a product over the tile's rows 16 s .. 16 s + 15, head elements 32 d .. 32 d + 31.  The transposing read gives lane j
    // of a block of 16 the four rows' values of head element j, lane 4 e + q holding the address of row e, elements 4 q .. 4 q + 3.  (Eight rows on,
    // bit 1 of the swizzle changes; sixteen on, none.)
    __device__ static __forceinline__ unsigned column_base(int lane) {
        const int row = 4 * (lane >> 5) + ((lane >> 2) & 3), chunk = 2 * ((lane >> 4) & 1) + ((lane >> 1) & 1);
        return row * kRowBytes + ((chunk ^ swizzle(row)) << 4) + (lane & 1) * 8;
    }
    __device__ static __forceinline__ bf16x8 by_column(unsigned base, int s, int d, int offset) {
        const unsigned at = base ^ (d << 6);
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t)static_cast<uintptr_t>(at + (16 * s * kRowBytes + offset)));
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t)static_cast<uintptr_t>((at ^ 32) + ((16 * s + 8) * kRowBytes + offset)));
        return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
};

// The same value, of which the compiler knows nothing: what is computed from it in a loop is not kept in registers over the loop.
__device__ __forceinline__ unsigned fresh(unsigned v) {
    asm volatile("" : "+v"(v));
    return v;
}

// In a branch that is seldom taken: keeps it one (the compiler would do its selects always, 64 instructions a tile).
__device__ __forceinline__ void stay_branch() { asm volatile(""); }

// ROWS rows on their way from memory straight into the LDS (16 bytes a lane, no registers): an instruction fills 1,024 bytes of the tile in order, so
// the lane that fills a position fetches the chunk that belongs there.  Rows past `valid` (>= 1) are the last valid row once more: what is made of them is masked, or
// multiplied by zeros of the other operand, or not stored, and it is never more than that row's own NaN that goes along.  Chunks past the head
// stay what they are, the zeros of clear_tiles: the other operand is 0 there, and 0 times an infinity of the head would be NaN in its products.
// Addresses are a scalar base and 32-bit offsets in the lanes.
template <int HD, int ROWS, int WAVES>
struct Stream {
    static constexpr int kPer = ROWS * Tile<HD>::kRowBytes / 1024 / WAVES;      // instructions of a wavefront
    static_assert(kPer * 1024 * WAVES == ROWS * Tile<HD>::kRowBytes, "whole instructions");
    static constexpr unsigned kNothing = ~0u;
    unsigned offset[kPer];
    __device__ __forceinline__ void point(unsigned stride_bytes, int valid, int hd, int wave, int lane) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int r = (wave * kPer + i) * (64 / Tile<HD>::kChunks) + lane / Tile<HD>::kChunks;
            const int c = (lane % Tile<HD>::kChunks) ^ Tile<HD>::swizzle(r);
            offset[i] = 8 * c < hd ? static_cast<unsigned>(r < valid ? r : valid - 1) * stride_bytes + static_cast<unsigned>(c) * 16 : kNothing;
        }
    }
    __device__ __forceinline__ void issue(const uint16_t* base, unsigned lds, int hd, int wave) const {
        if (hd == HD) {
#pragma unroll
            for (int i = 0; i < kPer; ++i) load(base, lds, i, wave);
        } else {
#pragma unroll
            for (int i = 0; i < kPer; ++i)
                if (offset[i] != kNothing) load(base, lds, i, wave);
        }
    }

private:
    __device__ __forceinline__ void load(const uint16_t* base, unsigned lds, int i, int wave) const {
        const unsigned to = lds + (wave * kPer + i) * 1024;
        asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(offset[i]), "s"(base), "s"(to) : "memory");
    }
};
// Zeros where no load will write: before the first load of a head shorter than the tile's rows.
template <int HD>
__device__ __forceinline__ void clear_tiles(unsigned char* lds, int bytes, int hd) {
    if (hd == HD) return;
    for (int i = threadIdx.x * 16; i < bytes; i += blockDim.x * 16) *reinterpret_cast<u32x4*>(lds + i) = u32x4{0, 0, 0, 0};
    __syncthreads();
}

__device__ __forceinline__ unsigned lds_address(const void* p) {
    return static_cast<unsigned>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) const unsigned char*)p));
}
template <class T>
__device__ __forceinline__ T* uniform(T* p) {       // the same pointer in every lane, in scalar registers
    const uint64_t u = reinterpret_cast<uint64_t>(p);
    const uint32_t lo = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(u)), hi = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(u >> 32));
    return reinterpret_cast<T*>(static_cast<uint64_t>(hi) << 32 | lo);
}
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
// Waits for this wavefront's loads into the LDS and its reads of it, then for the workgroup.
__device__ __forceinline__ void tiles_ready() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

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

// Own rows' results: lane l has elements 32 d + 8 b + 4 (l / 32) + r of row l % 32.  They go through `tile`, 32 rows of the LDS that are the
// wavefront's own by now, so that a store instruction writes whole rows: 8 bytes a lane, 32 rows apart, straight from the registers took 14 of 84 us on 64
// prompts of up to 512 tokens.
template <int HD>
__device__ __forceinline__ void store_own(const f32x16 (&acc)[HD / 32], float factor, unsigned char* tile, uint16_t* base, int64_t stride, int valid, int hd, int lane) {
    using T = Tile<HD>;
    typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
    const int mine = lane & 31;
    wave_lds_exchange();
#pragma unroll
    for (int d = 0; d < HD / 32; ++d)
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            const f32x4 v = {acc[d][4 * b] * factor, acc[d][4 * b + 1] * factor, acc[d][4 * b + 2] * factor, acc[d][4 * b + 3] * factor};
            *reinterpret_cast<bf16x4*>(tile + mine * T::kRowBytes + (((4 * d + b) ^ T::swizzle(mine)) << 4) + (lane >> 5) * 8) = __builtin_convertvector(v, bf16x4);
        }
    wave_lds_exchange();
    const int c = lane % T::kChunks;
#pragma unroll
    for (int i = 0; i < T::kChunks / 2; ++i) {
        const int row = i * (64 / T::kChunks) + lane / T::kChunks;
        const u32x4 x = *reinterpret_cast<const u32x4*>(tile + row * T::kRowBytes + ((c ^ T::swizzle(row)) << 4));
        if (row < valid && c * 8 < hd) *reinterpret_cast<u32x4*>(base + row * stride + c * 8) = x;
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

// Tiles of ROWS rows, none across two segments: segment s has the tiles from bound(s) / ROWS + s on, which leaves it at least as
// many as it needs whatever the lengths, and at most one spare.  So the grid is T / ROWS + n + 2 without a look at the offsets, and a workgroup finds
// its segment by a search that 64 lanes do together, two offsets each: one round for up to 126 sequences, two for 8,000, and the segment's own bounds
// come out of the last one (a chain of four loads, one for each question, was 2 us of a short workgroup's 8).  Offsets out of order give empty
// or misplaced tiles, all within [0, T).
__device__ __forceinline__ int64_t lane_value(int64_t lo64, int64_t hi64, int index) {      // of 128 values, two a lane
    const int64_t low = wave_bcast(lo64, index & 63), high = wave_bcast(hi64, index & 63);
    return index < 64 ? low : high;
}
template <unsigned ROWS, class Bound>
__device__ __forceinline__ bool find_tile(const Bound& bound, int segments, int64_t tile, int lane, int& segment, int64_t& first, int64_t& begin, int64_t& end) {
    const auto start_of = [&](int64_t b, int s) { return static_cast<int64_t>(static_cast<uint64_t>(b) / ROWS) + s; };
    int lo = 0, count = segments;
    for (;;) {
        const int step = (count + 127) >> 7, at0 = lane * step, at1 = (lane + 64) * step;
        const int64_t b0 = bound(lo + at0), b1 = bound(lo + at1);
        const uint64_t v0 = __ballot(at0 < count && start_of(b0, lo + at0) <= tile), v1 = __ballot(at1 < count && start_of(b1, lo + at1) <= tile);
        int k = v0 != ~0ull ? __builtin_ctzll(~v0) - 1 : v1 != ~0ull ? 63 + __builtin_ctzll(~v1) : 127;
        k = uniform(k < 0 ? 0 : k);
        if (step == 1) {
            segment = lo + k;
            begin = lane_value(b0, b1, k);
            end = k < 127 ? lane_value(b0, b1, k + 1) : bound(segment + 1);
            break;
        }
        lo += k * step;
        count = count - k * step < step ? count - k * step : step;
    }
    const int64_t start = start_of(begin, segment);
    first = begin + (tile - start) * ROWS;
    return tile >= start && first < end;
}
template <unsigned ROWS>
__device__ __forceinline__ bool find_tile(const Packed& p, int64_t tile, int lane, int& segment, int64_t& first, int64_t& begin, int64_t& end) {
    return find_tile<ROWS>([&](int s) { return p.bound(s); }, p.n + 2, tile, lane, segment, first, begin, end);
}
__host__ __device__ inline int64_t tile_bound(int64_t T, int n, int rows) { return T / rows + n + 2; }

}  // namespace attention
