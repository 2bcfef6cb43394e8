// Contraction of middle-sized tiles (gfx950, wave64): four wavefronts multiply BM values of A by BN values of B over a K extent,
//     acc[a][b] = sum_k A[a][k] * B[b][k]        (bf16 operands, fp32 accumulation, v_mfma_f32_16x16x32_bf16)
// with ring_nt.h's Walk and its result layout, for contractions that have too few 256 x 256 tiles to fill the chip, or too few rows to fill such tiles.
//
// K64 steps of both operands go straight to the LDS, NS stages deep.  An operand is given either row by row (K contiguous: 128 bytes of each row a step) or K-major (row k
// holds the tile's values side by side, so 64 rows of BM or BN values a step); the fragments of the latter come out through the transposing LDS read.  Where
// 16-byte chunk c lies (all free of conflicts under the serving rule that ring_nt.h states):
//   row by row, row r                 c ^ (r & 6) of 8
//   K-major, 128 values, row k        c ^ 2 ((k % 4) + 4 ((k / 8) % 2)) of 16
//   K-major, 64 values, row k         c ^ 2 ((k / 2) % 2) ^ 4 ((k / 8) % 2) of 8
// Rows, chunks and K rows past the end repeat the last ones: loads stay inside the operands.  Of K rows past the end one operand holds zeros; of the chunks past
// the end of a row (the last step of a K extent that is no multiple of 64, both operands row by row) the fragments are cleared.
//
// Bound by the LDS where the chip is full (a K64 step of 128 x 160: 72 KB of fragments at 128 bytes a cycle and 36 KB of loads at 64 are 1,150 cycles, the products 640; two workgroups
// to a compute unit), and by each step's chain of barrier, fragments and products where it is not (64 x 64: 0.2 to 0.3 us a step, however many stages the loads are ahead).
#pragma once
#include "common.h"
#include "ring_nt.h"

namespace mid_nt {

using ring_nt::bf16x8;
using ring_nt::f32x4;
using ring_nt::Walk;

template <int BM_, int BN_, int WM_, int WN_, int NS_>
struct Tile {
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, NS = NS_, NW = WM * WN, NT = NW * ARROL_WAVE;
    static constexpr int TI = BM / WM / 16, TJ = BN / WN / 16;
    static constexpr int LA = BM / 8 / NW, LB = BN / 8 / NW, LOADS = LA + LB;      // loads of a wavefront and step, 1 KiB each
    static constexpr int STAGE_BYTES = (BM + BN) * 128, LDS_BYTES = NS * STAGE_BYTES;
    static_assert((BM == 64 || BM == 128) && BN % 32 == 0 && BM % (8 * NW) == 0 && BN % (8 * NW) == 0 && NS >= 2, "tile");
    static_assert((NS - 2) * LOADS < 64, "loads that may be in flight behind a wait");
};

template <int N>
__device__ __forceinline__ void wait_vmcnt() {   // s_waitcnt vmcnt(N) only (gfx9 encoding: bits 3:0 and 15:14)
    __builtin_amdgcn_s_waitcnt(0x0F70 | (N & 15) | ((N >> 4) << 14));
}

// Row k and chunk of a lane in the u-th KiB of a K-major step of EXTENT values.
template <int EXTENT>
__device__ __forceinline__ int k_row(int u, int lane) { return EXTENT == 128 ? 4 * u + (lane >> 4) : 8 * u + (lane >> 3); }
template <int EXTENT>
__device__ __forceinline__ int k_swizzle(int k) { return EXTENT == 128 ? ((k & 3) | (((k >> 3) & 1) << 2)) << 1 : (((k >> 1) & 1) << 1) ^ (((k >> 3) & 1) << 2); }

// One operand's loads.
template <int EXTENT, int N, bool KMAJOR>
struct Stream {
    const char* base;
    unsigned voff[N], stride;
    int k[N], left;          // K-major: row of the step, and rows that exist from it on
    template <class RowOf>
    __device__ __forceinline__ void start(const char* b, unsigned s, int rows, int k_rows, int wave, int lane, RowOf row_of) {
        base = b;
        stride = s;
        left = k_rows;
#pragma unroll
        for (int q = 0; q < N; ++q) {
            const int u = wave * N + q;
            if (KMAJOR) {
                k[q] = k_row<EXTENT>(u, lane);
                const int valid = (rows < EXTENT ? rows : EXTENT) >> 3, c = (EXTENT == 128 ? lane & 15 : lane & 7) ^ k_swizzle<EXTENT>(k[q]);
                voff[q] = static_cast<unsigned>(c < valid ? c : valid - 1) * 16;
            } else {
                const int r = 8 * u + (lane >> 3);
                k[q] = 0;
                voff[q] = static_cast<unsigned>(row_of(r < rows ? r : rows - 1)) * stride + ((lane & 7) ^ (r & 6)) * 16;
            }
        }
    }
    __device__ __forceinline__ void issue(unsigned dst, int wave, unsigned back) {      // back: of a chunk past the end of its row to the last one
#pragma unroll
        for (int q = 0; q < N; ++q) {
            unsigned at = KMAJOR ? voff[q] : voff[q] - back;
            if (KMAJOR) at += static_cast<unsigned>(k[q] < left ? k[q] : left - 1) * stride;
            asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(at), "s"(base), "s"(dst + (wave * N + q) * 1024) : "memory");
        }
    }
    __device__ __forceinline__ void advance() {
        base += KMAJOR ? static_cast<int64_t>(64) * stride : 128;
        left -= 64;
    }
};

struct InOrder {
    __device__ __forceinline__ int operator()(int r) const { return r; }
};

// As ring_nt::walk, but the accumulators belong to C's tile; the LDS is not to be touched afterwards without a barrier.  tail: 16-byte chunks of a row that
// exist in the last step, 1 .. 8 (K-major operands: 8).  b_row: where row r of a B that is given row by row lies (rows of b_base, their bytes below 2^32).
template <class C, bool B_KMAJOR = false, bool A_KMAJOR = false, class RowOf = InOrder>
__device__ __forceinline__ void walk(const Walk& w, unsigned char* lds, f32x4 (&acc)[C::TI][C::TJ], int tail = 8, RowOf b_row = RowOf()) {
    constexpr int BM = C::BM, BN = C::BN, TI = C::TI, TJ = C::TJ, NS = C::NS;
    constexpr bool kTail = !A_KMAJOR && !B_KMAJOR;
    typedef __attribute__((address_space(3))) void* lds_ptr_t;
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) s16x4* lds_s16x4_t;
    const int tid = threadIdx.x, lane = tid & 63, l15 = lane & 15, lq = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave / C::WN, wn = wave % C::WN;
    const int steps = __builtin_amdgcn_readfirstlane(w.n_k64);
#pragma unroll
    for (int i = 0; i < TI; ++i)
#pragma unroll
        for (int j = 0; j < TJ; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    static_assert(!B_KMAJOR || BN == 64 || BN == 128, "swizzle");
    if (steps <= 0) return;
    Stream<BM, C::LA, A_KMAJOR> a;
    Stream<BN, C::LB, B_KMAJOR> b;
    a.start(w.a_base, w.a_stride, w.a_rows, w.a_k_rows, wave, lane, InOrder());
    b.start(w.b_base, w.b_stride, w.b_rows, w.b_k_rows, wave, lane, b_row);
    const unsigned lds0 = static_cast<unsigned>(reinterpret_cast<size_t>((lds_ptr_t)lds));
    unsigned dst = lds0;
    int issued = 0;
    const int chunk = (lane & 7) ^ ((lane >> 3) & 6);         // of every load row by row
    const unsigned past = chunk < tail ? 0 : static_cast<unsigned>(chunk - tail + 1) * 16;
    auto issue = [&]() {
        if (issued >= steps) return;
        const unsigned back = kTail && issued == steps - 1 ? past : 0;
        a.issue(dst, wave, back);
        b.issue(dst + BM * 128, wave, back);
        dst = dst == lds0 + (NS - 1) * C::STAGE_BYTES ? lds0 : dst + C::STAGE_BYTES;
        ++issued;
        a.advance();
        b.advance();
    };
    // fragments: row by row, lane -> row lane % 16, chunk lane / 16 (+ 4 for the step's second half); K-major, lane 16 lq + 4 e + q addresses row 8 lq + 4 h2 + e
    // (+ 32), values 4 q .. + 3 (block i: 16 i on, an exclusive or of the chunk)
    const int e = l15 >> 2, q = l15 & 3;
    const int pos[2] = {(lq ^ (l15 & 6)) * 16, ((lq + 4) ^ (l15 & 6)) * 16};
    const int a_off = (wm * (BM / C::WM) + l15) * 128, b_off = BM * 128 + (wn * (BN / C::WN) + l15) * 128;
    int at[2], bt[2];
#pragma unroll
    for (int h2 = 0; h2 < 2; ++h2) {
        const int k = 8 * lq + 4 * h2 + e;
        at[h2] = k * BM * 2 + (((wm * (BM / C::WM / 8) + (q >> 1)) ^ k_swizzle<BM>(k)) << 4) + (q & 1) * 8;
        bt[h2] = BM * 128 + k * BN * 2 + (((wn * (BN / C::WN / 8) + (q >> 1)) ^ k_swizzle<BN>(k)) << 4) + (q & 1) * 8;
    }
    auto down = [&](const unsigned char* base, const int (&off)[2], int h, int extent, int i) {
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t)(base + h * 64 * extent + (off[0] ^ (i << 5))));
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t)(base + h * 64 * extent + (off[1] ^ (i << 5))));
        return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    };
#pragma unroll
    for (int s = 0; s < NS - 1; ++s) issue();
    int slot = 0;
    for (int s = 0; s < steps; ++s) {
        // this step has landed (the NS - 2 after it, where there are so many, may fly), for every wavefront, and all have read the one before
        if (NS > 2 && steps - s >= NS - 1) wait_vmcnt<(NS - 2) * C::LOADS>();
        else wait_vmcnt<0>();
        __syncthreads();
        issue();
        const unsigned char* st = lds + slot;
        slot = slot == (NS - 1) * C::STAGE_BYTES ? 0 : slot + C::STAGE_BYTES;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            bf16x8 fa[TI], fb[TJ];
#pragma unroll
            for (int i = 0; i < TI; ++i) fa[i] = A_KMAJOR ? down(st, at, h, BM, i) : *reinterpret_cast<const bf16x8*>(st + a_off + i * 2048 + pos[h]);
#pragma unroll
            for (int j = 0; j < TJ; ++j) fb[j] = B_KMAJOR ? down(st, bt, h, BN, j) : *reinterpret_cast<const bf16x8*>(st + b_off + j * 2048 + pos[h]);
            if (kTail && tail < 8 && s == steps - 1 && h * 4 + lq >= tail) {
#pragma unroll
                for (int i = 0; i < TI; ++i) fa[i] = bf16x8{};
#pragma unroll
                for (int j = 0; j < TJ; ++j) fb[j] = bf16x8{};
            }
#pragma unroll
            for (int i = 0; i < TI; ++i)
#pragma unroll
                for (int j = 0; j < TJ; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fa[i], fb[j], acc[i][j], 0, 0, 0);
        }
    }
}

}  // namespace mid_nt
