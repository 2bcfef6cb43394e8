// Gradient of the per-token log-probability with respect to hidden states and LM head (gfx950, wave64).
//
//   logp_t = z_t[y_t] - lse_t,  z_t = W h_t;  with g_t = dL/dlogp_t
//   dz_tv = g_t ([v = y_t] - exp(z_tv - lse_t)),   dL/dh_t = sum_v dz_tv W_v,   dL/dW_v = sum_t dz_tv h_t
//
// Three contractions of 2 T V d flop; the logits are formed again, a piece of the vocabulary at a time, and of each piece only dz is kept, in bf16, as the operand of
// the two others.  Per piece of up to kPieceRows tokens:
//   gather     tokens that take part (g_t != 0 and a target inside the vocabulary) are counted and their hidden states put next to each other; the others' gradients are
//              zeros.  Whatever such a token's hidden state holds takes no part, and no product is spent on it
//   per piece of the vocabulary:
//   dz         tiles of W h, dz in the epilogue, stored token-major; what rounding it took at the tokens' targets is kept for the products
//   products   tiles of dL/dh (dz as it lies, W read in place down its rows) and of dL/dW (dz and the hidden states both read down their rows), in one launch, so that
//              the long walks of the first and the many short ones of the second fill the chip together.  Up to kResidentTokens tokens of a large vocabulary dL/dW keeps the hidden
//              states in registers instead
//   join       where K extents of the products are cut into parts, whose sums go to slabs: the slabs added in order
// Up to kFoundTokens tokens (and middle-sized tiles) there is no launch for the first step: every workgroup of the second finds the tokens by itself, and each copies some.
// No atomics: sums have a fixed order.
//
// What bounds it.  Large batches: the matrix cores under the card's power limit.  5,130 tokens (4,970 that take part) x 128,256 x 2048 6.6 to 6.8 ms, 1.16 to 1.19 PFLOP/s, on cards
// where torch's 16,384 x 16,384 x 8,192 product reaches 1.28 to 1.32 and its products of these three shapes 1.22, 1.19 and 1.04; 6,278 x 151,936 x 4096 18.0 to 18.7 ms, 1.21 to 1.26.
// Of the dz launches 13 % is the epilogue (2,253 us, 1,961 without, 2,145 without its stores, 2,229 without exponentials).  Few tokens: reading W twice and writing its
// gradient, 16 x 151,936 x 2048 397 us (1.87 GB: 4.7 TB/s).  Between them, 311 x 151,936 x 2048 711 us: the LDS, into which tiles of 128 x 160 bring 36 KB and out of which they read
// 72 KB a step of 640 cycles of products (matrix cores busy 40 % in the products' launch).  Small calls: three launches one after the other, 8.0, 7.5 and 2.4 us of 346 x 4,096 x 256; of its dz the
// tile's four steps are 2.2 by their measured costs, the rest the launch and finding the tokens before the first load.  Sums (lm_head_sum): read in the epilogue with nothing asked for before, 311 x 151,936 x 2048
// 1,198 us (721 in bf16, which moves 1.9 GB less), 5,130 x 128,256 x 2048 7,348 (6,937).
// Not kept: in 128 x 160 tiles the next but one step's loads before the products, with a second barrier (even), the last step peeled off (dz 258 to 363: registers), tiles of 128 x 320 and
// 256 x 320 for dz (even, and 8 % faster at 151,936 but 37 % slower at 32,000); 256 workgroups that walk over tiles, the next tile's loads under way during an epilogue (dz 1.4 % faster,
// products 3.5 % slower); the K-major offsets of the ring formed ahead (products 4.5 % slower); dL/dh with the operands' roles exchanged, bands of 4, pieces of 2^27 to 2^30 values (even).
#include "common.h"
#include "logprob_grad_plan.h"
#include "mid_nt.h"
#include "ring_nt.h"

namespace {

using namespace logprob_grad;
using ring_nt::bf16x8;
using ring_nt::f32x4;
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kXcds = 8, kRound = 256;

// The forms that the contractions come in.  BM: of the dimension that lies contiguous in the result (vocabulary of dz, columns of the gradients), BN: of its rows.
typedef ring_nt::RingTile<256, 256, 2, 4> Ring;
template <int BM, int BN, int NS> using Mid = mid_nt::Tile<BM, BN, 2, 2, NS>;
typedef Mid<128, 128, 2> Mid128;
typedef Mid<128, 160, 2> Mid160;
typedef Mid<128, 64, 3> MidFew;
typedef Mid<64, 64, 3> Mid64;
template <class C, bool B_KMAJOR, bool A_KMAJOR>
__device__ __forceinline__ void multiply(const ring_nt::Walk& w, unsigned char* lds, f32x4 (&acc)[C::TI][C::TJ], int tail = 8) {
    if constexpr (std::is_same_v<C, Ring>) ring_nt::walk<C, B_KMAJOR, A_KMAJOR>(w, lds, acc);
    else mid_nt::walk<C, B_KMAJOR, A_KMAJOR>(w, lds, acc, tail);
}

struct Grad {
    const uint16_t* W;              // of the vocabulary piece
    const uint16_t* H;              // gathered hidden states [n_active, d]
    uint16_t* dz;                   // [tokens][v_stride]
    const float *g, *lse;           // gathered
    const int32_t *target, *row;
    const int32_t* n_active;
    float* rest;                    // of dz at a token's target: what its rounding to bf16 left
    int d, v0, n_v;                 // first row of the piece, and how many
    int v_stride;                   // of dz, a multiple of 256
    // dL/dh
    float* slabs;                   // [parts][slab rows][d], NULL: straight to grad_hidden
    int64_t slab_stride;
    int k64_per_slab, add;          // add: to what the slabs hold of pieces before
    uint16_t* grad_hidden;
    int grid_h, grid_w;             // workgroups of dL/dh and of dL/dW, 0 where not wanted
    // dL/dW of the piece
    bool stream;                    // W and its gradient do not fit the caches: stored past them
    float* sum;                     // fp32 sums, read and / or written
    uint16_t* grad_w;
    int read_sum, write_sum;
    float* slabs_w;                 // [parts][piece's rows][d], NULL: no parts
    int64_t slab_w_stride;
    int k64_per_part;
    int blocks;                     // of 64 of the piece's rows that a workgroup of ResidentTiles walks over
};

// Place in a work order in which every round of 256 workgroups gives each XCD (workgroup ids congruent mod 8) 32 that follow each other.  -1: none.
__device__ __forceinline__ int place(int id, int total) {
    const int round0 = id / kRound * kRound, left = total - round0;
    const int in_round = left < kRound ? left : kRound, within = id % kRound;
    if (in_round <= 0) return -1;
    const int per_xcd = (in_round + kXcds - 1) / kXcds, p = within % kXcds * per_xcd + within / kXcds;
    return within / kXcds < per_xcd && p < in_round ? round0 + p : -1;
}
// Tile (row, col) of `rows` x `cols` at a position: bands of up to `most` rows, through which the columns run, so that neighbours share operands.
__device__ __forceinline__ void patch(int pos, int rows, int cols, int most, int& row, int& col) {
    const int bands = (rows + most - 1) / most, size = (rows + bands - 1) / bands;
    const int b = pos / (size * cols), r = pos - b * size * cols, mine = rows - b * size < size ? rows - b * size : size;
    col = __builtin_amdgcn_readfirstlane(r / mine);      // in scalar registers, as the walk wants its bases
    row = __builtin_amdgcn_readfirstlane(b * size + r - col * mine);
}

__device__ __forceinline__ bool takes_part(float g, int32_t target, int V) { return g != 0.f && target >= 0 && target < V; }      // NaN does

// Tokens that take part, packed.  A workgroup has kGatherRows tokens, a wavefront a quarter of them, and counts those before them itself.
constexpr int kGatherRows = 16;
struct Gather {
    const uint16_t* hidden;
    const int32_t* targets;
    const float *lse, *grad_logp;
    uint16_t *H, *grad_hidden;
    float *g, *lse_out;
    int32_t *target, *row, *n_active;
    int T, V, d;
};
__global__ __launch_bounds__(256) void gather_kernel(Gather a) {
    constexpr int kInFlight = 8, ROWS = kGatherRows;
    __shared__ int before[4];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), t0 = blockIdx.x * ROWS;
    const bool in = lane < ROWS && t0 + lane < a.T;
    const float g = in ? a.grad_logp[t0 + lane] : 0.f;
    const int32_t y = in ? a.targets[t0 + lane] : -1;
    int n = 0;
    for (int base = 0; base < t0; base += 256 * kInFlight) {
        float gs[kInFlight];
        int32_t ys[kInFlight];
#pragma unroll
        for (int i = 0; i < kInFlight; ++i) {
            const int t = base + i * 256 + tid;
            gs[i] = a.grad_logp[t < t0 ? t : 0];
            ys[i] = t < t0 ? a.targets[t] : -1;
        }
#pragma unroll
        for (int i = 0; i < kInFlight; ++i) n += __popcll(__ballot(takes_part(gs[i], ys[i], a.V)));
    }
    if (lane == 0) before[wave] = n;
    const uint64_t active = __ballot(takes_part(g, y, a.V));      // of the workgroup's tokens, in every wavefront
    __syncthreads();
    const int first = before[0] + before[1] + before[2] + before[3];
    if (wave == 0 && ((active >> lane) & 1)) {
        const int r = first + __popcll(active & ((uint64_t{1} << lane) - 1));
        a.g[r] = g;
        a.lse_out[r] = a.lse[t0 + lane];
        a.target[r] = y;
        a.row[r] = t0 + lane;
    }
    if (tid == 0 && t0 + ROWS >= a.T) *a.n_active = first + __popcll(active);
    const int vecs = a.d / 8;
#pragma unroll
    for (int i = 0; i < ROWS / 4; ++i) {
        const int r = wave * (ROWS / 4) + i, t = t0 + r;
        if (t >= a.T) break;
        const bool on = (active >> r) & 1;
        const uint16_t* from = a.hidden + static_cast<int64_t>(t) * a.d;
        uint16_t* to = on ? a.H + static_cast<int64_t>(first + __popcll(active & ((uint64_t{1} << r) - 1))) * a.d
                          : a.grad_hidden ? a.grad_hidden + static_cast<int64_t>(t) * a.d : nullptr;
        if (!to) continue;
        for (int c0 = lane; c0 < vecs; c0 += ARROL_WAVE * kInFlight) {
            u32x4 x[kInFlight];
#pragma unroll
            for (int k = 0; k < kInFlight; ++k) {
                const int c = c0 + k * ARROL_WAVE;
                x[k] = on && c < vecs ? *reinterpret_cast<const u32x4*>(from + c * 8) : u32x4{0, 0, 0, 0};
            }
#pragma unroll
            for (int k = 0; k < kInFlight; ++k) {
                const int c = c0 + k * ARROL_WAVE;
                if (c < vecs) *reinterpret_cast<u32x4*>(to + c * 8) = x[k];
            }
        }
    }
}

// A wavefront's results, 4 consecutive values of a row in a lane, as bf16: lanes of neighbouring quarters exchange halves of two blocks, so that each stores 16 bytes and the
// 16 lanes' rows get 64 bytes at a time.  x, y: blocks i and i + 1 of the row; the lane's 8 values start at 16 (i + lq % 2) + 4 (lq & 2).
__device__ __forceinline__ u32x4 exchange(f32x4 x, f32x4 y) {
    typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
    const u32x2 a = __builtin_bit_cast(u32x2, __builtin_convertvector(x, bf16x4)), b = __builtin_bit_cast(u32x2, __builtin_convertvector(y, bf16x4));
    const auto lo = __builtin_amdgcn_permlane16_swap(a[0], b[0], false, false), hi = __builtin_amdgcn_permlane16_swap(a[1], b[1], false, false);
    return u32x4{lo[0], hi[0], lo[1], hi[1]};
}

struct Lane {
    int lane, wave, l15, lq;
    __device__ __forceinline__ Lane() : lane(threadIdx.x & 63), wave(__builtin_amdgcn_readfirstlane(threadIdx.x >> 6)), l15(lane & 15), lq(lane >> 4) {}
    __device__ __forceinline__ int place(int i) const { return 16 * (i + (lq & 1)) + 4 * (lq & 2); }      // of exchange()'s values
};

// x, y: exchange()'s of 64 consecutive columns of the lane's row.  Lanes of rows r and r + 8 exchange halves: `first` belongs to row lane % 8 of the 16, `second` to the row
// 8 on, both at place(0), or place(2) for the upper lanes, so that a store is whole lines of eight rows.
__device__ __forceinline__ void whole_lines(const Lane& me, u32x4 x, u32x4 y, u32x4& first, u32x4& second) {
    const bool low = me.l15 < 8;
#pragma unroll
    for (int v = 0; v < 4; ++v) {
        const unsigned other = __builtin_amdgcn_update_dpp(0, low ? y[v] : x[v], 0x128, 0xf, 0xf, false);      // of lane l15 ^ 8
        first[v] = low ? x[v] : other;
        second[v] = low ? other : y[v];
    }
}

// The tokens that take part, found by a workgroup of 256 by itself, up to kFoundTokens of them: their numbers in `list`, the others' bits in `masks` clear; how many.
struct Found {
    uint64_t masks[kFoundTokens / ARROL_WAVE];
    int list[kFoundTokens];
};
__device__ __forceinline__ int find_tokens(const Gather& a, Found& found) {
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), rounds = (a.T + 255) / 256;
    float g[kFoundTokens / 256];
    int32_t y[kFoundTokens / 256];
#pragma unroll
    for (int i = 0; i < kFoundTokens / 256; ++i) {
        const int t = i * 256 + tid;
        g[i] = t < a.T ? a.grad_logp[t] : 0.f;
        y[i] = t < a.T ? a.targets[t] : -1;
    }
#pragma unroll
    for (int i = 0; i < kFoundTokens / 256; ++i) {
        const uint64_t active = __ballot(takes_part(g[i], y[i], a.V));
        if (lane == 0) found.masks[i * 4 + wave] = active;
    }
    __syncthreads();
    int n = 0;
    for (int i = 0; i < rounds; ++i) {
        int before = n;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const int count = __popcll(found.masks[i * 4 + w]);
            before += w < wave ? count : 0;
            n += count;
        }
        const uint64_t mine = found.masks[i * 4 + wave];
        if ((mine >> lane) & 1) found.list[before + __popcll(mine & ((uint64_t{1} << lane) - 1))] = i * 256 + tid;
    }
    __syncthreads();
    return __builtin_amdgcn_readfirstlane(n);
}
__device__ __forceinline__ void copy_row(const uint16_t* from, uint16_t* to, int vecs) {      // by a workgroup of 256; from NULL: zeros
    for (int c = threadIdx.x; c < vecs; c += 256)
        *reinterpret_cast<u32x4*>(to + c * 8) = from ? *reinterpret_cast<const u32x4*>(from + c * 8) : u32x4{0, 0, 0, 0};
}

// What the lane's tokens bring with them: of token 16 j + lane % 16 of the wavefront's part.  Fetched before the walk.
template <class C>
struct Tokens {
    float g[C::TJ], at[C::TJ];      // at: -lse log2 e
    int target[C::TJ];              // -1: none
    template <class RowOf>
    __device__ __forceinline__ Tokens(const float* gs, const float* lse, const int32_t* targets, const Lane& me, int tb, int n_active, RowOf row_of) {
#pragma unroll
        for (int j = 0; j < C::TJ; ++j) {
            const int t = tb * C::BN + me.wave % C::WN * (C::BN / C::WN) + j * 16 + me.l15;
            const bool live = t < n_active;
            const int r = live ? row_of(t) : 0;
            g[j] = live ? gs[r] : 0.f;
            at[j] = live ? -lse[r] * kLog2e : 0.f;
            target[j] = live ? targets[r] : -1;
        }
    }
};

// acc[i][j][v] = z of vocabulary row 16 i + 4 (lane / 16) + v and token 16 j + lane % 16 of the wavefront's part of the tile.  dz of rows past the vocabulary and of
// tokens past the last, up to a multiple of 64, are zeros: the products' K extents are whole steps of 64.
template <class C>
__device__ __forceinline__ void store_dz(const Grad& a, const Lane& me, const Tokens<C>& tokens, const f32x4 (&acc)[C::TI][C::TJ], int vt, int tb, int n_active) {
    const int v_first = vt * C::BM + me.wave / C::WN * (C::BM / C::WM), t_first = tb * C::BN + me.wave % C::WN * (C::BN / C::WN);
    const int rows = (n_active + 63) / 64 * 64;
    const bool edge = v_first + C::BM / C::WM > a.n_v || t_first + C::BN / C::WN > n_active;
#pragma unroll
    for (int j = 0; j < C::TJ; ++j) {
        if (t_first + j * 16 >= rows) break;
        const int t = t_first + j * 16 + me.l15;
        const float g = tokens.g[j], at = tokens.at[j];
        const int y = tokens.target[j] - a.v0 - v_first - 4 * me.lq;        // of this lane's rows: 16 i + v
        const bool mine = t < n_active && y >= 0 && y < C::BM / C::WM && (y & 12) == 0;
        uint16_t* to = a.dz + static_cast<int64_t>(t) * a.v_stride + v_first;
        auto plain = [&](int i) {
            f32x4 x;
#pragma unroll
            for (int v = 0; v < 4; ++v) x[v] = -g * __builtin_amdgcn_exp2f(fmaf(acc[i][j][v], kLog2e, at));
            return x;
        };
        auto whole = [&](int i) {
            f32x4 x = plain(i);
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                if (mine && y == 16 * i + v) {
                    x[v] += g;
                    const float rest = x[v] - static_cast<float>(static_cast<__bf16>(x[v]));
                    a.rest[t] = fabsf(rest) < 3e38f ? rest : 0.f;       // infinities and NaN are in dz itself
                }
                if (t >= n_active || v_first + 16 * i + 4 * me.lq + v >= a.n_v) x[v] = 0.f;
            }
            return x;
        };
        if (edge || __any(mine)) {
#pragma unroll
            for (int i = 0; i < C::TI; i += 2) *reinterpret_cast<u32x4*>(to + me.place(i)) = exchange(whole(i), whole(i + 1));
        } else {
#pragma unroll
            for (int i = 0; i < C::TI; i += 2) *reinterpret_cast<u32x4*>(to + me.place(i)) = exchange(plain(i), plain(i + 1));
        }
    }
    if constexpr (C::BN % 64 != 0) {        // the zeros of a multiple of 64 that ends behind the last tile, 32 tokens at most
        static_assert(C::BN % 64 == 32 && C::WN == 2, "tokens behind the tile");
        const int t = (tb + 1) * C::BN + me.wave % 2 * 16 + me.l15;
        if ((tb + 1) * C::BN >= n_active && t < rows)
#pragma unroll
            for (int i = 0; i < C::TI; i += 2) *reinterpret_cast<u32x4*>(a.dz + static_cast<int64_t>(t) * a.v_stride + v_first + me.place(i)) = u32x4{0, 0, 0, 0};
    }
}

// dz tile (vt, tb).
template <class C>
struct DzTiles {
    const Grad& a;
    const int n_active, n_tb, n_vt;
    __device__ __forceinline__ DzTiles(const Grad& a, int n) : a(a), n_active(n), n_tb((n + C::BN - 1) / C::BN), n_vt((a.n_v + C::BM - 1) / C::BM) {}
    __device__ __forceinline__ int total() const { return n_tb * n_vt; }
    __device__ __forceinline__ void at(int pos, int& vt, int& tb) const { patch(pos, n_tb, n_vt, 6, tb, vt); }
    __device__ __forceinline__ ring_nt::Walk walk(int vt, int tb) const {
        ring_nt::Walk w = {};
        const int64_t row = static_cast<int64_t>(a.d) * 2;
        w.a_base = reinterpret_cast<const char*>(a.W) + vt * C::BM * row;
        w.b_base = reinterpret_cast<const char*>(a.H) + tb * C::BN * row;
        w.a_stride = w.b_stride = static_cast<unsigned>(row);
        w.a_rows = a.n_v - vt * C::BM;
        w.b_rows = n_active - tb * C::BN < C::BN ? n_active - tb * C::BN : C::BN;
        w.n_k64 = (a.d + 63) / 64;
        return w;
    }
};

template <class C>
__global__ __launch_bounds__(C::NT) void dz_kernel(Grad a) {
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    const int n_active = __builtin_amdgcn_readfirstlane(*a.n_active);
    const DzTiles<C> tiles(a, n_active);
    const int pos = place(blockIdx.x, tiles.total());
    if (pos < 0) return;
    int vt, tb;
    tiles.at(pos, vt, tb);
    const Lane me;
    const Tokens<C> tokens(a.g, a.lse, a.target, me, tb, n_active, mid_nt::InOrder());
    f32x4 acc[C::TI][C::TJ];
    multiply<C, false, false>(tiles.walk(vt, tb), lds, acc, (a.d & 63) ? (a.d & 63) / 8 : 8);
    store_dz<C>(a, me, tokens, acc, vt, tb, n_active);
}

// The same where the tokens are found here.  Which they are is left behind for the products, and their hidden states, packed, if `g.H` is given.
template <class C>
__global__ __launch_bounds__(C::NT) void dz_found_kernel(Grad a, Gather g) {
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    Found& found = *reinterpret_cast<Found*>(lds + C::LDS_BYTES);
    const int n_active = find_tokens(g, found), vecs = a.d / 8;
    if (blockIdx.x == 0) {
        for (int r = threadIdx.x; r < n_active; r += 256) {
            g.row[r] = found.list[r];
            g.target[r] = g.targets[found.list[r]];
        }
        if (threadIdx.x == 0) *g.n_active = n_active;
    }
    if (g.grad_hidden && n_active < g.T)
        for (int t = blockIdx.x; t < g.T; t += gridDim.x)
            if (!((found.masks[t >> 6] >> (t & 63)) & 1)) copy_row(nullptr, g.grad_hidden + static_cast<int64_t>(t) * a.d, vecs);
    const DzTiles<C> tiles(a, n_active);
    const int pos = place(blockIdx.x, tiles.total());
    if (pos < 0) return;
    int vt, tb;
    tiles.at(pos, vt, tb);
    const int t0 = tb * C::BN;
    if (g.H)        // the tile's tokens, shared out over the vocabulary's tiles
        for (int t = t0 + vt; t < t0 + C::BN && t < n_active; t += tiles.n_vt)
            copy_row(g.hidden + static_cast<int64_t>(found.list[t]) * a.d, g.H + static_cast<int64_t>(t) * a.d, vecs);
    const Lane me;
    const Tokens<C> tokens(g.grad_logp, g.lse, g.targets, me, tb, n_active, [&](int t) { return found.list[t]; });
    f32x4 acc[C::TI][C::TJ];
    ring_nt::Walk w = tiles.walk(vt, tb);
    w.b_base = reinterpret_cast<const char*>(g.hidden);
    mid_nt::walk<C, false, false>(w, lds, acc, (a.d & 63) ? (a.d & 63) / 8 : 8, [&](int r) { return found.list[t0 + r]; });
    store_dz<C>(a, me, tokens, acc, vt, tb, n_active);
}

// The epilogue of both products: acc[i][j][v] belongs to column c0 + 16 i + 4 lq + v of row r0 + 16 j + l15.  sum: fp32, read and / or written; else bf16.
template <class C, bool PAST = false, class RowOf>
__device__ __forceinline__ void store_rows(const Lane& me, const f32x4 (&acc)[C::TI][C::TJ], int r0, int rows, int c0, int d, float* sum, bool read, bool write, uint16_t* out, RowOf row_of) {
#pragma unroll
    for (int j = 0; j < C::TJ; ++j) {
        const int r = r0 + j * 16 + me.l15;
        const bool live = r < rows;
        const int64_t line = static_cast<int64_t>(live ? r : 0) * d;
        uint16_t* to = write ? nullptr : out + static_cast<int64_t>(live ? row_of(r) : 0) * d;
        auto value = [&](int i) {
            const int c = c0 + 16 * i + 4 * me.lq;
            return read && live && c < d ? *reinterpret_cast<const f32x4*>(sum + line + c) + acc[i][j] : acc[i][j];
        };
        if constexpr (PAST && C::TI % 4 == 0) {
#pragma unroll
            for (int i = 0; i < C::TI; i += 4) {
                u32x4 first, second;
                whole_lines(me, exchange(value(i), value(i + 1)), exchange(value(i + 2), value(i + 3)), first, second);
                const int row = r0 + j * 16 + (me.l15 & 7), c = c0 + me.place(i + (me.l15 < 8 ? 0 : 2));
                if (row < rows && c < d) __builtin_nontemporal_store(first, reinterpret_cast<u32x4*>(out + static_cast<int64_t>(row_of(row)) * d + c));
                if (row + 8 < rows && c < d) __builtin_nontemporal_store(second, reinterpret_cast<u32x4*>(out + static_cast<int64_t>(row_of(row + 8)) * d + c));
            }
            continue;
        }
#pragma unroll
        for (int i = 0; i < C::TI; i += 2) {
            const f32x4 x = value(i), y = value(i + 1);
            if (write) {
                const int c = c0 + 16 * i + 4 * me.lq;
                if (live && c < d) *reinterpret_cast<f32x4*>(sum + line + c) = x;
                if (live && c + 16 < d) *reinterpret_cast<f32x4*>(sum + line + c + 16) = y;
            } else {
                const u32x4 packed = exchange(x, y);      // by all lanes
                const int c = c0 + me.place(i);
                if (live && c < d) {
                    if constexpr (PAST) __builtin_nontemporal_store(packed, reinterpret_cast<u32x4*>(to + c));
                    else *reinterpret_cast<u32x4*>(to + c) = packed;
                }
            }
        }
    }
}

__device__ __forceinline__ void add_times(f32x4& x, float f, bf16x4 four) {
    const f32x4 y = __builtin_convertvector(four, f32x4);
#pragma unroll
    for (int v = 0; v < 4; ++v) x[v] = fmaf(f, y[v], x[v]);
}

// dz is largest at a token's target by far, and that one rounding, 2^-8 at most, counts beside a result's own: in dL/dh_t, where no other token averages it out, and in the row of dL/dW
// that it is the target of, where gradients of either sign average out as little.  What dz lost there is added in fp32.  To dL/dh_t it is one row of W, a token's for itself: 5,130 x 128,256 x 2048 6,905 us and
// without 6,965, 8,777 x 4,096 x 1024 317 and 315, at worst 4,000 x 300 x 1088 39.8 and 37.8.  To dL/dW it is a hidden state for every token whose target a row is.  The resident form has
// that for nothing; tiles have to find their tokens and fetch them one after the other, so there it is up to kResidentTokens, where the forms meet, and beyond a gradient is 2.4e-3 off
// in norm instead of 1.7e-3 (up to 1,024 tokens: 640 x 32,000 x 2048 292 us and without 267, 500 x 18,920 x 3128 275 and 256, 510 x 391 x 128 25.9 and 13.2).  What an epilogue
// needs is asked for before its walk.

// dL/dh: columns of W, which is read down its rows, times tokens' rows of dz; K = the vocabulary piece or a part of it.  Tile (s, at, db): part, tokens, columns.
template <class C>
struct HiddenTiles {
    const Grad& a;
    const int n_active, n_tb, n_db, n_k64, n_parts;
    __device__ __forceinline__ HiddenTiles(const Grad& a, int n)
        : a(a), n_active(n), n_tb((n + C::BN - 1) / C::BN), n_db((a.d + C::BM - 1) / C::BM), n_k64((a.n_v + 63) / 64), n_parts((n_k64 + a.k64_per_slab - 1) / a.k64_per_slab) {}
    __device__ __forceinline__ int total() const { return a.grid_h ? n_tb * n_db * n_parts : 0; }
    __device__ __forceinline__ void at(int pos, int& s, int& tb, int& db) const {
        s = __builtin_amdgcn_readfirstlane(pos / (n_tb * n_db));
        patch(pos - s * n_tb * n_db, n_db, n_tb, 8, db, tb);
    }
    __device__ __forceinline__ ring_nt::Walk walk(int s, int tb, int db) const {
        ring_nt::Walk w = {};
        const int64_t row = static_cast<int64_t>(a.d) * 2;
        const int k_lo = s * a.k64_per_slab, k_hi = k_lo + a.k64_per_slab < n_k64 ? k_lo + a.k64_per_slab : n_k64;
        w.a_base = reinterpret_cast<const char*>(a.W) + static_cast<int64_t>(k_lo) * 64 * row + db * C::BM * 2;
        w.a_stride = static_cast<unsigned>(row);
        w.a_rows = a.d - db * C::BM;
        w.a_k_rows = a.n_v - k_lo * 64;
        w.b_base = reinterpret_cast<const char*>(a.dz + static_cast<int64_t>(tb) * C::BN * a.v_stride) + static_cast<int64_t>(k_lo) * 128;
        w.b_stride = static_cast<unsigned>(a.v_stride) * 2;
        w.b_rows = n_active - tb * C::BN < C::BN ? n_active - tb * C::BN : C::BN;
        w.n_k64 = k_hi - k_lo;
        return w;
    }
    // The rests of the piece's targets and where their rows of W are, for the first part; 0 and -1 otherwise.
    struct Rests {
        int y[C::TJ];
        float rest[C::TJ];
    };
    __device__ __forceinline__ Rests rests(const Lane& me, int s, int tb) const {
        Rests r;
        const int t_first = tb * C::BN + me.wave % C::WN * (C::BN / C::WN) + me.l15;
#pragma unroll
        for (int j = 0; j < C::TJ; ++j) {
            const int t = t_first + 16 * j;
            const bool on = s == 0 && t < n_active;
            r.y[j] = on ? a.target[t] - a.v0 : -1;
            r.rest[j] = on ? a.rest[t] : 0.f;
        }
        return r;
    }
    __device__ __forceinline__ void store(const Lane& me, const Rests& rests, f32x4 (&acc)[C::TI][C::TJ], int s, int tb, int db) const {
        const Grad& a = this->a;
        if (s == 0) {
            const int c0 = db * C::BM + me.wave / C::WN * (C::BM / C::WM) + 4 * me.lq;
            constexpr int kAtOnce = C::TI > 4 ? 1 : C::TJ % 2 ? C::TJ : 2;
#pragma unroll
            for (int j0 = 0; j0 < C::TJ; j0 += kAtOnce) {
                bf16x4 w[kAtOnce][C::TI];
#pragma unroll
                for (int k = 0; k < kAtOnce; ++k) {
                    const int y = rests.y[j0 + k];
                    const uint16_t* row = a.W + static_cast<int64_t>(y >= 0 && y < a.n_v ? y : 0) * a.d;
#pragma unroll
                    for (int i = 0; i < C::TI; ++i) w[k][i] = *reinterpret_cast<const bf16x4*>(row + (c0 + 16 * i < a.d ? c0 + 16 * i : 0));
                }
#pragma unroll
                for (int k = 0; k < kAtOnce; ++k) {
                    if (rests.y[j0 + k] < 0 || rests.y[j0 + k] >= a.n_v || rests.rest[j0 + k] == 0.f) continue;      // 0 times infinity
#pragma unroll
                    for (int i = 0; i < C::TI; ++i) add_times(acc[i][j0 + k], rests.rest[j0 + k], w[k][i]);
                }
            }
        }
        store_rows<C>(me, acc, tb * C::BN + me.wave % C::WN * (C::BN / C::WN), n_active, db * C::BM + me.wave / C::WN * (C::BM / C::WM), a.d, a.slabs + s * a.slab_stride, a.add,
                      a.slabs != nullptr, a.grad_hidden, [&](int t) { return a.row[t]; });
    }
};

// dL/dW: columns of the hidden states times the piece's rows, both read down the tokens or a part of them.  Tile (s, vt, db).
template <class C>
struct HeadTiles {
    const Grad& a;
    const int n_active, n_vt, n_db, n_k64, n_parts;
    __device__ __forceinline__ HeadTiles(const Grad& a, int n)
        : a(a), n_active(n), n_vt((a.n_v + C::BN - 1) / C::BN), n_db((a.d + C::BM - 1) / C::BM), n_k64((n + 63) / 64), n_parts(a.slabs_w ? (n_k64 + a.k64_per_part - 1) / a.k64_per_part : 1) {}
    __device__ __forceinline__ int total() const { return n_vt * n_db * n_parts; }
    __device__ __forceinline__ void at(int pos, int& s, int& vt, int& db) const {
        s = __builtin_amdgcn_readfirstlane(pos / (n_vt * n_db));
        patch(pos - s * n_vt * n_db, n_db, n_vt, 8, db, vt);
    }
    __device__ __forceinline__ ring_nt::Walk walk(int s, int vt, int db) const {
        ring_nt::Walk w = {};
        const int64_t row = static_cast<int64_t>(a.d) * 2;
        const int k_lo = a.slabs_w ? s * a.k64_per_part : 0, k_hi = a.slabs_w && k_lo + a.k64_per_part < n_k64 ? k_lo + a.k64_per_part : n_k64;
        w.a_base = reinterpret_cast<const char*>(a.H) + static_cast<int64_t>(k_lo) * 64 * row + db * C::BM * 2;
        w.a_stride = static_cast<unsigned>(row);
        w.a_rows = a.d - db * C::BM;
        w.a_k_rows = n_active - k_lo * 64;
        w.b_base = reinterpret_cast<const char*>(a.dz + static_cast<int64_t>(k_lo) * 64 * a.v_stride + static_cast<int64_t>(vt) * C::BN);
        w.b_stride = static_cast<unsigned>(a.v_stride) * 2;
        w.b_rows = C::BN;                                // v_stride is a multiple of 256, and zeros follow the piece's last row up to a multiple of 64
        w.n_k64 = k_hi - k_lo;
        w.b_k_rows = w.n_k64 * 64;                       // rows of zeros behind n_active
        return w;
    }
    // The wavefront's rows that are targets, of token lane and every 64th from it on, for the first part.
    struct Rests {
        int row[kResidentTokens / ARROL_WAVE];
    };
    __device__ __forceinline__ int first_row(const Lane& me, int vt) const { return vt * C::BN + me.wave % C::WN * (C::BN / C::WN); }
    __device__ __forceinline__ Rests rests(const Lane& me, int s, int vt) const {
        Rests r;
#pragma unroll
        for (int u = 0; u < kResidentTokens / ARROL_WAVE; ++u) {
            const int t = u * ARROL_WAVE + me.lane;
            r.row[u] = s == 0 && n_active <= kResidentTokens && t < n_active ? a.target[t] - a.v0 - first_row(me, vt) : -1;
        }
        return r;
    }
    // Their rests times the hidden states, token by token.
    __device__ __forceinline__ void add_rests(const Lane& me, const Rests& rests, f32x4 (&acc)[C::TI][C::TJ], int vt, int db) const {
        constexpr int kAtOnce = C::TI > 4 ? 2 : 4, kRows = C::BN / C::WN;
        uint64_t mine = 0;                  // of 64 tokens, lane by lane
#pragma unroll
        for (int u = 0; u < kResidentTokens / ARROL_WAVE; ++u) {
            const uint64_t mask = __ballot(rests.row[u] >= 0 && rests.row[u] < kRows);
            mine = me.lane == u ? mask : mine;
        }
        const int c0 = db * C::BM + me.wave / C::WN * (C::BM / C::WM) + 4 * me.lq, first = first_row(me, vt);
        uint64_t some = __ballot(mine != 0), tokens = 0;
        int at = 0;
        for (;;) {
            int t[kAtOnce], row[kAtOnce];
            float rest[kAtOnce];
            bf16x4 h[kAtOnce][C::TI];
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k) {
                if (!tokens && some) {
                    at = __builtin_ctzll(some);
                    some &= some - 1;
                    tokens = static_cast<uint64_t>(__builtin_amdgcn_readlane(static_cast<unsigned>(mine >> 32), at)) << 32 |
                             static_cast<unsigned>(__builtin_amdgcn_readlane(static_cast<unsigned>(mine), at));
                }
                t[k] = tokens ? at * 64 + __builtin_ctzll(tokens) : -1;
                tokens &= tokens - 1;
            }
            if (t[0] < 0) break;
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k) {
                const int from = t[k] < 0 ? 0 : t[k];
                row[k] = a.target[from];
                rest[k] = a.rest[from];
#pragma unroll
                for (int i = 0; i < C::TI; ++i) h[k][i] = *reinterpret_cast<const bf16x4*>(a.H + static_cast<int64_t>(from) * a.d + (c0 + 16 * i < a.d ? c0 + 16 * i : 0));
            }
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k) {
                if (t[k] < 0) break;
                const int r = __builtin_amdgcn_readfirstlane(row[k]) - a.v0 - first;
#pragma unroll
                for (int j = 0; j < C::TJ; ++j) {
                    if (r >> 4 != j || (r & 15) != me.l15 || rest[k] == 0.f) continue;
#pragma unroll
                    for (int i = 0; i < C::TI; ++i) add_times(acc[i][j], rest[k], h[k][i]);
                }
            }
        }
    }
    __device__ __forceinline__ void store(const Lane& me, const Rests& rests, f32x4 (&acc)[C::TI][C::TJ], int s, int vt, int db) const {
        if (s == 0 && n_active <= kResidentTokens) add_rests(me, rests, acc, vt, db);
        const int r0 = vt * C::BN + me.wave % C::WN * (C::BN / C::WN), c0 = db * C::BM + me.wave / C::WN * (C::BM / C::WM);
        const bool parts = a.slabs_w != nullptr;
        const auto same = [](int r) { return r; };
        if (a.stream && !a.write_sum) store_rows<C, true>(me, acc, r0, a.n_v, c0, a.d, a.sum, a.read_sum, false, a.grad_w, same);      // of such a size there are no parts: part_floats()
        else store_rows<C>(me, acc, r0, a.n_v, c0, a.d, parts ? a.slabs_w + s * a.slab_w_stride : a.sum, !parts && a.read_sum, parts || a.write_sum, a.grad_w, same);
    }
};

// dL/dW of up to kResidentTokens tokens.  A wavefront keeps 64 columns of the hidden states of all tokens in registers (160 of its 254) and walks down the vocabulary, 64 rows
// of dz at a time, which its workgroup of 256 columns shares: one barrier for the products of all tokens, and the next rows' loads and the last ones' stores under way meanwhile.
// The accesses of a wavefront complete in the order of their issue, so a wait for the loads counts the eight stores behind them, which come on no branch where a block is whole.
// 151,936 x 2048, this launch's dL/dW alone: 64 tokens 130 us (4.8 TB/s, bound by the stores), 192 177, 311 205 (622 MB at 3.0 TB/s and 0.94 PFLOP/s; matrix cores busy 41 %); tiles of 128 x 128
// take 190 at 64 tokens and 332 at 311.  Stores of whole lines of 128 bytes instead of halves: 64 tokens 185 to 130, 311 214 to 205.  Blocks to a workgroup, 311 tokens, both products: 4 736, 8 717, 16 722.
struct ResidentTiles {
    static constexpr int kStage = kResidentSteps * 8192, LDS_BYTES = 2 * kStage;
    struct Part {                   // for store_rows
        static constexpr int TI = 4, TJ = 2;
    };
    typedef __attribute__((address_space(3))) void* lds_ptr_t;
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) s16x4* lds_s16x4_t;

    const Grad& a;
    const int n_active, n_db, n_vb;
    __device__ __forceinline__ ResidentTiles(const Grad& a, int n) : a(a), n_active(n), n_db((a.d + 255) / 256), n_vb((a.n_v + 63) / 64) {}
    __device__ __forceinline__ int total() const { return (n_vb + a.blocks - 1) / a.blocks * n_db; }

    static __device__ __forceinline__ void load(const char* base, unsigned off, unsigned dst) {
        asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(off), "s"(base), "s"(dst) : "memory");
    }
    // Eight consecutive rows 8 (lane / 16) .. of column lane % 16 of block i, from a step of 64 rows of 128 bytes (off as in mid_nt::walk).
    static __device__ __forceinline__ bf16x8 down(const unsigned char* at, const int (&off)[2], int i) {
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t)(at + (off[0] ^ (i << 5))));
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t)(at + (off[1] ^ (i << 5))));
        return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }

    // The rests of the tokens whose targets are among the 32 rows from `first` on times their hidden states, token by token.  target: of token 64 k + lane.
    __device__ __forceinline__ void add_rests(const Lane& me, const int (&target)[kResidentSteps], f32x4 (&acc)[4][2], int first, int c0) const {
#pragma unroll
        for (int k = 0; k < kResidentSteps; ++k)
            for (uint64_t tokens = __ballot(target[k] >= first && target[k] < first + 32); tokens; tokens &= tokens - 1) {
                const int at = __builtin_ctzll(tokens), row = __builtin_amdgcn_readlane(target[k], at) - first;
                const float rest = a.rest[k * 64 + at];
                bf16x4 h[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int c = c0 + 4 * me.lq + 16 * i;
                    h[i] = *reinterpret_cast<const bf16x4*>(a.H + static_cast<int64_t>(k * 64 + at) * a.d + (c < a.d ? c : 0));
                }
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    if (row >> 4 != j || (row & 15) != me.l15 || rest == 0.f) continue;
#pragma unroll
                    for (int i = 0; i < 4; ++i) add_times(acc[i][j], rest, h[i]);
                }
            }
        mid_nt::wait_vmcnt<0>();        // or the compiler would wait for loads of this branch, and so for the stores, wherever it is left
    }
    template <bool PAST>
    __device__ __forceinline__ void run(const Lane& me, unsigned char* lds, int pos) const {
        const Grad& a = this->a;
        const int db = __builtin_amdgcn_readfirstlane(pos % n_db), b0 = __builtin_amdgcn_readfirstlane(pos / n_db * a.blocks), b1 = b0 + a.blocks < n_vb ? b0 + a.blocks : n_vb;
        const int steps = (n_active + 63) / 64, c0 = db * 256 + me.wave * 64;
        const bool idle = c0 >= a.d;
        const unsigned lds0 = static_cast<unsigned>(reinterpret_cast<size_t>((lds_ptr_t)lds));
        int off[2];
#pragma unroll
        for (int h2 = 0; h2 < 2; ++h2) {
            const int e = me.l15 >> 2, q = me.l15 & 3, k = 8 * me.lq + 4 * h2 + e;
            off[h2] = k * 128 + (((q >> 1) ^ mid_nt::k_swizzle<64>(k)) << 4) + (q & 1) * 8;
        }
        const int row = me.lane >> 3;       // of 8 that a load fetches

        // the hidden states, two steps at a time through the wavefront's own quarter of the LDS
        bf16x8 h[kResidentSteps][2][4];
        const int valid = a.d - c0 < 64 ? (a.d - c0) / 8 : 8;
        const unsigned own = lds0 + me.wave * (LDS_BYTES / 4);
        const char* const h_base = reinterpret_cast<const char*>(a.H) + c0 * 2;
#pragma unroll
        for (int k0 = 0; k0 < kResidentSteps; k0 += 2) {
            if (idle || k0 >= steps) break;
#pragma unroll
            for (int u = 0; u < 16; ++u) {
                if (k0 + u / 8 >= kResidentSteps || k0 + u / 8 >= steps) break;
                const int r = 8 * u + row, t = k0 * 64 + r, c = (me.lane & 7) ^ mid_nt::k_swizzle<64>(r & 63);
                load(h_base, static_cast<unsigned>(t < n_active ? t : n_active - 1) * (a.d * 2u) + (c < valid ? c : valid - 1) * 16, own + u * 1024);
            }
            mid_nt::wait_vmcnt<0>();
            asm volatile("" ::: "memory");
#pragma unroll
            for (int k = k0; k < k0 + 2 && k < kResidentSteps; ++k)
#pragma unroll
                for (int half = 0; half < 2; ++half)
#pragma unroll
                    for (int i = 0; i < 4; ++i) h[k][half][i] = down(lds + me.wave * (LDS_BYTES / 4) + (k - k0) * 8192 + half * 4096, off, i);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        }
        int target[kResidentSteps];         // rows of the workgroup's
        unsigned targets = 0;               // blocks that hold one
#pragma unroll
        for (int k = 0; k < kResidentSteps; ++k) {
            const int t = k * 64 + me.lane;
            target[k] = t < n_active ? a.target[t] - a.v0 - b0 * 64 : -1;
            if (target[k] >= 0 && target[k] < (b1 - b0) * 64) targets |= 1u << (target[k] / 64);
        }
#pragma unroll
        for (int o = 32; o > 0; o /= 2) targets |= __shfl_xor(targets, o);
        targets = __builtin_amdgcn_readfirstlane(targets);
        __syncthreads();

        const char* base = reinterpret_cast<const char*>(a.dz) + static_cast<int64_t>(b0) * 128;
        const unsigned stride = static_cast<unsigned>(a.v_stride) * 2;
        unsigned voff[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int r = (me.wave * 2 + u) * 8 + row;
            voff[u] = r * stride + ((me.lane & 7) ^ mid_nt::k_swizzle<64>(r)) * 16;
        }
        auto issue = [&](int stage) {
            const char* from = base;
            for (int k = 0; k < steps; ++k) {
#pragma unroll
                for (int u = 0; u < 2; ++u) load(from, voff[u], lds0 + stage * kStage + k * 8192 + (me.wave * 2 + u) * 1024);
                from += static_cast<int64_t>(stride) * 64;
            }
            base += 128;
        };
        if (b0 < b1) issue(0);
        const bool rows_out = !a.write_sum && !a.read_sum && c0 + 64 <= a.d;
        bool counted = false;               // the wavefront's last eight accesses are the stores of the block before
        for (int b = b0; b < b1; ++b) {
            if (counted) mid_nt::wait_vmcnt<8>();
            else mid_nt::wait_vmcnt<0>();
            __syncthreads();
            const int stage = (b - b0) & 1;
            if (b + 1 < b1) issue(stage ^ 1);
            if (idle) continue;
            const unsigned char* st = lds + stage * kStage;
            counted = rows_out && b * 64 + 64 <= a.n_v;
#pragma unroll
            for (int j = 0; j < 4; j += 2) {
                f32x4 acc[4][2];
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[i][0] = acc[i][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int k = 0; k < kResidentSteps; ++k) {
                    if (k >= steps) break;
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        const unsigned char* at = st + k * 8192 + half * 4096;
                        const bf16x8 f0 = down(at, off, j), f1 = down(at, off, j + 1);
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            acc[i][0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(h[k][half][i], f0, acc[i][0], 0, 0, 0);
                            acc[i][1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(h[k][half][i], f1, acc[i][1], 0, 0, 0);
                        }
                    }
                }
                const int r0 = b * 64 + j * 16;
                if ((targets >> (b - b0)) & 1) add_rests(me, target, acc, r0 - b0 * 64, c0);
                if (counted) {
#pragma unroll
                    for (int jj = 0; jj < 2; ++jj) {
                        uint16_t* to = a.grad_w + static_cast<int64_t>(r0 + jj * 16 + (me.l15 & 7)) * a.d + c0 + me.place(me.l15 < 8 ? 0 : 2);
                        u32x4 first, second;
                        whole_lines(me, exchange(acc[0][jj], acc[1][jj]), exchange(acc[2][jj], acc[3][jj]), first, second);
                        if constexpr (PAST) {
                            __builtin_nontemporal_store(first, reinterpret_cast<u32x4*>(to));
                            __builtin_nontemporal_store(second, reinterpret_cast<u32x4*>(to + 8 * static_cast<int64_t>(a.d)));
                        } else {
                            *reinterpret_cast<u32x4*>(to) = first;
                            *reinterpret_cast<u32x4*>(to + 8 * static_cast<int64_t>(a.d)) = second;
                        }
                    }
                } else store_rows<Part>(me, acc, r0, a.n_v, c0, a.d, a.sum, a.read_sum, a.write_sum, a.grad_w, [](int r) { return r; });
            }
        }
    }
};

template <class CH>
__global__ __launch_bounds__(CH::NT, 2) void products_resident_kernel(Grad a) {
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    const int n_active = __builtin_amdgcn_readfirstlane(*a.n_active);
    if (static_cast<int>(blockIdx.x) < a.grid_h) {
        const HiddenTiles<CH> tiles(a, n_active);
        const int pos = place(blockIdx.x, tiles.total());
        if (pos < 0) return;
        int s, tb, db;
        tiles.at(pos, s, tb, db);
        const auto rests = tiles.rests(Lane(), s, tb);
        f32x4 acc[CH::TI][CH::TJ];
        multiply<CH, false, true>(tiles.walk(s, tb, db), lds, acc);
        tiles.store(Lane(), rests, acc, s, tb, db);
        return;
    }
    const ResidentTiles tiles(a, n_active);
    const int pos = place(blockIdx.x - a.grid_h, tiles.total());
    if (pos < 0) return;
    if (a.stream && !a.write_sum) tiles.run<true>(Lane(), lds, pos);
    else tiles.run<false>(Lane(), lds, pos);
}

template <class CH, class CW>
__global__ __launch_bounds__(CH::NT) void products_kernel(Grad a) {
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    const int n_active = __builtin_amdgcn_readfirstlane(*a.n_active);
    if (static_cast<int>(blockIdx.x) < a.grid_h) {
        const HiddenTiles<CH> tiles(a, n_active);
        const int pos = place(blockIdx.x, tiles.total());
        if (pos < 0) return;
        int s, tb, db;
        tiles.at(pos, s, tb, db);
        const auto rests = tiles.rests(Lane(), s, tb);
        f32x4 acc[CH::TI][CH::TJ];
        multiply<CH, false, true>(tiles.walk(s, tb, db), lds, acc);
        tiles.store(Lane(), rests, acc, s, tb, db);
        return;
    }
    const HeadTiles<CW> tiles(a, n_active);
    const int pos = place(blockIdx.x - a.grid_h, tiles.total());
    if (pos < 0) return;
    int s, vt, db;
    tiles.at(pos, s, vt, db);
    const auto rests = tiles.rests(Lane(), s, vt);
    f32x4 acc[CW::TI][CW::TJ];
    multiply<CW, true, true>(tiles.walk(s, vt, db), lds, acc);
    tiles.store(Lane(), rests, acc, s, vt, db);
}

// Slabs added in order: of dL/dh to the tokens' own rows (blocks up to blocks_h), of dL/dW to what its tiles would have written.
__device__ __forceinline__ f32x4 slab_sum(const float* slabs, int64_t stride, int n) {
    constexpr int kInFlight = 8;
    f32x4 x = {0.f, 0.f, 0.f, 0.f};
    for (int s0 = 0; s0 < n; s0 += kInFlight) {
        f32x4 y[kInFlight];
#pragma unroll
        for (int s = 0; s < kInFlight; ++s) y[s] = *reinterpret_cast<const f32x4*>(slabs + (s0 + s < n ? s0 + s : s0) * stride);
#pragma unroll
        for (int s = 0; s < kInFlight; ++s)
            if (s0 + s < n) x += y[s];
    }
    return x;
}
__global__ __launch_bounds__(256) void join_kernel(Grad a, int n_slabs, int blocks_h) {
    const int vecs = a.d / 4, n_active = *a.n_active;
    if (static_cast<int>(blockIdx.x) < blocks_h) {
        const int64_t total = static_cast<int64_t>(n_active) * vecs;
        for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < total; i += static_cast<int64_t>(blocks_h) * 256) {
            const int t = static_cast<int>(i / vecs), c = static_cast<int>(i - static_cast<int64_t>(t) * vecs) * 4;
            *reinterpret_cast<bf16x4*>(a.grad_hidden + static_cast<int64_t>(a.row[t]) * a.d + c) = __builtin_convertvector(slab_sum(a.slabs + i * 4, a.slab_stride, n_slabs), bf16x4);
        }
        return;
    }
    const int parts = ((n_active + 63) / 64 + a.k64_per_part - 1) / a.k64_per_part, first = blockIdx.x - blocks_h, blocks = gridDim.x - blocks_h;
    const int64_t total = static_cast<int64_t>(a.n_v) * vecs;
    for (int64_t i = static_cast<int64_t>(first) * 256 + threadIdx.x; i < total; i += static_cast<int64_t>(blocks) * 256) {
        f32x4 x = slab_sum(a.slabs_w + i * 4, a.slab_w_stride, parts);
        if (a.read_sum) x += *reinterpret_cast<const f32x4*>(a.sum + i * 4);
        if (a.write_sum) *reinterpret_cast<f32x4*>(a.sum + i * 4) = x;
        else *reinterpret_cast<bf16x4*>(a.grad_w + i * 4) = __builtin_convertvector(x, bf16x4);
    }
}

__global__ __launch_bounds__(256) void zero_kernel(u32x4* out, int64_t n) {
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < n; i += static_cast<int64_t>(gridDim.x) * 256) out[i] = u32x4{0, 0, 0, 0};
}

template <void (*KERNEL)(Grad), int NT, int LDS>
bool start(unsigned grid, const Grad& a, hipStream_t st) {
    static arrol_device_flags ok;
    if (!arrol_allow_lds(KERNEL, LDS, ok)) return false;
    arrol_launch(KERNEL, dim3(grid), dim3(NT), LDS, st, a);
    return true;
}
template <class C>
bool start_dz(unsigned grid, const Grad& a, hipStream_t st) { return start<dz_kernel<C>, C::NT, C::LDS_BYTES>(grid, a, st); }
template <class CH, class CW>
bool start_products(unsigned grid, const Grad& a, hipStream_t st) {
    static_assert(CH::NT == CW::NT, "one launch");
    return start<products_kernel<CH, CW>, CH::NT, (CH::LDS_BYTES > CW::LDS_BYTES ? CH::LDS_BYTES : CW::LDS_BYTES)>(grid, a, st);
}
bool launch_dz(Form f, unsigned grid, const Grad& a, hipStream_t st) {
    return f == kRing ? start_dz<Ring>(grid, a, st) : f == kMid160 ? start_dz<Mid160>(grid, a, st) : f == kMid128 ? start_dz<Mid128>(grid, a, st) : f == kMidFew ? start_dz<MidFew>(grid, a, st) : start_dz<Mid64>(grid, a, st);
}
template <class C>
bool start_found(unsigned grid, const Grad& a, const Gather& g, hipStream_t st) {
    static arrol_device_flags ok;
    constexpr int kBytes = C::LDS_BYTES + sizeof(Found);
    if (!arrol_allow_lds(&dz_found_kernel<C>, kBytes, ok)) return false;
    arrol_launch(dz_found_kernel<C>, dim3(grid), dim3(C::NT), kBytes, st, a, g);
    return true;
}
bool launch_found(Form f, unsigned grid, const Grad& a, const Gather& g, hipStream_t st) {
    return f == kMid160 ? start_found<Mid160>(grid, a, g, st) : f == kMid128 ? start_found<Mid128>(grid, a, g, st) : f == kMidFew ? start_found<MidFew>(grid, a, g, st) : start_found<Mid64>(grid, a, g, st);
}
template <class CH>
bool start_resident(unsigned grid, const Grad& a, hipStream_t st) {
    return start<products_resident_kernel<CH>, CH::NT, (CH::LDS_BYTES > ResidentTiles::LDS_BYTES ? CH::LDS_BYTES : ResidentTiles::LDS_BYTES)>(grid, a, st);
}
bool launch_products(Form f, const Grad& a, hipStream_t st) {
    const unsigned grid = static_cast<unsigned>(a.grid_h + a.grid_w);
    if (a.blocks)
        return f == kMid160 ? start_resident<Mid160>(grid, a, st) : f == kMid128 ? start_resident<Mid128>(grid, a, st)
             : f == kMidFew ? start_resident<MidFew>(grid, a, st) : start_resident<Mid64>(grid, a, st);
    return f == kRing ? start_products<Ring, Ring>(grid, a, st) : f == kMid160 ? start_products<Mid160, Mid128>(grid, a, st) : f == kMid128 ? start_products<Mid128, Mid128>(grid, a, st)
         : f == kMidFew ? start_products<MidFew, Mid128>(grid, a, st) : start_products<Mid64, Mid64>(grid, a, st);
}

unsigned rounded(int64_t n) { return static_cast<unsigned>((n + kXcds - 1) / kXcds * kXcds); }

}  // namespace

static int refused() {
    arrol_launch_status();      // empties the slot of earlier launches
    return ARROL_EHIP;
}

extern "C" size_t arrol_logprob_grad_workspace_bytes(int64_t T, int32_t V, int32_t d, int32_t want_lm_head) {
    return sizes_ok(T, V, d) && T > 0 ? workspace(T, V, d, want_lm_head != 0).bytes : 0;
}

extern "C" int arrol_logprob_grad_kernels(int64_t T, int32_t V, int32_t d, int32_t* logit_rows, int32_t* logit_tokens, int32_t* product_columns, int32_t* product_tokens,
                                          int32_t* slabs, int32_t* parts, int32_t* n_pieces, int32_t* found) {
    if (!sizes_ok(T, V, d) || T < 1 || !logit_rows || !logit_tokens || !product_columns || !product_tokens || !slabs || !parts || !n_pieces || !found) return ARROL_EINVAL;
    const Pieces p = pieces(T, V, d);
    *logit_rows = kSize[p.dz].bm, *logit_tokens = kSize[p.dz].bn, *product_columns = kSize[p.products].bm, *product_tokens = kSize[p.products].bn;
    *slabs = p.slabs, *parts = p.blocks ? 0 : p.parts, *n_pieces = static_cast<int32_t>(p.n_rows * p.n_v < 0x7fffffff ? p.n_rows * p.n_v : 0x7fffffff), *found = found_by_dz(p, p.rows);
    return ARROL_OK;
}

extern "C" int arrol_logprob_grad(const void* hidden, const void* lm_head, const int32_t* targets, const float* lse, const float* grad_logp, int64_t T, int32_t V,
                                  int32_t d, void* grad_hidden, void* grad_lm_head, float* lm_head_sum, void* workspace_, size_t workspace_bytes, void* stream) {
    if (!sizes_ok(T, V, d) || (!grad_hidden && !grad_lm_head && !lm_head_sum && T > 0) || (grad_lm_head && lm_head_sum)) return ARROL_EINVAL;
    if (T > 0 && (!hidden || !lm_head || !targets || !lse || !grad_logp)) return ARROL_EINVAL;
    for (const void* p : {hidden, lm_head, static_cast<const void*>(grad_hidden), static_cast<const void*>(grad_lm_head), static_cast<const void*>(lm_head_sum)})
        if (!arrol_aligned16(p)) return ARROL_EINVAL;
    const auto st = static_cast<hipStream_t>(stream);
    if (T == 0) {
        if (grad_lm_head) {
            const int64_t vecs = static_cast<int64_t>(V) * d / 8, blocks = (vecs + 255) / 256;
            arrol_launch(zero_kernel, dim3(static_cast<unsigned>(blocks < 4096 ? blocks : 4096)), dim3(256), 0, st, static_cast<u32x4*>(grad_lm_head), vecs);
        }
        return arrol_launch_status();
    }
    const Workspace ws = workspace(T, V, d, grad_lm_head != nullptr);
    if (!workspace_ || !arrol_aligned16(workspace_) || workspace_bytes < ws.bytes) return ARROL_EWORKSPACE;
    auto* base = static_cast<unsigned char*>(workspace_);
    const Pieces p = pieces(T, V, d);
    Grad a = {};
    a.H = reinterpret_cast<uint16_t*>(base + ws.H), a.dz = reinterpret_cast<uint16_t*>(base + ws.dz);
    a.g = reinterpret_cast<float*>(base + ws.g), a.lse = reinterpret_cast<float*>(base + ws.lse);
    a.target = reinterpret_cast<int32_t*>(base + ws.target), a.row = reinterpret_cast<int32_t*>(base + ws.row), a.rest = reinterpret_cast<float*>(base + ws.rest);
    a.n_active = reinterpret_cast<int32_t*>(base + ws.n_active);
    a.d = d, a.stream = static_cast<int64_t>(V) * d > kCachedElements;
    const Size& size = kSize[p.products];
    for (int64_t piece = 0; piece < p.n_rows; ++piece) {
        const int64_t t0 = piece * p.rows, rows = T - t0 < p.rows ? T - t0 : p.rows;
        Gather g;
        g.hidden = static_cast<const uint16_t*>(hidden) + t0 * d, g.targets = targets + t0, g.lse = lse + t0, g.grad_logp = grad_logp + t0;
        g.H = const_cast<uint16_t*>(a.H), g.grad_hidden = grad_hidden ? static_cast<uint16_t*>(grad_hidden) + t0 * d : nullptr;
        g.g = const_cast<float*>(a.g), g.lse_out = const_cast<float*>(a.lse), g.target = const_cast<int32_t*>(a.target), g.row = const_cast<int32_t*>(a.row);
        g.n_active = const_cast<int32_t*>(a.n_active), g.T = static_cast<int>(rows), g.V = V, g.d = d;
        const bool found = found_by_dz(p, rows), want_head = grad_lm_head || lm_head_sum;
        if (!found) arrol_launch(gather_kernel, dim3(static_cast<unsigned>((rows + kGatherRows - 1) / kGatherRows)), dim3(256), 0, st, g);
        if (!want_head) g.H = nullptr;
        const bool direct = p.slabs == 1 && p.n_v == 1;
        a.slab_stride = rows * d;
        a.slabs = direct ? nullptr : reinterpret_cast<float*>(base + ws.slabs);
        a.grad_hidden = g.grad_hidden;
        for (int64_t q = 0; q < p.n_v; ++q) {
            const int64_t v0 = q * p.v, n_v = V - v0 < p.v ? V - v0 : p.v;
            a.W = static_cast<const uint16_t*>(lm_head) + v0 * d, a.v0 = static_cast<int>(v0), a.n_v = static_cast<int>(n_v), a.v_stride = static_cast<int>(p.v);
            const unsigned grid = rounded(tiles_of(rows, n_v, kSize[p.dz].bn, kSize[p.dz].bm));
            if (!(found ? launch_found(p.dz, grid, a, g, st) : launch_dz(p.dz, grid, a, st))) return refused();
            a.k64_per_slab = p.k64_per_slab, a.add = q > 0;
            a.grid_h = grad_hidden ? static_cast<int>(rounded(tiles_of(rows, d, size.bn, size.bm) * p.slabs)) : 0;
            a.grid_w = 0;
            if (want_head) {
                a.grid_w = static_cast<int>(rounded(p.blocks ? tiles_of(n_v, d, 64 * p.blocks, 256) : tiles_of(n_v, d, size.bn_w, size.bm_w) * p.parts));
                a.blocks = p.blocks;
                a.slabs_w = p.parts > 1 ? reinterpret_cast<float*>(base + ws.slabs_w) : nullptr;
                a.slab_w_stride = n_v * d, a.k64_per_part = static_cast<int>(((rows + 63) / 64 + p.parts - 1) / p.parts);
                a.sum = (lm_head_sum ? lm_head_sum : reinterpret_cast<float*>(base + ws.sum)) + v0 * d;
                a.grad_w = grad_lm_head ? static_cast<uint16_t*>(grad_lm_head) + v0 * d : nullptr;
                a.read_sum = lm_head_sum || piece > 0, a.write_sum = lm_head_sum || piece + 1 < p.n_rows;
            }
            if (!launch_products(p.products, a, st)) return refused();
            const bool join_h = grad_hidden && !direct && q + 1 == p.n_v, join_w = want_head && p.parts > 1;
            const int64_t blocks_h = join_h ? (rows * (d / 4) + 255) / 256 : 0, blocks_w = join_w ? (n_v * (d / 4) + 255) / 256 : 0;
            const unsigned of_h = static_cast<unsigned>(blocks_h < 4096 ? blocks_h : 4096), of_w = static_cast<unsigned>(blocks_w < 4096 ? blocks_w : 4096);
            if (join_h || join_w) arrol_launch(join_kernel, dim3(of_h + of_w), dim3(256), 0, st, a, p.slabs, static_cast<int>(of_h));
        }
    }
    return arrol_launch_status();
}
