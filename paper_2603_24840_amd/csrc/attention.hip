// Attention over packed sequences and its gradient (the prompts' pass, and the survivors' forward and backward pass of the update).
//
// Per sequence with nq queries and nk keys, query head h and its kv head:
//   z_ij = scale <q_i, k_j>,  visible j: j + nq <= i + nk (causal, the ends aligned) or all;  lse_i = log sum_j exp z_ij
//   o_i = sum_j exp(z_ij - lse_i) v_j
//   p_ij = exp(z_ij - lse_i),  D_i = <do_i, o_i>,  ds_ij = p_ij (<do_i, v_j> - D_i)
//   dv_j = sum_i p_ij do_i,  dk_j = scale sum_i ds_ij q_i (both over every query head of the kv head),  dq_i = scale sum_j ds_ij k_j
// No [queries, keys] matrix reaches memory: the forward pass keeps a running maximum and sum per row, the gradient forms z again
// from lse.
#include "attention_tile.h"

namespace {
using namespace attention;

constexpr int kThreads = 256, kWaves = kThreads / ARROL_WAVE, kOwn = 32 * kWaves;   // 32 own rows a wavefront

struct Problem {
    const uint16_t *q, *k, *v;
    int64_t q_stride, k_stride, v_stride;   // elements between rows
    Packed pq, pk;
    int heads, kv_heads, hd, causal;
    float scale;
};

// What a workgroup works on: tiles of the packed rows x heads.  Consecutive workgroups take consecutive kv heads (with 8 of
// them an XCD's L2 sees one kv head), then the query heads that share it, and tiles from the last one down where late ones are long.
__device__ __forceinline__ void split_block(unsigned block, int kv_heads, int& kvh, int& rest) {      // (a grid has fewer than 2^24 workgroups)
    kvh = static_cast<int>(block % static_cast<unsigned>(kv_heads));
    rest = static_cast<int>(block / static_cast<unsigned>(kv_heads));
}

__device__ __forceinline__ int clamp32(int64_t n) { return uniform(static_cast<int>(n < 0 ? 0 : n < 32 ? n : 32)); }

// Where a workgroup's queries lie, and which keys they see.  Its four wavefronts have 32 rows each: 32 rows of HEADS = 4 heads of a kv head, 64 of 2, or
// 128 of one - as many heads as share it, so that few rows (short or ragged sequences) fill the workgroup, and its wavefronts see the same keys: 64 prompts
// of up to 512 tokens, 32 heads over 8, 70 us, with one head a workgroup 77.
template <int HEADS>
struct QueryBlock {
    static constexpr int kRows = kOwn / HEADS;
    int64_t row0, k_begin;          // the wavefront's first row; the sequence's first key
    int head, nk, own_valid;        // the wavefront's; keys; rows of the wavefront that there are
    int sees;                       // keys that this lane's row sees
    int sees_least, sees_most;      // over the wavefront's rows (causal: its first and its last valid row)
    int reach;                      // most over the workgroup's rows
    __device__ __forceinline__ bool find(const Problem& a, int64_t tile, int first_head, int wave, int lane) {
        int segment;
        int64_t first, q_begin, end;
        if (!find_tile<kRows>(a.pq, tile, lane, segment, first, q_begin, end)) return false;
        head = first_head + wave % HEADS;
        const int nq = uniform(static_cast<int>(end - q_begin));
        k_begin = 0, nk = 0;
        if (segment >= 1 && segment <= a.pq.n) {       // rows of no sequence see no keys: zeros
            const bool same = a.pk.cu == a.pq.cu && a.pk.T == a.pq.T;
            k_begin = same ? q_begin : a.pk.bound(segment);
            const int64_t n = (same ? end : a.pk.bound(segment + 1)) - k_begin;
            nk = uniform(static_cast<int>(n < 0 ? 0 : n));
        }
        row0 = first + 32 * (wave / HEADS);
        own_valid = clamp32(end - row0);
        // query i of its sequence sees keys j < min(nk, i + 1 + nk - nq)
        const auto seen_by = [&](int i) {
            const int s = a.causal ? nk + (i + 1 - nq) : nk;
            return s < 0 ? 0 : s < nk ? s : nk;
        };
        const int at = uniform(static_cast<int>(first - q_begin)), i0 = at + 32 * (wave / HEADS);
        sees = seen_by(i0 + (lane & 31));
        sees_least = seen_by(i0);
        sees_most = own_valid > 0 ? seen_by(i0 + own_valid - 1) : 0;
        reach = seen_by((nq - at < kRows ? nq - at : kRows) - 1 + at);
        return true;
    }
};

// What a wavefront of the forward pass leaves: the output, or, where the keys of a sequence are cut into several ranges, its part of it.
struct Output {
    uint16_t* out;
    float* lse;
    int splits;                     // ranges of the keys
    float *part_o, *part_ml;        // [split][row][head][hd], [split][row][head][2] where there are several
};

// O of a wavefront's rows over the keys [from, to), once more and by themselves: key by key, so that a key takes no part in a row that does not see it.  Where
// all rows see all keys of whole tiles, or V is finite, the matrix instructions give the same; but the product of a hidden key's weight, 0, and an
// infinity or NaN of its value is NaN, and so is that of a place past the last key, which holds this one's value once more.  Only rows that hold such values come here.
template <int HD, class Block>
__device__ __forceinline__ void repair_rows(const Problem& a, const Block& w, const bf16x8 (&qf)[HD / 16], int kvh, int from, int to, float base, int lane, f32x16 (&o)[HD / 32]) {
    const int half = lane >> 5;
    const float c = a.scale * kLog2e;
#pragma unroll
    for (int d = 0; d < HD / 32; ++d) o[d] = 0.f;
    for (int j = from; j < to; ++j) {
        const uint16_t* k = a.k + (w.k_begin + j) * a.k_stride + static_cast<int64_t>(kvh) * a.hd;
        const uint16_t* v = a.v + (w.k_begin + j) * a.v_stride + static_cast<int64_t>(kvh) * a.hd;
        float z = 0.f;
#pragma unroll
        for (int s = 0; s < HD / 16; ++s) {
            const int e = 16 * s + 8 * half;
            if (e >= a.hd) continue;
            const bf16x8 x = *reinterpret_cast<const bf16x8*>(k + e);
#pragma unroll
            for (int i = 0; i < 8; ++i) z = fmaf(static_cast<float>(x[i]), static_cast<float>(qf[s][i]), z);
        }
        z = half_sum(z);
        const bool seen = j < w.sees;
        const float p = __builtin_amdgcn_exp2f(fmaf(z, c, -base));
#pragma unroll
        for (int d = 0; d < HD / 32; ++d)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int e = 32 * d + 8 * (r >> 2) + 4 * half + (r & 3);
                if (e >= a.hd) continue;
                const float x = bf16_lo(v[e]);
                o[d][r] = seen ? fmaf(p, x, o[d][r]) : o[d][r];
            }
    }
}

// Forward pass: a workgroup walks over the keys in tiles of 64, a wavefront with 32 queries of a head.
// S^T = K Q^T and O^T += V^T P^T, so that a query's statistics are its lane's.  The tiles that come next are on their way into the other halves of the
// LDS.  With heads of 128, whose registers leave two wavefronts to a SIMD, the scores of the next tile are formed while the exponentials of this one
// are (K runs a tile ahead of V): 4 survivors of up to 4,096 tokens, 32 heads over 8, 297 us against 331.  With heads of 64 four fit, which
// do that for each other: 64 prompts of up to 512 tokens 70 us, and 84 the other way.
template <int HD, int HEADS>
__global__ __launch_bounds__(kThreads, 2) void attention_forward_kernel(Problem a, int64_t tiles, Output to) {
    constexpr int BK = 64;
    constexpr bool kAhead = HD == 128;
    using T = Tile<HD>;
    constexpr int kTileBytes = BK * T::kRowBytes;
    __shared__ __align__(1024) unsigned char lds[2][2][kTileBytes];      // [slot][K, V]
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
    const int per = a.heads / a.kv_heads, head_blocks = per / HEADS;
    int kvh, rest;
    split_block(blockIdx.x, a.kv_heads, kvh, rest);
    const int first_head = kvh * per + rest % head_blocks * HEADS;
    rest /= head_blocks;
    const int split = rest % to.splits;
    QueryBlock<HEADS> w;
    if (!w.find(a, tiles - 1 - rest / to.splits, first_head, wave, lane)) return;
    const int head = w.head;
    // this workgroup's tiles of 64 keys: those that some of its rows see, or a range of them
    const int all = (w.reach + BK - 1) / BK, t_lo = all * split / to.splits, n_tiles = all * (split + 1) / to.splits - t_lo;      // (fewer than 2^25 tiles, at most 16 ranges)

    bf16x8 qf[HD / 16];
    load_own<HD>(qf, a.q + w.row0 * a.q_stride + static_cast<int64_t>(head) * a.hd, a.q_stride, w.own_valid, a.hd, lane);
    const uint16_t* kp = uniform(a.k + (w.k_begin + static_cast<int64_t>(t_lo) * BK) * a.k_stride + static_cast<int64_t>(kvh) * a.hd);
    const uint16_t* vp = uniform(a.v + (w.k_begin + static_cast<int64_t>(t_lo) * BK) * a.v_stride + static_cast<int64_t>(kvh) * a.hd);
    f32x16 o[HD / 32];
#pragma unroll
    for (int d = 0; d < HD / 32; ++d) o[d] = 0.f;
    float m = -INFINITY, l = 0.f;                 // of z * log2 e; l is this lane's half of the row
    const float c = a.scale * kLog2e;

    Stream<HD, BK, kWaves> ks, vs;
    const int keys = w.nk - t_lo * BK, whole = keys / BK;      // from the first tile on; tiles of 64 keys that exist
    const unsigned lds0 = lds_address(lds), row_at = T::row_base(lane), column_at = T::column_base(lane);
    const auto fetch_k = [&](int t) {
        if (t == whole) ks.point(static_cast<unsigned>(a.k_stride) * 2, keys - t * BK, a.hd, wave, lane);
        ks.issue(kp, lds0 + (t & 1) * 2 * kTileBytes, a.hd, wave);
        kp += BK * a.k_stride;
    };
    const auto fetch_v = [&](int t) {
        if (t == whole) vs.point(static_cast<unsigned>(a.v_stride) * 2, keys - t * BK, a.hd, wave, lane);
        vs.issue(vp, lds0 + ((t & 1) * 2 + 1) * kTileBytes, a.hd, wave);
        vp += BK * a.v_stride;
    };
    const auto fetch_for = [&](int t) {           // what iteration t + 1 needs
        if (t + 2 < n_tiles) fetch_k(t + 2);
        if (t + 1 < n_tiles) fetch_v(t + 1);
    };
    const int clear = w.sees_least / BK - t_lo, most = (w.sees_most + BK - 1) / BK - t_lo, needed = most < 0 ? 0 : most < n_tiles ? most : n_tiles;
    const auto scores = [&](int t, int b, f32x16 (&s)[BK / 32]) {
        const unsigned rows = fresh(lds0 + (t & 1) * 2 * kTileBytes + row_at);
        s[b] = 0.f;
#pragma unroll
        for (int e = 0; e < HD / 16; ++e) s[b] = mfma32(T::by_row(rows, e, 32 * b * T::kRowBytes), qf[e], s[b]);
    };
    // weights and output of tile t from its scores s; NEXT: and the scores of the next one
    const auto step = [&](auto more, int t, f32x16 (&s)[BK / 32], f32x16 (&next)[BK / 32]) {
        constexpr bool NEXT = decltype(more)::value;
        const unsigned columns = fresh(lds0 + (t & 1) * 2 * kTileBytes + column_at);
        if (t >= clear) {       // some row of the wavefront does not see all of the tile
            stay_branch();
            const int limit = w.sees - (t_lo + t) * BK - 4 * half;
#pragma unroll
            for (int b = 0; b < BK / 32; ++b)
#pragma unroll
                for (int r = 0; r < 16; ++r) s[b][r] = 32 * b + 8 * (r >> 2) + (r & 3) < limit ? s[b][r] : -INFINITY;
        }
        if constexpr (NEXT) scores(t + 1, 0, next);
        float top = -INFINITY;
#pragma unroll
        for (int b = 0; b < BK / 32; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) top = fmaxf(top, s[b][r]);
        top = half_max(top) * c;
        // the sums are moved to a new maximum only where it has grown by 2^8: exp2 then stays below 256 and nothing is lost
        if (__any(top > m + 8.f)) {
            const float up = fmaxf(m, top);
            const float f = up == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - up);
            m = up;
            l *= f;
#pragma unroll
            for (int d = 0; d < HD / 32; ++d) o[d] *= f;
        }
        const float base = m == -INFINITY ? 0.f : m;
        if constexpr (NEXT) scores(t + 1, 1, next);
#pragma unroll
        for (int b = 0; b < BK / 32; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                s[b][r] = __builtin_amdgcn_exp2f(fmaf(s[b][r], c, -base));
                l += s[b][r];
            }
#pragma unroll
        for (int b = 0; b < BK / 32; ++b)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const bf16x8 p = as_fragment(s[b], e);      // weights in bf16: at most 2^-8 off each, their sum l is of the unrounded ones
#pragma unroll
                for (int d = 0; d < HD / 32; ++d) o[d] = mfma32(T::by_column(columns, 2 * b + e, d, kTileBytes), p, o[d]);
            }
    };
    clear_tiles<HD>(&lds[0][0][0], sizeof lds, a.hd);
    if (n_tiles > 0) {
        ks.point(static_cast<unsigned>(a.k_stride) * 2, BK, a.hd, wave, lane);
        vs.point(static_cast<unsigned>(a.v_stride) * 2, BK, a.hd, wave, lane);
        fetch_k(0);
        fetch_v(0);
        if (kAhead && n_tiles > 1) fetch_k(1);
    }
    tiles_ready();
    int t = 0;
    f32x16 x[BK / 32];
    if constexpr (!kAhead) {
        for (; t < n_tiles; ++t) {
            if (t + 1 < n_tiles) {
                fetch_k(t + 1);
                fetch_v(t + 1);
            }
            if (t < needed) {
#pragma unroll
                for (int b = 0; b < BK / 32; ++b) scores(t, b, x);
                step(std::false_type{}, t, x, x);
            }
            tiles_ready();
        }
    } else if (needed > 0) {
        f32x16 y[BK / 32];
#pragma unroll
        for (int b = 0; b < BK / 32; ++b) scores(0, b, x);
        if (n_tiles > 2) tiles_ready();           // every wavefront has read K's first tile, whose place the third one takes
        for (; t + 2 < needed; t += 2) {
            fetch_for(t);
            step(std::true_type{}, t, x, y);
            tiles_ready();
            fetch_for(t + 1);
            step(std::true_type{}, t + 1, y, x);
            tiles_ready();
        }
        if (t + 1 < needed) {
            fetch_for(t);
            step(std::true_type{}, t, x, y);
            tiles_ready();
            ++t;
#pragma unroll
            for (int b = 0; b < BK / 32; ++b) x[b] = y[b];
        }
        fetch_for(t);
        step(std::false_type{}, t, x, y);
        tiles_ready();
        ++t;
    } else if (n_tiles > 2) {
        tiles_ready();
    }
    for (; t < n_tiles; ++t) {                    // tiles of the other wavefronts
        fetch_for(t);
        tiles_ready();
    }
    l = half_sum(l);
    // An output that is no number: is it from a value that some of the rows do not see, or from the last key's, whose place in the last tile's end it has as
    // well (Stream), with weights 0?
    const int end = (t_lo + needed) * BK < w.nk ? (t_lo + needed) * BK : w.nk, least = end < (t_lo + needed) * BK && w.sees_least >= end ? end - 1 : w.sees_least;
    const int hidden = least > t_lo * BK ? least : t_lo * BK;
    if (hidden < end) {
        float odd = 0.f;
#pragma unroll
        for (int d = 0; d < HD / 32; ++d)
#pragma unroll
            for (int r = 0; r < 16; ++r) odd = fmaf(o[d][r], 0.f, odd);        // NaN if any is NaN or infinite
        if (__any(odd != 0.f)) {
            bool found = false;
            for (int j = hidden + lane; j < end; j += 64) {
                const uint16_t* v = a.v + (w.k_begin + j) * a.v_stride + static_cast<int64_t>(kvh) * a.hd;
                for (int e = 0; e < a.hd; ++e) found |= (v[e] & 0x7f80) == 0x7f80;
            }
            if (__any(found)) {
                const int last = w.sees_most < end ? w.sees_most : end;
                repair_rows<HD>(a, w, qf, kvh, t_lo * BK, last, m == -INFINITY ? 0.f : m, lane, o);
            }
        }
    }
    const int64_t row_heads = static_cast<int64_t>(a.heads) * a.hd;
    if (to.splits == 1) {
        store_own<HD>(o, l == 0.f ? 0.f : 1.f / l, &lds[0][0][0] + wave * 32 * T::kRowBytes, to.out + (w.row0 * a.heads + head) * a.hd, row_heads, w.own_valid, a.hd, lane);
        if (to.lse && lane < w.own_valid) to.lse[static_cast<int64_t>(head) * a.pq.T + w.row0 + lane] = l == 0.f ? -INFINITY : m * kLn2 + logf(l);
        return;
    }
    const int64_t at = (split * a.pq.T + w.row0 + (lane & 31)) * a.heads + head;
    if ((lane & 31) >= w.own_valid) return;
    if (half == 0) *reinterpret_cast<f32x2*>(to.part_ml + 2 * at) = f32x2{m, l};
#pragma unroll
    for (int d = 0; d < HD / 32; ++d)
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            const int e = 32 * d + 8 * b + 4 * half;
            if (e < a.hd) *reinterpret_cast<f32x4*>(to.part_o + at * a.hd + e) = f32x4{o[d][4 * b], o[d][4 * b + 1], o[d][4 * b + 2], o[d][4 * b + 3]};
        }
}

// Joins the ranges: 16 lanes a row of a head, 8 head elements each.
__global__ __launch_bounds__(kThreads) void attention_join_kernel(Output to, int64_t T, int heads, int hd) {
    const int64_t rows = T * heads, at = (static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x) / 16;
    const int e = (threadIdx.x & 15) * 8;
    if (at >= rows) return;
    float top = -INFINITY;
    for (int s = 0; s < to.splits; ++s) top = fmaxf(top, to.part_ml[2 * (s * rows + at)]);
    const float base = top == -INFINITY ? 0.f : top;
    float sum = 0.f;
    f32x4 x = {0.f, 0.f, 0.f, 0.f}, y = x;
    for (int s = 0; s < to.splits; ++s) {
        const f32x2 ml = *reinterpret_cast<const f32x2*>(to.part_ml + 2 * (s * rows + at));
        if (ml.x == -INFINITY && ml.y == 0.f) continue;        // nothing seen.  (All scores NaN: the maximum is -inf as well, the sums are NaN.)
        const float f = __builtin_amdgcn_exp2f(ml.x - base);
        sum += f * ml.y;
        if (e < hd) {
            const f32x4* p = reinterpret_cast<const f32x4*>(to.part_o + (s * rows + at) * hd + e);
            x += p[0] * f, y += p[1] * f;
        }
    }
    const float inverse = sum == 0.f ? 0.f : 1.f / sum;
    if (e < hd) {
        typedef float f32x8 __attribute__((ext_vector_type(8)));
        const f32x8 z = {x[0] * inverse, x[1] * inverse, x[2] * inverse, x[3] * inverse, y[0] * inverse, y[1] * inverse, y[2] * inverse, y[3] * inverse};
        *reinterpret_cast<bf16x8*>(to.out + at * hd + e) = __builtin_convertvector(z, bf16x8);
    }
    if (to.lse && e == 0) to.lse[at % heads * T + at / heads] = sum == 0.f ? -INFINITY : top * kLn2 + logf(sum);
}

// A gradient on its way out: bf16 rows [T, heads, hd], or, where the walk is cut into ranges because there are few workgroups, every range's fp32 sums
// [range][T, heads, hd], which attention_grad_join_kernel adds in order.
struct Sums {
    uint16_t* out;
    float* part;
    int64_t T;
    int heads;
};
template <int HD>
__device__ __forceinline__ void store_sums(const f32x16 (&acc)[HD / 32], float factor, unsigned char* tile, const Sums& to, int splits, int split, int64_t row0, int head, int valid,
                                           int hd, int lane) {
    const int64_t stride = static_cast<int64_t>(to.heads) * hd, at = row0 * stride + static_cast<int64_t>(head) * hd;
    if (splits == 1) {
        store_own<HD>(acc, factor, tile, to.out + at, stride, valid, hd, lane);
        return;
    }
    if ((lane & 31) >= valid) return;
    float* mine = to.part + split * to.T * stride + at + (lane & 31) * stride;
#pragma unroll
    for (int d = 0; d < HD / 32; ++d)
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            const int e = 32 * d + 8 * b + 4 * (lane >> 5);
            if (e < hd) *reinterpret_cast<f32x4*>(mine + e) = f32x4{acc[d][4 * b], acc[d][4 * b + 1], acc[d][4 * b + 2], acc[d][4 * b + 3]} * factor;
        }
}
// 8 elements a lane
__global__ __launch_bounds__(kThreads) void attention_grad_join_kernel(const float* __restrict__ part, int64_t n, int splits, uint16_t* __restrict__ out) {
    const int64_t i = (static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x) * 8;
    if (i >= n) return;
    f32x4 x = {0.f, 0.f, 0.f, 0.f}, y = x;
    for (int s = 0; s < splits; ++s) {
        const f32x4* p = reinterpret_cast<const f32x4*>(part + s * n + i);
        x += p[0], y += p[1];
    }
    typedef float f32x8 __attribute__((ext_vector_type(8)));
    *reinterpret_cast<bf16x8*>(out + i) = __builtin_convertvector((f32x8{x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]}), bf16x8);
}

// dK and dV: a workgroup takes 128 keys of a kv head and walks over the queries of every head that reads them in tiles of 64, a wavefront with 32
// of the keys (K and V as fragments in registers); the sum over the shared heads is made in registers, in a fixed order.
// With heads of 128, whose registers leave two wavefronts to a SIMD, these are two groups of four of one workgroup: each takes every other tile (with its own
// part of the LDS), and their sums are added at the end.  That halves the longest walk - the first keys of a long sequence, all heads - which
// bounds the launch where there are few sequences: 4 survivors of up to 4,096 tokens, 32 heads over 8, 1,130 us for the whole gradient with one group and
// 1,030 with two.  With heads of 64 three workgroups of one group fit: 16 survivors of up to 1,000 tokens 199.6 us, and 203 with two groups.
// S = Q K^T and dP = dO V^T have the own key as column and start from -lse / scale and -D of their rows, so that z / scale - lse / scale and
// dp - D come out of the matrix cores (a row that sees nothing has lse = -inf, and is masked everywhere); dV^T += dO^T P, dK^T += Q^T dS.
template <int HD, int GROUPS>
__global__ __launch_bounds__(GROUPS * kThreads, GROUPS == 1 ? 3 : 1) void attention_grad_kv_kernel(Problem a, const uint16_t* __restrict__ go, const float* __restrict__ stats,
                                                                                           int splits, Sums dk, Sums dv) {
    constexpr int BQ = 64;
    using T = Tile<HD>;
    constexpr int kTileBytes = BQ * T::kRowBytes, kSlot = 2 * kTileBytes + 2 * BQ * 4;
    extern __shared__ __align__(1024) unsigned char lds[];       // [group][slot][kSlot]
    const int lane = threadIdx.x & 63, wave8 = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
    const int wave = wave8 & (kWaves - 1), group = wave8 / kWaves;
    const int per = a.heads / a.kv_heads;
    int kvh, tile;
    split_block(blockIdx.x, a.kv_heads, kvh, tile);
    const int split = tile % splits;
    tile /= splits;
    int segment;
    int64_t first, k_begin, end;
    if (!find_tile<kOwn>(a.pk, tile, lane, segment, first, k_begin, end)) return;
    const int64_t row0 = first + 32 * wave;
    const int nk = uniform(static_cast<int>(end - k_begin)), own_valid = clamp32(end - row0), j0 = uniform(static_cast<int>(row0 - k_begin));
    int64_t q_begin = 0;
    int nq = 0;
    if (segment >= 1 && segment <= a.pk.n) {
        const bool same = a.pk.cu == a.pq.cu && a.pk.T == a.pq.T;
        q_begin = same ? k_begin : a.pq.bound(segment);
        const int64_t n = (same ? end : a.pq.bound(segment + 1)) - q_begin;
        nq = uniform(static_cast<int>(n < 0 ? 0 : n));
    }
    // key j is seen by queries i >= j + nq - nk (causal)
    const auto seen_from = [&](int j) {
        const int i = a.causal ? nq + (j - nk) : 0;
        return i < 0 ? 0 : i;
    };
    const int from = seen_from(j0 + (lane & 31)), from_least = seen_from(j0), from_most = seen_from(j0 + 31);
    const int t_first = seen_from(j0 - 32 * wave) / BQ;
    const int n_t = (nq + BQ - 1) / BQ > t_first ? (nq + BQ - 1) / BQ - t_first : 0;
    // tiles, head by head; this workgroup's are those from t_lo on
    const int t_lo = n_t * per * split / splits, total = n_t * per * (split + 1) / splits - t_lo;      // (fewer than 2^25 tiles, at most 16 ranges)

    bf16x8 kf[HD / 16], vf[HD / 16];
    load_own<HD>(kf, a.k + row0 * a.k_stride + static_cast<int64_t>(kvh) * a.hd, a.k_stride, own_valid, a.hd, lane);
    load_own<HD>(vf, a.v + row0 * a.v_stride + static_cast<int64_t>(kvh) * a.hd, a.v_stride, own_valid, a.hd, lane);
    f32x16 gk[HD / 32], gv[HD / 32];
#pragma unroll
    for (int d = 0; d < HD / 32; ++d) gk[d] = 0.f, gv[d] = 0.f;
    const float c = a.scale * kLog2e;
    const int64_t go_stride = static_cast<int64_t>(a.heads) * a.hd;

    Stream<HD, BQ, kWaves> qs, gs;
    const unsigned lds0 = lds_address(lds) + group * 2 * kSlot, row_at = T::row_base(lane), column_at = T::column_base(lane);
    int h = n_t > 0 ? t_lo / n_t : 0, ti = t_lo - h * n_t + group, at = ti, pointed = 0;      // head and tile that are fetched next, tile that is worked on
    const auto wrap = [&](int& tile_of, int* head_of) {
        while (tile_of >= n_t) {
            tile_of -= n_t;
            if (head_of) ++*head_of;
        }
    };
    const auto fetch = [&](int slot) {
        wrap(ti, &h);
        const int i0 = (t_first + ti) * BQ, valid = nq - i0 < BQ ? nq - i0 : BQ;
        if (valid != pointed) {
            qs.point(static_cast<unsigned>(a.q_stride) * 2, valid, a.hd, wave, lane);
            gs.point(static_cast<unsigned>(go_stride) * 2, valid, a.hd, wave, lane);
            pointed = valid;
        }
        const int head = kvh * per + h;
        const unsigned to = lds0 + slot * kSlot;
        qs.issue(uniform(a.q + (q_begin + i0) * a.q_stride + static_cast<int64_t>(head) * a.hd), to, a.hd, wave);
        gs.issue(uniform(go + (q_begin + i0) * go_stride + static_cast<int64_t>(head) * a.hd), to + kTileBytes, a.hd, wave);
        if (wave < 2) {       // 64 rows' statistics, 4 bytes a lane, one kind a wavefront
            const float* from_row = stats + (wave * a.heads + head) * a.pq.T + q_begin + i0 + (lane < valid ? lane : valid - 1);
            asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, off" ::"v"(from_row), "s"(to + 2 * kTileBytes + wave * 256) : "memory");
        }
        ti += GROUPS;
    };
    // 32 queries of a tile
    const auto step = [&](int slot_index, int b, int i0) {
        const unsigned slot = lds0 + slot_index * kSlot, block = slot + b * 32 * T::kRowBytes;
        const unsigned rows = fresh(block + row_at), columns = fresh(block + column_at), st = slot + 2 * kTileBytes + b * 128 + half * 16;
        f32x16 s, dp;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const f32x4 x = *(lds_f32x4_t)static_cast<uintptr_t>(st + 32 * r), y = *(lds_f32x4_t)static_cast<uintptr_t>(st + 32 * r + BQ * 4);
#pragma unroll
            for (int i = 0; i < 4; ++i) s[4 * r + i] = x[i], dp[4 * r + i] = y[i];
        }
#pragma unroll
        for (int e = 0; e < HD / 16; ++e) s = mfma32(T::by_row(rows, e, 0), kf[e], s);
#pragma unroll
        for (int e = 0; e < HD / 16; ++e) dp = mfma32(T::by_row(rows, e, kTileBytes), vf[e], dp);
        if (i0 < from_most || i0 + 32 > nq) {       // some pair is not visible: its weight, exp2 of -inf, is 0
            stay_branch();
            const int lo = from - i0 - 4 * half, hi = nq - i0 - 4 * half;
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int i = 8 * (r >> 2) + (r & 3);
                const bool seen = i >= lo && i < hi;
                s[r] = seen ? s[r] : -INFINITY;
                dp[r] = seen ? dp[r] : 0.f;
            }
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            s[r] = __builtin_amdgcn_exp2f(s[r] * c);
            dp[r] *= s[r];
        }
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const bf16x8 p = as_fragment(s, e), ds = as_fragment(dp, e);    // both at most 2^-8 off, as in the forward pass
#pragma unroll
            for (int d = 0; d < HD / 32; ++d) {
                gv[d] = mfma32(T::by_column(columns, e, d, kTileBytes), p, gv[d]);
                gk[d] = mfma32(T::by_column(columns, e, d, 0), ds, gk[d]);
            }
        }
    };
    const int mine = (total - group + GROUPS - 1) / GROUPS;      // this group's tiles: group, group + GROUPS, ...
    clear_tiles<HD>(lds, GROUPS * 2 * kSlot, a.hd);
    if (mine > 0) fetch(0);
    tiles_ready();
    for (int t = 0; t < (total + GROUPS - 1) / GROUPS; ++t) {
        if (t + 1 < mine) fetch((t + 1) & 1);
        if (t < mine) {
            wrap(at, nullptr);
            const int i0 = (t_first + at) * BQ;
            at += GROUPS;
#pragma unroll 1
            for (int b = 0; b < 2; ++b) {
                const int i = i0 + 32 * b;
                if (own_valid == 0 || i >= nq || i + 31 < from_least) continue;
                step(t & 1, b, i);
            }
        }
        tiles_ready();
    }
    // group 1's sums by way of the LDS, a quarter of HD 128's at a time
    if constexpr (GROUPS == 2) {
        f32x16* parts = reinterpret_cast<f32x16*>(lds);
        for (int which = 0; which < 2; ++which)
#pragma unroll
            for (int d = 0; d < HD / 32; ++d) {
                f32x16& sum = which ? gv[d] : gk[d];
                if (group == 1) parts[wave * 64 + lane] = sum;
                __syncthreads();
                if (group == 0) sum += parts[wave * 64 + lane];
                __syncthreads();
            }
        if (group == 1) return;
    }
    unsigned char* own = lds + wave * 32 * T::kRowBytes;
    store_sums<HD>(gk, a.scale, own, dk, splits, split, row0, kvh, own_valid, a.hd, lane);
    store_sums<HD>(gv, 1.f, own, dv, splits, split, row0, kvh, own_valid, a.hd, lane);
}
constexpr int groups_of(int hd) { return hd > 64 ? 2 : 1; }
template <int HD, int GROUPS>
bool launch_grad_kv(const Problem& a, unsigned blocks, const uint16_t* go, const float* stats, int splits, const Sums& dk, const Sums& dv, hipStream_t st) {
    constexpr int kLds = GROUPS * 2 * (2 * 64 * Tile<HD>::kRowBytes + 512);
    static arrol_device_flags allowed;
    if (!arrol_allow_lds(attention_grad_kv_kernel<HD, GROUPS>, kLds, allowed)) return false;
    arrol_launch(attention_grad_kv_kernel<HD, GROUPS>, dim3(blocks), dim3(GROUPS * kThreads), kLds, st, a, go, stats, splits, dk, dv);
    return true;
}

// dQ: a workgroup walks over the keys in tiles of 64, a wavefront with 32 queries of a head (Q and dO as fragments in registers).
// S^T = K Q^T, dP^T = V dO^T, dQ^T += K^T dS^T.  It goes first, and leaves what the other kernel needs of a row: -lse / scale, and behind all
// of those -D, D_i = <do_i, o_i>, in fp32.
template <int HD, int HEADS>
__global__ __launch_bounds__(kThreads, 2) void attention_grad_q_kernel(Problem a, int64_t tiles, const uint16_t* __restrict__ out, const uint16_t* __restrict__ go,
                                                                       const float* __restrict__ lse, float* __restrict__ stats, int splits, Sums dq) {
    constexpr int BK = 64;
    using T = Tile<HD>;
    constexpr int kTileBytes = BK * T::kRowBytes;
    __shared__ __align__(1024) unsigned char lds[2][2][kTileBytes];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
    const int per = a.heads / a.kv_heads, head_blocks = per / HEADS;
    int kvh, rest;
    split_block(blockIdx.x, a.kv_heads, kvh, rest);
    const int first_head = kvh * per + rest % head_blocks * HEADS;
    rest /= head_blocks;
    const int split = rest % splits;
    QueryBlock<HEADS> w;
    if (!w.find(a, tiles - 1 - rest / splits, first_head, wave, lane)) return;
    const int head = w.head, all = (w.reach + BK - 1) / BK, t_lo = all * split / splits,
              n_tiles = all * (split + 1) / splits - t_lo;

    const int64_t go_stride = static_cast<int64_t>(a.heads) * a.hd;
    bf16x8 qf[HD / 16], gf[HD / 16];
    load_own<HD>(qf, a.q + w.row0 * a.q_stride + static_cast<int64_t>(head) * a.hd, a.q_stride, w.own_valid, a.hd, lane);
    load_own<HD>(gf, go + w.row0 * go_stride + static_cast<int64_t>(head) * a.hd, go_stride, w.own_valid, a.hd, lane);
    float mine[2] = {0.f, 0.f};
    {
        bf16x8 of[HD / 16];
        load_own<HD>(of, out + w.row0 * go_stride + static_cast<int64_t>(head) * a.hd, go_stride, w.own_valid, a.hd, lane);
        float dot = 0.f;
#pragma unroll
        for (int s = 0; s < HD / 16; ++s)
#pragma unroll
            for (int e = 0; e < 8; ++e) dot = fmaf(static_cast<float>(of[s][e]), static_cast<float>(gf[s][e]), dot);
        mine[1] = -half_sum(dot);
        if ((lane & 31) < w.own_valid) {
            const int64_t at = static_cast<int64_t>(head) * a.pq.T + w.row0 + (lane & 31);
            mine[0] = -lse[at] / a.scale;
            if (split == 0) stats[half ? static_cast<int64_t>(a.heads) * a.pq.T + at : at] = mine[half];
        }
    }
    const uint16_t* kp = uniform(a.k + (w.k_begin + static_cast<int64_t>(t_lo) * BK) * a.k_stride + static_cast<int64_t>(kvh) * a.hd);
    const uint16_t* vp = uniform(a.v + (w.k_begin + static_cast<int64_t>(t_lo) * BK) * a.v_stride + static_cast<int64_t>(kvh) * a.hd);
    f32x16 gq[HD / 32];
#pragma unroll
    for (int d = 0; d < HD / 32; ++d) gq[d] = 0.f;
    const float c = a.scale * kLog2e;

    Stream<HD, BK, kWaves> ks, vs;
    const int keys = w.nk - t_lo * BK, whole = keys / BK;
    const auto point = [&](int valid) {
        ks.point(static_cast<unsigned>(a.k_stride) * 2, valid, a.hd, wave, lane);
        vs.point(static_cast<unsigned>(a.v_stride) * 2, valid, a.hd, wave, lane);
    };
    const unsigned lds0 = lds_address(lds), row_at = T::row_base(lane), column_at = T::column_base(lane);
    const auto fetch = [&](int t) {
        if (t == whole) point(keys - t * BK);
        const unsigned to = lds0 + (t & 1) * 2 * kTileBytes;
        ks.issue(kp, to, a.hd, wave);
        vs.issue(vp, to + kTileBytes, a.hd, wave);
        kp += BK * a.k_stride;
        vp += BK * a.v_stride;
    };
    const auto step = [&](int t, int b, int j0) {
        const unsigned block = lds0 + (t & 1) * 2 * kTileBytes + b * 32 * T::kRowBytes, rows = fresh(block + row_at), columns = fresh(block + column_at);
        f32x16 s, dp;
        s = mine[0];
        dp = mine[1];
#pragma unroll
        for (int e = 0; e < HD / 16; ++e) s = mfma32(T::by_row(rows, e, 0), qf[e], s);
#pragma unroll
        for (int e = 0; e < HD / 16; ++e) dp = mfma32(T::by_row(rows, e, kTileBytes), gf[e], dp);
        if (j0 + 32 > w.sees_least) {       // some row does not see all of the keys
            stay_branch();
            const int limit = w.sees - j0 - 4 * half;
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const bool seen = 8 * (r >> 2) + (r & 3) < limit;
                s[r] = seen ? s[r] : -INFINITY;
                dp[r] = seen ? dp[r] : 0.f;
            }
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) dp[r] *= __builtin_amdgcn_exp2f(s[r] * c);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const bf16x8 ds = as_fragment(dp, e);
#pragma unroll
            for (int d = 0; d < HD / 32; ++d) gq[d] = mfma32(T::by_column(columns, e, d, 0), ds, gq[d]);
        }
    };
    clear_tiles<HD>(&lds[0][0][0], sizeof lds, a.hd);
    if (n_tiles > 0) {
        point(BK);
        fetch(0);
    }
    tiles_ready();
    for (int t = 0; t < n_tiles; ++t) {
        if (t + 1 < n_tiles) fetch(t + 1);
#pragma unroll 1
        for (int b = 0; b < 2; ++b) {
            const int j = (t_lo + t) * BK + 32 * b;
            if (j < w.sees_most) step(t, b, j);
        }
        tiles_ready();
    }
    store_sums<HD>(gq, a.scale, &lds[0][0][0] + wave * 32 * T::kRowBytes, dq, splits, split, w.row0, head, w.own_valid, a.hd, lane);
}

bool row_stride_ok(int64_t stride, int64_t rows, int heads, int hd) {
    return stride % 8 == 0 && stride >= static_cast<int64_t>(heads) * hd && stride <= (int64_t{1} << 24) && rows <= (int64_t{1} << 30);
}

// ARROL_OK, or what is wrong with the arguments that both calls share
int check(const Problem& a, int64_t T_q, int64_t T_k) {
    if (T_q < 0 || T_k < 0 || a.pq.n < 0 || a.heads < 1 || a.kv_heads < 1 || a.heads % a.kv_heads || a.heads > 65536 || a.hd < 8 || a.hd > 128 || a.hd % 8) return ARROL_EINVAL;
    if (!(a.scale > 0.f) || a.scale > 3e38f) return ARROL_EINVAL;
    if (a.pk.cu == a.pq.cu && T_q != T_k) return ARROL_EINVAL;      // the keys' offsets are the queries'
    if (!row_stride_ok(a.q_stride, T_q, a.heads, a.hd) || !row_stride_ok(a.k_stride, T_k, a.kv_heads, a.hd) || !row_stride_ok(a.v_stride, T_k, a.kv_heads, a.hd)) return ARROL_EINVAL;
    if (T_q > 0 && (!a.q || !arrol_aligned16(a.q) || !a.pq.cu || !a.pk.cu)) return ARROL_EINVAL;
    if (T_k > 0 && (!a.k || !a.v || !arrol_aligned16(a.k) || !arrol_aligned16(a.v) || !a.pq.cu || !a.pk.cu)) return ARROL_EINVAL;
    const int64_t most = T_q > T_k ? T_q : T_k;
    if (tile_bound(most, a.pq.n, kOwn) * a.heads >= (1 << 24)) return ARROL_EINVAL;      // lanes of a launch are counted in 32 bits
    return ARROL_OK;
}

Problem problem(const void* q, int64_t q_stride, const void* k, int64_t k_stride, const void* v, int64_t v_stride, const int64_t* cu_q, const int64_t* cu_k,
                int64_t T_q, int64_t T_k, int n_seq, int heads, int kv_heads, int hd, int causal, float scale) {
    Problem a;
    a.q = static_cast<const uint16_t*>(q), a.k = static_cast<const uint16_t*>(k), a.v = static_cast<const uint16_t*>(v);
    a.q_stride = q_stride, a.k_stride = k_stride, a.v_stride = v_stride;
    a.pq = {cu_q, T_q, n_seq}, a.pk = {cu_k ? cu_k : cu_q, T_k, n_seq};
    a.heads = heads, a.kv_heads = kv_heads, a.hd = hd, a.causal = causal != 0, a.scale = scale;
    return a;
}

// Heads of a kv head that a workgroup takes.
int heads_together(int per) { return per % 4 == 0 ? 4 : per % 2 == 0 ? 2 : 1; }
int64_t query_tiles(int64_t T, int n_seq, int per) { return tile_bound(T, n_seq, kOwn / heads_together(per)); }

template <int HD>
void launch_forward(const Problem& a, const Output& to, hipStream_t st) {
    const int per = a.heads / a.kv_heads, together = heads_together(per);
    const int64_t tiles = query_tiles(a.pq.T, a.pq.n, per);
    const dim3 grid(static_cast<unsigned>(tiles * (a.heads / together) * to.splits));
    if (together == 4) arrol_launch(attention_forward_kernel<HD, 4>, grid, dim3(kThreads), 0, st, a, tiles, to);
    else if (together == 2) arrol_launch(attention_forward_kernel<HD, 2>, grid, dim3(kThreads), 0, st, a, tiles, to);
    else arrol_launch(attention_forward_kernel<HD, 1>, grid, dim3(kThreads), 0, st, a, tiles, to);
}
template <int HD>
void launch_grad_q(const Problem& a, const uint16_t* out, const uint16_t* go, const float* lse, float* stats, int splits, const Sums& dq, hipStream_t st) {
    const int per = a.heads / a.kv_heads, together = heads_together(per);
    const int64_t tiles = query_tiles(a.pq.T, a.pq.n, per);
    const dim3 grid(static_cast<unsigned>(tiles * (a.heads / together) * splits));
    if (together == 4) arrol_launch(attention_grad_q_kernel<HD, 4>, grid, dim3(kThreads), 0, st, a, tiles, out, go, lse, stats, splits, dq);
    else if (together == 2) arrol_launch(attention_grad_q_kernel<HD, 2>, grid, dim3(kThreads), 0, st, a, tiles, out, go, lse, stats, splits, dq);
    else arrol_launch(attention_grad_q_kernel<HD, 1>, grid, dim3(kThreads), 0, st, a, tiles, out, go, lse, stats, splits, dq);
}

// Ranges that the keys of a sequence are cut into: enough for 1,024 workgroups, as long as a range keeps 256 keys of an average sequence.
int key_splits(int64_t T_q, int64_t T_k, int n_seq, int heads) {
    const int64_t blocks = (T_q / kOwn + n_seq) * heads, by_work = (1024 + blocks - 1) / (blocks > 0 ? blocks : 1), by_keys = n_seq > 0 ? T_k / n_seq / 256 : 1;
    const int64_t s = by_work < by_keys ? by_work : by_keys;
    return static_cast<int>(s < 1 ? 1 : s < 16 ? s : 16);
}
// Ranges of the gradient's walks, in the same manner: dQ's over the keys, dK/dV's over the queries of all heads that share a kv head.
struct GradPlan {
    int q_splits, kv_splits;
    size_t stats, q, kv;            // floats
};
GradPlan grad_plan(int64_t T_q, int64_t T_k, int n_seq, int heads, int kv_heads, int hd) {
    const auto cut = [](int64_t blocks, int64_t enough, int64_t steps) {       // a range keeps 2 tiles of 64 rows of an average sequence
        const int64_t by_work = enough / (blocks > 0 ? blocks : 1), s = by_work < steps / 2 ? by_work : steps / 2;
        return static_cast<int>(s < 1 ? 1 : s < 16 ? s : 16);
    };
    const int64_t per = heads / kv_heads, seqs = n_seq > 0 ? n_seq : 1;
    GradPlan p;
    p.q_splits = cut((T_q / kOwn + n_seq) * heads, 512, T_k / seqs / 64);
    p.kv_splits = cut((T_k / kOwn + n_seq) * kv_heads, 512, T_q / seqs / 64 * per);
    p.stats = static_cast<size_t>(T_q) * heads * 2;
    p.q = p.q_splits > 1 ? static_cast<size_t>(p.q_splits) * T_q * heads * hd : 0;
    p.kv = p.kv_splits > 1 ? static_cast<size_t>(p.kv_splits) * T_k * kv_heads * hd : 0;
    return p;
}
// Partial sums begin on 16 bytes behind the statistics.
size_t up4(size_t floats) { return (floats + 3) / 4 * 4; }
size_t part_bytes(int64_t T, int heads, int hd, int splits) { return splits == 1 ? 0 : static_cast<size_t>(splits) * T * heads * (hd + 2) * sizeof(float); }
}  // namespace

extern "C" size_t arrol_attention_workspace_bytes(int64_t T_q, int64_t T_k, int32_t n_seq, int32_t n_heads, int32_t head_dim) {
    if (T_q <= 0 || T_k < 0 || n_seq < 0 || n_heads < 1 || head_dim < 8 || head_dim > 128) return 0;
    return part_bytes(T_q, n_heads, head_dim, key_splits(T_q, T_k, n_seq, n_heads));
}

extern "C" int arrol_attention(const void* q, int64_t q_stride, const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                               const int64_t* cu_seqlens_q, const int64_t* cu_seqlens_k, int64_t T_q, int64_t T_k, int32_t n_seq,
                               int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, int32_t causal, float scale, void* out,
                               float* lse_out, void* workspace, size_t workspace_bytes, void* stream) {
    const Problem a = problem(q, q_stride, k, k_stride, v, v_stride, cu_seqlens_q, cu_seqlens_k, T_q, T_k, n_seq, n_heads, n_kv_heads, head_dim, causal, scale);
    if (const int rc = check(a, T_q, T_k)) return rc;
    if (T_q == 0) return ARROL_OK;
    if (!out || !arrol_aligned16(out) || (workspace && !arrol_aligned16(workspace))) return ARROL_EINVAL;
    const int64_t rows = T_q * n_heads;
    int splits = key_splits(T_q, T_k, n_seq, n_heads);
    if (!workspace || workspace_bytes < part_bytes(T_q, n_heads, head_dim, splits)) splits = 1;
    auto* ws = static_cast<float*>(workspace);
    const Output to = {static_cast<uint16_t*>(out), lse_out, splits, ws, splits > 1 ? ws + static_cast<size_t>(splits) * rows * head_dim : nullptr};
    const auto st = static_cast<hipStream_t>(stream);
    if (head_dim <= 64) launch_forward<64>(a, to, st);
    else launch_forward<128>(a, to, st);
    if (splits > 1) arrol_launch(attention_join_kernel, dim3(static_cast<unsigned>((rows + 15) / 16)), dim3(kThreads), 0, st, to, T_q, n_heads, head_dim);
    return arrol_launch_status();
}

extern "C" size_t arrol_attention_grad_workspace_bytes(int64_t T_q, int64_t T_k, int32_t n_seq, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim) {
    if (T_q < 0 || T_k < 0 || n_seq < 0 || n_heads < 1 || n_kv_heads < 1 || n_heads % n_kv_heads || head_dim < 8 || head_dim > 128) return 0;
    const GradPlan p = grad_plan(T_q, T_k, n_seq, n_heads, n_kv_heads, head_dim);
    return (up4(p.stats) + p.q + 2 * p.kv) * sizeof(float);
}

extern "C" int arrol_attention_grad(const void* q, int64_t q_stride, const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                                    const void* out, const float* lse, const void* grad_out, const int64_t* cu_seqlens_q,
                                    const int64_t* cu_seqlens_k, int64_t T_q, int64_t T_k, int32_t n_seq, int32_t n_heads,
                                    int32_t n_kv_heads, int32_t head_dim, int32_t causal, float scale, void* grad_q, void* grad_k,
                                    void* grad_v, void* workspace, size_t workspace_bytes, void* stream) {
    const Problem a = problem(q, q_stride, k, k_stride, v, v_stride, cu_seqlens_q, cu_seqlens_k, T_q, T_k, n_seq, n_heads, n_kv_heads, head_dim, causal, scale);
    if (const int rc = check(a, T_q, T_k)) return rc;
    if (T_q > 0 && (!out || !lse || !grad_out || !grad_q || !arrol_aligned16(out) || !arrol_aligned16(grad_out) || !arrol_aligned16(grad_q))) return ARROL_EINVAL;
    if (T_k > 0 && (!grad_k || !grad_v || !arrol_aligned16(grad_k) || !arrol_aligned16(grad_v))) return ARROL_EINVAL;
    const GradPlan p = grad_plan(T_q, T_k, n_seq, n_heads, n_kv_heads, head_dim);
    const int64_t kv_blocks = tile_bound(T_k, n_seq, kOwn) * n_kv_heads * p.kv_splits;
    if (kv_blocks * groups_of(head_dim) >= (1 << 24)) return ARROL_EINVAL;      // as in check(), of a workgroup's 256 or 512 lanes
    const size_t need = (up4(p.stats) + p.q + 2 * p.kv) * sizeof(float);
    if (need > 0 && (!workspace || !arrol_aligned16(workspace) || workspace_bytes < need)) return ARROL_EWORKSPACE;
    const auto st = static_cast<hipStream_t>(stream);
    const auto* go = static_cast<const uint16_t*>(grad_out);
    auto* stats = static_cast<float*>(workspace);
    const Sums dq = {static_cast<uint16_t*>(grad_q), p.q ? stats + up4(p.stats) : nullptr, T_q, n_heads};
    const Sums dk = {static_cast<uint16_t*>(grad_k), p.kv ? stats + up4(p.stats) + p.q : nullptr, T_k, n_kv_heads};
    const Sums dv = {static_cast<uint16_t*>(grad_v), p.kv ? stats + up4(p.stats) + p.q + p.kv : nullptr, T_k, n_kv_heads};
    const auto join = [&](const Sums& to, int splits) {
        const int64_t n = to.T * to.heads * head_dim;
        if (splits > 1) arrol_launch(attention_grad_join_kernel, dim3(static_cast<unsigned>((n / 8 + kThreads - 1) / kThreads)), dim3(kThreads), 0, st, to.part, n, splits, to.out);
    };
    if (T_q > 0) {
        const auto* o = static_cast<const uint16_t*>(out);
        if (head_dim <= 64) launch_grad_q<64>(a, o, go, lse, stats, p.q_splits, dq, st);
        else launch_grad_q<128>(a, o, go, lse, stats, p.q_splits, dq, st);
        join(dq, p.q_splits);
    }
    if (T_k > 0) {
        const auto blocks = static_cast<unsigned>(kv_blocks);
        const bool ok = head_dim > 64 ? launch_grad_kv<128, groups_of(128)>(a, blocks, go, stats, p.kv_splits, dk, dv, st)
                                      : launch_grad_kv<64, groups_of(64)>(a, blocks, go, stats, p.kv_splits, dk, dv, st);
        if (!ok) {
            arrol_launch_status();
            return ARROL_EHIP;
        }
        join(dk, p.kv_splits);
        join(dv, p.kv_splits);
    }
    return arrol_launch_status();
}
