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
constexpr int64_t kDotBlocks = 1 << 20;

struct Problem {
    const uint16_t *q, *k, *v;
    int64_t q_stride, k_stride, v_stride;   // elements between rows
    Packed pq, pk;
    int heads, kv_heads, hd, causal;
    float scale;
};

// What a workgroup works on: tiles of the packed rows x heads.  Consecutive workgroups take consecutive kv heads (with 8 of
// them an XCD's L2 sees one kv head), then the query heads that share it, and tiles from the last one down where late ones are long.
__device__ __forceinline__ void split_block(unsigned block, int kv_heads, int& kvh, int64_t& rest) {
    kvh = static_cast<int>(block % static_cast<unsigned>(kv_heads));
    rest = block / static_cast<unsigned>(kv_heads);
}

// Forward pass: a workgroup takes 128 queries of a head, a wavefront 32 of them, and walks over the keys in tiles of 64.
// S^T = K Q^T and O^T += V^T P^T, so that a query's statistics are its lane's.
template <int HD>
__global__ __launch_bounds__(kThreads, 2) void attention_forward_kernel(Problem a, int64_t tiles, uint16_t* __restrict__ out, float* __restrict__ lse_out) {
    constexpr int BK = 64;
    using T = Tile<HD>;
    __shared__ __align__(16) unsigned char lds[2][2][BK * T::kRowBytes];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
    const int per = a.heads / a.kv_heads;
    int kvh;
    int64_t rest;
    split_block(blockIdx.x, a.kv_heads, kvh, rest);
    const int head = kvh * per + static_cast<int>(rest % per);
    const int64_t tile = tiles - 1 - rest / per;
    int segment;
    int64_t first, end;
    if (!find_tile<kOwn>(a.pq, tile, lane, segment, first, end)) return;
    const int64_t q_begin = a.pq.bound(segment);
    int64_t k_begin = 0, nk = 0;
    if (segment >= 1 && segment <= a.pq.n) {       // rows of no sequence see no keys: zeros
        k_begin = a.pk.bound(segment);
        nk = a.pk.bound(segment + 1) - k_begin;
        if (nk < 0) nk = 0;
    }
    const int64_t nq = end - q_begin;
    // query at offset i of its sequence sees keys j < min(nk, i + 1 + nk - nq)
    const int64_t shift = a.causal ? nk - nq : nk;
    const int64_t row0 = first + 32 * wave;           // this wavefront's first row
    const int own_valid = static_cast<int>(end - row0 < 32 ? (end - row0 < 0 ? 0 : end - row0) : 32);
    const int64_t my_i = row0 - q_begin + (lane & 31);
    int64_t sees = a.causal ? my_i + 1 + shift : nk;
    sees = sees < 0 ? 0 : sees < nk ? sees : nk;
    // keys that any of the workgroup's rows, and any / all of the wavefront's rows see
    const int64_t last_i = (end - first < kOwn ? end - first : kOwn) - 1 + first - q_begin;
    int64_t reach = a.causal ? last_i + 1 + shift : nk;
    reach = reach < 0 ? 0 : reach < nk ? reach : nk;
    const int n_tiles = static_cast<int>((reach + BK - 1) / BK);

    bf16x8 qf[HD / 16];
    load_own<HD>(qf, a.q + row0 * a.q_stride + static_cast<int64_t>(head) * a.hd, a.q_stride, own_valid, a.hd, lane);
    const uint16_t* kp = a.k + k_begin * a.k_stride + static_cast<int64_t>(kvh) * a.hd;
    const uint16_t* vp = a.v + k_begin * a.v_stride + static_cast<int64_t>(kvh) * a.hd;

    f32x16 o[HD / 32];
#pragma unroll
    for (int d = 0; d < HD / 32; ++d) o[d] = 0.f;
    float m = -INFINITY, l = 0.f;                 // of z * log2 e; l is this lane's half of the row
    const float c = a.scale * kLog2e;

    Staged<HD, BK, kThreads> ks, vs;
    const auto fetch = [&](int t) {
        const int64_t j0 = static_cast<int64_t>(t) * BK;
        const int valid = static_cast<int>(nk - j0 < BK ? nk - j0 : BK);
        ks.load(kp + j0 * a.k_stride, a.k_stride, valid, a.hd);
        vs.load(vp + j0 * a.v_stride, a.v_stride, valid, a.hd);
    };
    if (n_tiles > 0) {
        fetch(0);
        ks.store(lds[0][0]);
        vs.store(lds[0][1]);
    }
    __syncthreads();
    for (int t = 0; t < n_tiles; ++t) {
        const int cur = t & 1;
        if (t + 1 < n_tiles) fetch(t + 1);
        const unsigned char *kt = lds[cur][0], *vt = lds[cur][1];
        f32x16 s[BK / 32];
#pragma unroll
        for (int b = 0; b < BK / 32; ++b) {
            s[b] = 0.f;
#pragma unroll
            for (int e = 0; e < HD / 16; ++e) s[b] = mfma32(T::by_row(kt, 32 * b + (lane & 31), e, half), qf[e], s[b]);
        }
        const int64_t j0 = static_cast<int64_t>(t) * BK;
        float top = -INFINITY;
#pragma unroll
        for (int b = 0; b < BK / 32; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int64_t j = j0 + 32 * b + 8 * (r >> 2) + 4 * half + (r & 3);
                s[b][r] = j < sees ? s[b][r] * c : -INFINITY;
                top = fmaxf(top, s[b][r]);
            }
        top = half_max(top);
        // the sums are moved to a new maximum only where it has grown by 2^8: exp2 then stays below 256 and nothing is lost
        if (__any(top > m + 8.f)) {
            const float to = fmaxf(m, top);
            const float f = to == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - to);
            m = to;
            l *= f;
#pragma unroll
            for (int d = 0; d < HD / 32; ++d) o[d] *= f;
        }
        const float base = m == -INFINITY ? 0.f : m;
#pragma unroll
        for (int b = 0; b < BK / 32; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                s[b][r] = __builtin_amdgcn_exp2f(s[b][r] - base);
                l += s[b][r];
            }
#pragma unroll
        for (int b = 0; b < BK / 32; ++b)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const bf16x8 p = as_fragment(s[b], e);      // weights in bf16: at most 2^-9 off each, their sum l is of the unrounded ones
#pragma unroll
                for (int d = 0; d < HD / 32; ++d) o[d] = mfma32(T::by_column(vt, 2 * b + e, d, lane), p, o[d]);
            }
        if (t + 1 < n_tiles) {
            ks.store(lds[cur ^ 1][0]);
            vs.store(lds[cur ^ 1][1]);
        }
        __syncthreads();
    }
    l = half_sum(l);
    store_own<HD>(o, l == 0.f ? 0.f : 1.f / l, out + (row0 * a.heads + head) * a.hd, static_cast<int64_t>(a.heads) * a.hd, own_valid, a.hd, lane);
    if (lse_out && lane < own_valid && lane < 32)
        lse_out[static_cast<int64_t>(head) * a.pq.T + row0 + lane] = l == 0.f ? -INFINITY : m * kLn2 + logf(l);
}

// D_i = <do_i, o_i> in fp32: a group of 16 lanes takes a row of a head, 8 elements a lane.
__global__ __launch_bounds__(256) void attention_row_dot_kernel(const uint16_t* __restrict__ o, const uint16_t* __restrict__ go, int64_t rows, int64_t T, int heads,
                                                               int hd, float* __restrict__ dot) {
    const int e = (threadIdx.x & 15) * 8;
    for (int64_t base = static_cast<int64_t>(blockIdx.x) * 16; base < rows; base += static_cast<int64_t>(gridDim.x) * 16) {
        const int64_t row = base + (threadIdx.x >> 4);       // token * heads + head
        float sum = 0.f;
        if (row < rows && e < hd) {
            const u32x4 x = *reinterpret_cast<const u32x4*>(o + row * hd + e), y = *reinterpret_cast<const u32x4*>(go + row * hd + e);
#pragma unroll
            for (int i = 0; i < 4; ++i) sum += bf16_lo(x[i]) * bf16_lo(y[i]) + bf16_hi(x[i]) * bf16_hi(y[i]);
        }
        const auto add = [](float u, float w) { return u + w; };
        sum = wave_step<1>(wave_step<2>(wave_step<4>(wave_step<8>(sum, add), add), add), add);
        if (row < rows && (threadIdx.x & 15) == 0) dot[(row % heads) * T + row / heads] = sum;
    }
}

// dK and dV: a workgroup takes 128 keys of a kv head, a wavefront 32 of them (K and V as fragments in registers), and walks over the
// queries of every head that reads them, 32 at a time: the sum over the shared heads is made in registers, in a fixed order.
// S = Q K^T and dP = dO V^T have the own key as column; dV^T += dO^T P and dK^T += Q^T dS.
template <int HD>
__global__ __launch_bounds__(kThreads, 2) void attention_grad_kv_kernel(Problem a, const uint16_t* __restrict__ go, const float* __restrict__ lse,
                                                                        const float* __restrict__ dot, uint16_t* __restrict__ dk, uint16_t* __restrict__ dv) {
    constexpr int BQ = 32;
    using T = Tile<HD>;
    __shared__ __align__(16) unsigned char lds[2][2][BQ * T::kRowBytes];
    __shared__ __align__(16) float stats[2][2][BQ];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
    const int per = a.heads / a.kv_heads;
    int kvh;
    int64_t tile;
    split_block(blockIdx.x, a.kv_heads, kvh, tile);
    int segment;
    int64_t first, end;
    if (!find_tile<kOwn>(a.pk, tile, lane, segment, first, end)) return;
    const int64_t k_begin = a.pk.bound(segment), nk = end - k_begin;
    int64_t q_begin = 0, nq = 0;
    if (segment >= 1 && segment <= a.pk.n) {
        q_begin = a.pq.bound(segment);
        nq = a.pq.bound(segment + 1) - q_begin;
        if (nq < 0) nq = 0;
    }
    const int64_t row0 = first + 32 * wave;
    const int own_valid = static_cast<int>(end - row0 < 32 ? (end - row0 < 0 ? 0 : end - row0) : 32);
    const int64_t my_j = row0 - k_begin + (lane & 31);
    // key j is seen by queries i >= j + nq - nk (causal)
    int64_t from = a.causal ? my_j + nq - nk : 0;
    from = from < 0 ? 0 : from;
    int64_t i_first = a.causal ? first - k_begin + nq - nk : 0;
    i_first = i_first < 0 ? 0 : i_first;
    const int64_t t_first = i_first / BQ;
    int64_t n_t = (nq + BQ - 1) / BQ - t_first;
    n_t = n_t < 0 ? 0 : n_t;
    const int total = static_cast<int>(n_t) * per;

    bf16x8 kf[HD / 16], vf[HD / 16];
    load_own<HD>(kf, a.k + row0 * a.k_stride + static_cast<int64_t>(kvh) * a.hd, a.k_stride, own_valid, a.hd, lane);
    load_own<HD>(vf, a.v + row0 * a.v_stride + static_cast<int64_t>(kvh) * a.hd, a.v_stride, own_valid, a.hd, lane);
    f32x16 gk[HD / 32], gv[HD / 32];
#pragma unroll
    for (int d = 0; d < HD / 32; ++d) gk[d] = 0.f, gv[d] = 0.f;
    const float c = a.scale * kLog2e;
    const int64_t go_stride = static_cast<int64_t>(a.heads) * a.hd;

    Staged<HD, BQ, kThreads> qs, gs;
    float stat = 0.f;
    int h = 0;
    int64_t ti = t_first;                             // what is fetched next
    const auto fetch = [&]() {
        const int64_t i0 = ti * BQ;
        const int head = kvh * per + h;
        const int valid = static_cast<int>(nq - i0 < BQ ? nq - i0 : BQ);
        qs.load(a.q + (q_begin + i0) * a.q_stride + static_cast<int64_t>(head) * a.hd, a.q_stride, valid, a.hd);
        gs.load(go + (q_begin + i0) * go_stride + static_cast<int64_t>(head) * a.hd, go_stride, valid, a.hd);
        if (threadIdx.x < 2 * BQ) {
            const int r = threadIdx.x & (BQ - 1);
            const float* from_array = threadIdx.x < BQ ? lse : dot;
            stat = r < valid ? from_array[static_cast<int64_t>(head) * a.pq.T + q_begin + i0 + r] : 0.f;
            if (threadIdx.x < BQ) stat *= kLog2e;
        }
    };
    const auto put = [&](int b) {
        qs.store(lds[b][0]);
        gs.store(lds[b][1]);
        if (threadIdx.x < 2 * BQ) stats[b][threadIdx.x / BQ][threadIdx.x & (BQ - 1)] = stat;
    };
    const auto next = [&]() {
        if (++ti == t_first + n_t) ti = t_first, ++h;
    };
    if (total > 0) {
        fetch();
        put(0);
    }
    __syncthreads();
    for (int t = 0; t < total; ++t) {
        const int cur = t & 1;
        const int64_t i0 = ti * BQ;
        next();
        if (t + 1 < total) fetch();
        const unsigned char *qt = lds[cur][0], *gt = lds[cur][1];
        f32x16 s, dp;
        s = 0.f;
        dp = 0.f;
#pragma unroll
        for (int e = 0; e < HD / 16; ++e) s = mfma32(T::by_row(qt, lane & 31, e, half), kf[e], s);
#pragma unroll
        for (int e = 0; e < HD / 16; ++e) dp = mfma32(T::by_row(gt, lane & 31, e, half), vf[e], dp);
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            const f32x4 ls = *reinterpret_cast<const f32x4*>(&stats[cur][0][8 * b + 4 * half]);
            const f32x4 ds = *reinterpret_cast<const f32x4*>(&stats[cur][1][8 * b + 4 * half]);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int64_t i = i0 + 8 * b + 4 * half + r;
                const bool seen = i >= from && i < nq;
                const float p = seen ? __builtin_amdgcn_exp2f(s[4 * b + r] * c - ls[r]) : 0.f;
                dp[4 * b + r] = seen ? p * (dp[4 * b + r] - ds[r]) : 0.f;
                s[4 * b + r] = p;
            }
        }
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const bf16x8 p = as_fragment(s, e), ds = as_fragment(dp, e);    // both at most 2^-9 off, as in the forward pass
#pragma unroll
            for (int d = 0; d < HD / 32; ++d) {
                gv[d] = mfma32(T::by_column(gt, e, d, lane), p, gv[d]);
                gk[d] = mfma32(T::by_column(qt, e, d, lane), ds, gk[d]);
            }
        }
        if (t + 1 < total) put(cur ^ 1);
        __syncthreads();
    }
    const int64_t out_stride = static_cast<int64_t>(a.kv_heads) * a.hd, at = row0 * out_stride + static_cast<int64_t>(kvh) * a.hd;
    store_own<HD>(gk, a.scale, dk + at, out_stride, own_valid, a.hd, lane);
    store_own<HD>(gv, 1.f, dv + at, out_stride, own_valid, a.hd, lane);
}

// dQ: a workgroup takes 128 queries of a head (Q and dO as fragments in registers) and walks over the keys, 32 at a time.
// S^T = K Q^T, dP^T = V dO^T, dQ^T += K^T dS^T.
template <int HD>
__global__ __launch_bounds__(kThreads, 2) void attention_grad_q_kernel(Problem a, int64_t tiles, const uint16_t* __restrict__ go, const float* __restrict__ lse,
                                                                       const float* __restrict__ dot, uint16_t* __restrict__ dq) {
    constexpr int BK = 32;
    using T = Tile<HD>;
    __shared__ __align__(16) unsigned char lds[2][2][BK * T::kRowBytes];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
    const int per = a.heads / a.kv_heads;
    int kvh;
    int64_t rest;
    split_block(blockIdx.x, a.kv_heads, kvh, rest);
    const int head = kvh * per + static_cast<int>(rest % per);
    const int64_t tile = tiles - 1 - rest / per;
    int segment;
    int64_t first, end;
    if (!find_tile<kOwn>(a.pq, tile, lane, segment, first, end)) return;
    const int64_t q_begin = a.pq.bound(segment), nq = end - q_begin;
    int64_t k_begin = 0, nk = 0;
    if (segment >= 1 && segment <= a.pq.n) {
        k_begin = a.pk.bound(segment);
        nk = a.pk.bound(segment + 1) - k_begin;
        if (nk < 0) nk = 0;
    }
    const int64_t row0 = first + 32 * wave;
    const int own_valid = static_cast<int>(end - row0 < 32 ? (end - row0 < 0 ? 0 : end - row0) : 32);
    int64_t sees = a.causal ? row0 - q_begin + (lane & 31) + 1 + nk - nq : nk;
    sees = sees < 0 ? 0 : sees < nk ? sees : nk;
    const int64_t last_i = (end - first < kOwn ? end - first : kOwn) - 1 + first - q_begin;
    int64_t reach = a.causal ? last_i + 1 + nk - nq : nk;
    reach = reach < 0 ? 0 : reach < nk ? reach : nk;
    const int n_tiles = static_cast<int>((reach + BK - 1) / BK);

    const int64_t go_stride = static_cast<int64_t>(a.heads) * a.hd;
    bf16x8 qf[HD / 16], gf[HD / 16];
    load_own<HD>(qf, a.q + row0 * a.q_stride + static_cast<int64_t>(head) * a.hd, a.q_stride, own_valid, a.hd, lane);
    load_own<HD>(gf, go + row0 * go_stride + static_cast<int64_t>(head) * a.hd, go_stride, own_valid, a.hd, lane);
    float my_lse = 0.f, my_dot = 0.f;
    if ((lane & 31) < own_valid) {
        const int64_t at = static_cast<int64_t>(head) * a.pq.T + row0 + (lane & 31);
        my_lse = lse[at] * kLog2e;
        my_dot = dot[at];
    }
    const uint16_t* kp = a.k + k_begin * a.k_stride + static_cast<int64_t>(kvh) * a.hd;
    const uint16_t* vp = a.v + k_begin * a.v_stride + static_cast<int64_t>(kvh) * a.hd;
    f32x16 gq[HD / 32];
#pragma unroll
    for (int d = 0; d < HD / 32; ++d) gq[d] = 0.f;
    const float c = a.scale * kLog2e;
    Staged<HD, BK, kThreads> ks, vs;
    const auto fetch = [&](int t) {
        const int64_t j0 = static_cast<int64_t>(t) * BK;
        const int valid = static_cast<int>(nk - j0 < BK ? nk - j0 : BK);
        ks.load(kp + j0 * a.k_stride, a.k_stride, valid, a.hd);
        vs.load(vp + j0 * a.v_stride, a.v_stride, valid, a.hd);
    };
    if (n_tiles > 0) {
        fetch(0);
        ks.store(lds[0][0]);
        vs.store(lds[0][1]);
    }
    __syncthreads();
    for (int t = 0; t < n_tiles; ++t) {
        const int cur = t & 1;
        if (t + 1 < n_tiles) fetch(t + 1);
        const unsigned char *kt = lds[cur][0], *vt = lds[cur][1];
        f32x16 s, dp;
        s = 0.f;
        dp = 0.f;
#pragma unroll
        for (int e = 0; e < HD / 16; ++e) s = mfma32(T::by_row(kt, lane & 31, e, half), qf[e], s);
#pragma unroll
        for (int e = 0; e < HD / 16; ++e) dp = mfma32(T::by_row(vt, lane & 31, e, half), gf[e], dp);
        const int64_t j0 = static_cast<int64_t>(t) * BK;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int64_t j = j0 + 8 * (r >> 2) + 4 * half + (r & 3);
            dp[r] = j < sees ? __builtin_amdgcn_exp2f(s[r] * c - my_lse) * (dp[r] - my_dot) : 0.f;
        }
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const bf16x8 ds = as_fragment(dp, e);
#pragma unroll
            for (int d = 0; d < HD / 32; ++d) gq[d] = mfma32(T::by_column(kt, e, d, lane), ds, gq[d]);
        }
        if (t + 1 < n_tiles) {
            ks.store(lds[cur ^ 1][0]);
            vs.store(lds[cur ^ 1][1]);
        }
        __syncthreads();
    }
    store_own<HD>(gq, a.scale, dq + (row0 * a.heads + head) * a.hd, go_stride, own_valid, a.hd, lane);
}

bool row_stride_ok(int64_t stride, int64_t rows, int heads, int hd) {
    return stride % 8 == 0 && stride >= static_cast<int64_t>(heads) * hd && stride <= (int64_t{1} << 31) && rows <= (int64_t{1} << 31);
}

// ARROL_OK, or what is wrong with the arguments that both calls share
int check(const Problem& a, int64_t T_q, int64_t T_k) {
    if (T_q < 0 || T_k < 0 || a.pq.n < 0 || a.heads < 1 || a.kv_heads < 1 || a.heads % a.kv_heads || a.heads > 65536 || a.hd < 8 || a.hd > 128 || a.hd % 8) return ARROL_EINVAL;
    if (!(a.scale > 0.f) || a.scale > 3e38f) return ARROL_EINVAL;
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

size_t dot_bytes(int64_t T, int heads) { return (static_cast<size_t>(T) * heads * sizeof(float) + 255) / 256 * 256; }

}  // namespace

extern "C" int arrol_attention(const void* q, int64_t q_stride, const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                               const int64_t* cu_seqlens_q, const int64_t* cu_seqlens_k, int64_t T_q, int64_t T_k, int32_t n_seq,
                               int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, int32_t causal, float scale, void* out,
                               float* lse_out, void* stream) {
    const Problem a = problem(q, q_stride, k, k_stride, v, v_stride, cu_seqlens_q, cu_seqlens_k, T_q, T_k, n_seq, n_heads, n_kv_heads, head_dim, causal, scale);
    if (const int rc = check(a, T_q, T_k)) return rc;
    if (T_q == 0) return ARROL_OK;
    if (!out || !arrol_aligned16(out)) return ARROL_EINVAL;
    const int64_t tiles = tile_bound(T_q, n_seq, kOwn);
    const dim3 grid(static_cast<unsigned>(tiles * n_heads));
    const auto st = static_cast<hipStream_t>(stream);
    if (head_dim <= 64) arrol_launch(attention_forward_kernel<64>, grid, dim3(kThreads), 0, st, a, tiles, static_cast<uint16_t*>(out), lse_out);
    else arrol_launch(attention_forward_kernel<128>, grid, dim3(kThreads), 0, st, a, tiles, static_cast<uint16_t*>(out), lse_out);
    return arrol_launch_status();
}

extern "C" size_t arrol_attention_grad_workspace_bytes(int64_t T_q, int32_t n_heads) {
    return T_q <= 0 || n_heads <= 0 ? 0 : dot_bytes(T_q, n_heads);
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
    if (T_q > 0 && (!workspace || !arrol_aligned16(workspace) || workspace_bytes < dot_bytes(T_q, n_heads))) return ARROL_EWORKSPACE;
    const auto st = static_cast<hipStream_t>(stream);
    const auto *go = static_cast<const uint16_t*>(grad_out);
    float* dot = static_cast<float*>(workspace);
    if (T_q > 0) {
        const int64_t rows = T_q * n_heads;
        arrol_launch(attention_row_dot_kernel, dim3(static_cast<unsigned>((rows + 15) / 16 < kDotBlocks ? (rows + 15) / 16 : kDotBlocks)), dim3(256), 0, st, static_cast<const uint16_t*>(out), go, rows, T_q,
                     n_heads, head_dim, dot);
    }
    if (T_k > 0) {
        const dim3 grid(static_cast<unsigned>(tile_bound(T_k, n_seq, kOwn) * n_kv_heads));
        auto *dk = static_cast<uint16_t*>(grad_k), *dv = static_cast<uint16_t*>(grad_v);
        if (head_dim <= 64) arrol_launch(attention_grad_kv_kernel<64>, grid, dim3(kThreads), 0, st, a, go, lse, dot, dk, dv);
        else arrol_launch(attention_grad_kv_kernel<128>, grid, dim3(kThreads), 0, st, a, go, lse, dot, dk, dv);
    }
    if (T_q > 0) {
        const int64_t tiles = tile_bound(T_q, n_seq, kOwn);
        const dim3 grid(static_cast<unsigned>(tiles * n_heads));
        if (head_dim <= 64) arrol_launch(attention_grad_q_kernel<64>, grid, dim3(kThreads), 0, st, a, tiles, go, lse, dot, static_cast<uint16_t*>(grad_q));
        else arrol_launch(attention_grad_q_kernel<128>, grid, dim3(kThreads), 0, st, a, tiles, go, lse, dot, static_cast<uint16_t*>(grad_q));
    }
    return arrol_launch_status();
}
