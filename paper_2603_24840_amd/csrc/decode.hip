// Attention of one new token per rollout over the paged KV pool.  The rollouts of a prompt share the prompt's pages: their
// queries are one matrix, and the prompt's keys and values are read once for all of them.
//
//   keys of rollout r: the prefix pages of its group, then its own pages;  one softmax over both
//   o = sum_t p_t v_t,  p_t = exp(z_t - lse),  z_t = scale <q, k_t>
//   weight of token t += sum of p_t over the query heads (for a prefix token: over the group's rollouts as well)
//
// Bound by reading the cache (2 flop per byte and query row), so the work is cut for bytes in flight: a workgroup takes a range of tokens for a kv
// head and 16 or 32 query rows, its four wavefronts every fourth step of 32 tokens, and consecutive workgroups take consecutive kv heads, which
// together read whole pages.  K and V go, in whole rows of the head, through a part of the LDS that is the wavefront's own (V for the transposing
// read), and the next step's loads go out as soon as the registers are free, before the products: no barriers until the four wavefronts are joined.  Ranges are joined by a second launch; weights need the joined lse, so the scores are kept (4 bytes a query row and
// token against 4 head_dim of cache) and a third launch sums them.
#include "attention_tile.h"

namespace {
using namespace attention;

constexpr int kThreads = 256, kWaves = kThreads / ARROL_WAVE;
constexpr int kStep = 32;                  // tokens a wavefront takes at a time

__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

// (Query rows and tokens of a table row are counted in 32 bits, places in the pool too; offsets into memory in 64.)
// Block tables of one kind of rows: the rollouts' own, or the groups' prefixes.
struct Pages {
    const int32_t *table, *len;
    int per_row, chunk, splits, first_slot;     // pages of a row; tokens of a range; ranges; the first one's slot among a query's partials
    float* scores;                              // [query rows][cap], where weights are wanted
    int cap;
};

struct Decode {
    const uint16_t *q, *k, *v;
    Pages own, pre;
    Packed groups;                // of rollouts
    int64_t n_pages;
    int n, heads, kv_heads, hd, page, slots;
    float c;                      // scale * log2 e
    float *part_o, *part_ml, *lse2;
};

__device__ __forceinline__ int row_tokens(const Pages& p, int row, const Decode& a) {
    const int64_t cap = a.n_pages > 0 ? static_cast<int64_t>(p.per_row) * a.page : 0;      // no pool: nothing may be read
    const int len = p.len[row];
    return len < 0 ? 0 : static_cast<int>(len < cap ? len : cap);
}

// A tile of 32 rows of K in the LDS, read by rows (lane = key lane % 16, K32 step s): 16 lanes that a 128-bit read serves together have 16
// different rows and so positions.
template <int HD>
struct KeyTile {
    static constexpr int kRowBytes = 2 * HD, kChunks = HD / 8;
    __device__ static __forceinline__ int at(int r, int c) { return r * kRowBytes + ((c ^ (HD == 128 ? r & 15 : (r >> 1) & 7)) << 4); }
    __device__ static __forceinline__ bf16x8 by_row(const unsigned char* tile, int block, int s, int lane) {
        return *reinterpret_cast<const bf16x8*>(tile + at(16 * block + (lane & 15), 4 * s + (lane >> 4)));
    }
};

// A tile of 32 rows of V for the transposing read of 16 head elements x 32 keys: the 8 keys x 32 bytes of a half-wavefront
// fall on all banks once.
template <int HD>
struct ValueTile {
    static constexpr int kRowBytes = 2 * HD, kChunks = HD / 8, kBytes = kStep * kRowBytes;
    __device__ static __forceinline__ int at(int r, int c) {
        const int swizzle = HD == 128 ? (r & 7) << 1 : ((r >> 1) & 3) << 1;
        return r * kRowBytes + ((c ^ swizzle) << 4);
    }
    __device__ static __forceinline__ bf16x8 by_column(const unsigned char* tile, int d, int lane) {
        const int row = 4 * (lane >> 4) + ((lane >> 2) & 3), chunk = 2 * d + ((lane >> 1) & 1), within = (lane & 1) * 8;
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t)(tile + at(row, chunk) + within));
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t)(tile + at(row + 16, chunk) + within));
        return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
};

// One workgroup: query rows [first, first + 16 NQ) of a kv head (row = rollout * per + head of the kv head; past `end` the last one
// once more) against tokens [t0, t1) of table row `row`.
template <int HD, int NQ, bool SCORES>
__device__ __forceinline__ void decode_range(const Decode& a, const Pages& p, int row, int kvh, int first, int end, int t0, int t1, int slot,
                                             unsigned char (*lds)[2 * ValueTile<HD>::kBytes], float (*stat)[2][16 * NQ]) {
    constexpr int KS = HD / 32, DB = HD / 16, VL = kStep * HD / 8 / 64;
    using VT = ValueTile<HD>;
    const int lane = threadIdx.x & 63, wave = uniform(static_cast<int>(threadIdx.x >> 6));
    const int per = a.heads / a.kv_heads, l15 = lane & 15, g = lane >> 4;
    const int active = end - first > 16 ? NQ : 1;      // blocks of 16 query rows that there are
    unsigned char* tile = lds[wave];
    bf16x8 qf[NQ][KS];
    int64_t at[NQ];                        // this lane's query rows as (rollout, head) indices
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
        const int r = first + 16 * n + l15 < end ? first + 16 * n + l15 : end - 1;
        at[n] = static_cast<int64_t>(r / per) * a.heads + kvh * per + r % per;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            const int e = 32 * s + 8 * g;
            u32x4 x = {0, 0, 0, 0};
            if (e < a.hd) x = *reinterpret_cast<const u32x4*>(a.q + at[n] * a.hd + e);
            qf[n][s] = __builtin_bit_cast(bf16x8, x);
        }
    }
    f32x4 o[NQ][DB];
    float m[NQ], l[NQ];
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
        m[n] = -INFINITY, l[n] = 0.f;
#pragma unroll
        for (int d = 0; d < DB; ++d) o[n][d] = 0.f;
    }
    const int64_t token_stride = static_cast<int64_t>(a.kv_heads) * a.hd;
    const int32_t* table = p.table + static_cast<int64_t>(row) * p.per_row;
    // Chunks past the head are the head's last ones once more (Q is 0 there, and what V gives is not stored).
    const int last = a.hd / 8 - 1;
    const int64_t in_row = static_cast<int64_t>(kvh) * a.hd + (lane % VT::kChunks < last ? lane % VT::kChunks : last) * 8;
    const uint16_t *k = a.k + in_row, *v = a.v + in_row;

    // page id of token t + lane % 32; its place in the pool.  A token that does not exist (past the range, or a page id out of range) takes the place of
    // one of the step that does: its weight is 0, and that one's NaN would be in every sum anyway.  A step of none is left out.
    const auto page_of = [&](int t) {
        const int mine = t + (lane & 31);
        return mine < t1 ? table[mine / a.page] : -1;
    };
    uint32_t there;
    int place;
    const auto resolve = [&](int t, int id) {
        const bool exists = id >= 0 && id < a.n_pages;
        there = static_cast<uint32_t>(__ballot(exists));
        place = exists ? id * a.page + (t + (lane & 31)) % a.page : 0;
        const int other = there ? __builtin_amdgcn_readlane(place, __builtin_ctz(there)) : 0;
        place = exists ? place : other;
    };
    u32x4 kx[VL], vx[VL];
    const auto load = [&]() {
#pragma unroll
        for (int i = 0; i < VL; ++i) {
            const int64_t row_at = __shfl(place, i * (64 / VT::kChunks) + lane / VT::kChunks) * token_stride;
            kx[i] = *reinterpret_cast<const u32x4*>(k + row_at);
            vx[i] = *reinterpret_cast<const u32x4*>(v + row_at);
        }
    };
    constexpr int kStride = kWaves * kStep;
    int t = t0 + wave * kStep, id = -1;
    if (t < t1) {
        resolve(t, page_of(t));
        load();
        id = page_of(t + kStride);
    }
    for (; t < t1; t += kStride) {
        const uint32_t now = there;
        wave_lds_exchange();               // the reads of the last step are done
#pragma unroll
        for (int i = 0; i < VL; ++i) {
            const int r = i * (64 / VT::kChunks) + lane / VT::kChunks, c = lane % VT::kChunks;
            *reinterpret_cast<u32x4*>(tile + KeyTile<HD>::at(r, c)) = kx[i];
            *reinterpret_cast<u32x4*>(tile + VT::kBytes + VT::at(r, c)) = vx[i];
        }
        wave_lds_exchange();
        if (t + kStride < t1) {
            resolve(t + kStride, id);
            load();
            id = page_of(t + 2 * kStride);
        }
        f32x4 s[NQ][2];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
#pragma unroll
            for (int n = 0; n < NQ; ++n) s[n][b] = 0.f;
#pragma unroll
            for (int e = 0; e < KS; ++e) {
                const bf16x8 x = KeyTile<HD>::by_row(tile, b, e, lane);
#pragma unroll
                for (int n = 0; n < NQ; ++n)
                    s[n][b] = mfma16(x, qf[n][e], s[n][b]);
            }
        }
        float top_of[NQ];
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
            top_of[n] = -INFINITY;
#pragma unroll
            for (int b = 0; b < 2; ++b) {
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    s[n][b][r] = now >> (16 * b + 4 * g + r) & 1 ? s[n][b][r] * a.c : -INFINITY;
                    top_of[n] = fmaxf(top_of[n], s[n][b][r]);
                }
                // Stored by every lane (rows past the end store the last one's once more): on a branch, the wait for the loads that are
                // under way would have to allow for fewer stores behind them than there are, and wait for those.
                if constexpr (SCORES) *reinterpret_cast<f32x4*>(p.scores + at[n] * p.cap + t + 16 * b + 4 * g) = s[n][b];
            }
        }
        bf16x8 w[NQ];
#pragma unroll
        for (int n = 0; n < NQ; ++n)
            if (n < active) {
                float top = top_of[n];
                const auto larger = [](float x, float y) { return fmaxf(x, y); };
                top = wave_step<16>(wave_step<32>(top, larger), larger);
                if (__any(top > m[n] + 8.f)) {      // as in the packed form: moved on only where it has grown by 2^8
                    const float to = fmaxf(m[n], top), f = to == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m[n] - to);
                    m[n] = to;
                    l[n] *= f;
#pragma unroll
                    for (int d = 0; d < DB; ++d) o[n][d] *= f;
                }
                const float base = m[n] == -INFINITY ? 0.f : m[n];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float e = __builtin_amdgcn_exp2f(s[n][i >> 2][i & 3] - base);
                    l[n] += e;
                    w[n][i] = static_cast<__bf16>(e);      // weights in bf16 for the product with V, their sum l in fp32 of the unrounded ones
                }
            }
        if (now)
#pragma unroll
            for (int d = 0; d < DB; ++d) {
                const bf16x8 x = VT::by_column(tile + VT::kBytes, d, lane);
#pragma unroll
                for (int n = 0; n < NQ; ++n)
                    if (n < active) o[n][d] = mfma16(x, w[n], o[n][d]);
            }
    }
    // The four wavefronts' parts, brought to one maximum and added in a fixed order.
    const auto add = [](float x, float y) { return x + y; };
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
        l[n] = wave_step<16>(wave_step<32>(l[n], add), add);
        if (g == 0) stat[wave][0][16 * n + l15] = m[n], stat[wave][1][16 * n + l15] = l[n];
    }
    __syncthreads();
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
        if (n >= active) break;
        const int r = 16 * n + l15;
        const float top = fmaxf(fmaxf(stat[0][0][r], stat[1][0][r]), fmaxf(stat[2][0][r], stat[3][0][r]));
        const float f = m[n] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m[n] - top);
        constexpr int kRowFloats = HD + 4;          // 16 rows x HD floats, padded against bank conflicts
        float* part = reinterpret_cast<float*>(lds) + wave * 16 * kRowFloats;
#pragma unroll
        for (int d = 0; d < DB; ++d) *reinterpret_cast<f32x4*>(part + l15 * kRowFloats + 16 * d + 4 * g) = o[n][d] * f;
        __syncthreads();
        const float* parts = reinterpret_cast<const float*>(lds);
        for (int i = threadIdx.x; i < 16 * HD / 4; i += kThreads) {
            const int rr = i / (HD / 4), e = i % (HD / 4) * 4;
            const int query = first + 16 * n + rr;
            if (query < end && e < a.hd) {
                const int64_t out = (static_cast<int64_t>(query / per) * a.heads + kvh * per + query % per) * a.slots + slot;
                f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int w = 0; w < kWaves; ++w) sum += *reinterpret_cast<const f32x4*>(parts + (w * 16 + rr) * kRowFloats + e);
                *reinterpret_cast<f32x4*>(a.part_o + out * a.hd + e) = sum;
                if (e == 0) {
                    const int q = 16 * n + rr;
                    const float mm = fmaxf(fmaxf(stat[0][0][q], stat[1][0][q]), fmaxf(stat[2][0][q], stat[3][0][q]));
                    float ll = 0.f;
                    for (int w = 0; w < kWaves; ++w) ll += stat[w][0][q] == -INFINITY ? 0.f : stat[w][1][q] * __builtin_amdgcn_exp2f(stat[w][0][q] - mm);
                    *reinterpret_cast<f32x2*>(a.part_ml + 2 * out) = f32x2{mm, ll};
                }
            }
        }
        __syncthreads();
    }
}

// Blocks: first the groups' prefixes - (tile of a group's query rows, range, kv head) - then the rollouts' own tokens -
// ((rollout, tile of query rows), range, kv head).
template <int HD, int NQ, bool SCORES>
__global__ __launch_bounds__(kThreads, 2) void decode_kernel(Decode a, int64_t prefix_blocks) {
    __shared__ __align__(16) unsigned char lds[kWaves][2 * ValueTile<HD>::kBytes];
    static_assert(2 * ValueTile<HD>::kBytes >= 16 * (HD + 4) * 4, "a wavefront's part when they are joined");
    __shared__ float stat[kWaves][2][16 * NQ];
    const int lane = threadIdx.x & 63, per = a.heads / a.kv_heads;
    int64_t block = blockIdx.x;
    const bool prefix = block < prefix_blocks;
    block -= prefix ? 0 : prefix_blocks;
    const Pages& p = prefix ? a.pre : a.own;
    const int64_t rest = block / a.kv_heads;
    const int kvh = static_cast<int>((block + rest) % a.kv_heads);
    int row, split;
    int64_t first, begin, end;
    if (prefix) {
        const int64_t tiles = tile_bound(static_cast<int64_t>(a.n) * per, a.groups.n, 16 * NQ);       // tiles of the same range lie next to each other
        split = static_cast<int>(rest / tiles);
        int segment;
        if (!find_tile<16 * NQ>([&](int s) { return a.groups.bound(s) * per; }, a.groups.n + 2, rest % tiles, lane, segment, first, begin, end)) return;
        if (segment < 1 || segment > a.groups.n) return;
        row = segment - 1;
    } else {
        const int tiles = (per + 16 * NQ - 1) / (16 * NQ);
        split = static_cast<int>(rest % p.splits);
        const int64_t which = rest / p.splits;
        row = static_cast<int>(which / tiles);
        first = static_cast<int64_t>(row) * per + which % tiles * (16 * NQ);
        end = static_cast<int64_t>(row + 1) * per;
    }
    const int len = row_tokens(p, row, a), t0 = split * p.chunk;
    if (t0 >= len) return;
    decode_range<HD, NQ, SCORES>(a, p, row, kvh, static_cast<int>(first), static_cast<int>(end), t0, len - t0 < p.chunk ? len : t0 + p.chunk, p.first_slot + split,
                         lds, stat);
}

// The group of a rollout, -1 if it is in none: the last one that begins at or before it.
__device__ __forceinline__ int group_of(const Packed& groups, int64_t r, int lane) {
    int segment;
    int64_t first, end;
    if (groups.n <= 0) return -1;
    int lo = 0, count = groups.n + 2;
    while (count > 1) {
        const int step = (count + 63) >> 6, at = lane * step;
        const uint64_t votes = __ballot(at < count && groups.bound(lo + at) <= r);
        const int k = votes == ~0ull ? 63 : __builtin_ctzll(~votes) - 1, skip = (k < 0 ? 0 : k) * step;
        lo += skip;
        count = count - skip < step ? count - skip : step;
    }
    segment = __builtin_amdgcn_readfirstlane(lo);
    first = groups.bound(segment), end = groups.bound(segment + 1);
    return segment >= 1 && segment <= groups.n && r >= first && r < end ? segment - 1 : -1;
}

// Joins the ranges of a rollout's head, lane = 2 head elements.  WAVES wavefronts share a row's ranges: one where there are few.
template <int WAVES>
__global__ __launch_bounds__(kThreads) void decode_join_kernel(Decode a, uint16_t* __restrict__ out, float* __restrict__ lse_out) {
    constexpr int kInFlight = 4;
    __shared__ float parts[kWaves][3][64];
    const int lane = threadIdx.x & 63, wave = uniform(static_cast<int>(threadIdx.x >> 6)), part = wave % WAVES;
    const int64_t at = (static_cast<int64_t>(blockIdx.x) * kWaves + wave) / WAVES, rows = static_cast<int64_t>(a.n) * a.heads;
    float top = -INFINITY, sum = 0.f, x = 0.f, y = 0.f;
    if (at < rows) {
        const int r = static_cast<int>(at / a.heads);
        const int n_own = (row_tokens(a.own, r, a) + a.own.chunk - 1) / a.own.chunk;
        const int group = group_of(a.groups, r, lane);
        const int n_pre = group < 0 ? 0 : (row_tokens(a.pre, group, a) + a.pre.chunk - 1) / a.pre.chunk;
        const float* ml = a.part_ml + 2 * at * a.slots;
        const float* o = a.part_o + at * a.slots * a.hd + (2 * lane < a.hd ? 2 * lane : 0);
        const int n = n_pre + n_own;
        const auto slot_of = [&](int i) { return i < n_pre ? a.pre.first_slot + i : a.own.first_slot + i - n_pre; };
        for (int i = lane; i < n; i += 64) top = fmaxf(top, ml[2 * slot_of(i)]);
        top = wave_reduce(top, [](float u, float v) { return fmaxf(u, v); });
        const float base = top == -INFINITY ? 0.f : top;
        for (int i = part; i < n; i += WAVES * kInFlight) {
            f32x2 s[kInFlight], v[kInFlight];
#pragma unroll
            for (int u = 0; u < kInFlight; ++u) {       // past the end the first one again, so that no load waits on a branch
                const int slot = slot_of(i + u * WAVES < n ? i + u * WAVES : i);
                s[u] = *reinterpret_cast<const f32x2*>(ml + 2 * slot);
                v[u] = *reinterpret_cast<const f32x2*>(o + static_cast<int64_t>(slot) * a.hd);
            }
#pragma unroll
            for (int u = 0; u < kInFlight; ++u) {
                const float f = i + u * WAVES < n ? __builtin_amdgcn_exp2f(s[u].x - base) : 0.f;
                if (f != 0.f) sum += f * s[u].y, x += f * v[u].x, y += f * v[u].y;
            }
        }
    }
    if constexpr (WAVES > 1) {
        parts[wave][0][lane] = sum, parts[wave][1][lane] = x, parts[wave][2][lane] = y;
        __syncthreads();
        if (part != 0) return;
#pragma unroll
        for (int w = 1; w < WAVES; ++w) sum += parts[wave + w][0][lane], x += parts[wave + w][1][lane], y += parts[wave + w][2][lane];
    }
    if (at >= rows) return;
    const float inverse = sum == 0.f ? 0.f : 1.f / sum;
    if (2 * lane < a.hd)
        *reinterpret_cast<uint32_t*>(out + at * a.hd + 2 * lane) = f32_to_bf16_rne(x * inverse) | static_cast<uint32_t>(f32_to_bf16_rne(y * inverse)) << 16;
    if (lane == 0) {
        const float lse2 = sum == 0.f ? -INFINITY : top + log2f(sum);
        if (lse_out) lse_out[at] = lse2 * kLn2;
        if (a.lse2) a.lse2[at] = lse2;
    }
}

// Weights: the sum of exp2(score - lse) over the query rows that read a token, 4 tokens a lane.  A wavefront takes a rollout's own 256 tokens with all
// of its heads; a prefix' 256 tokens, which as many query rows read as its group has, are a workgroup's, its wavefronts every
// fourth row, added in a fixed order.  Table rows: the rollouts', then the groups'.
struct Weights {
    const float *in[2];
    float* out[2];
    int rows[2];        // of the rollouts, of the groups; 0: not wanted
    int64_t own_blocks; // a rollout row's
    int64_t own_total;  // all of them
    int64_t pre_blocks;
};
__global__ __launch_bounds__(kThreads) void decode_weight_kernel(Decode a, Weights w) {
    constexpr int kInFlight = 8;
    __shared__ f32x4 parts[kWaves][64];
    const int lane = threadIdx.x & 63, wave = uniform(static_cast<int>(threadIdx.x >> 6));
    const int prefix = static_cast<int64_t>(blockIdx.x) >= w.own_total;
    const int64_t block = blockIdx.x - (prefix ? w.own_total : 0), per_row = prefix ? w.pre_blocks : w.own_blocks;
    const int row = static_cast<int>(block / per_row);
    const Pages& p = prefix ? a.pre : a.own;
    const int64_t cap = static_cast<int64_t>(p.per_row) * a.page, t = ((block % per_row * (prefix ? 1 : kWaves) + (prefix ? 0 : wave)) * 64 + lane) * 4;
    const int len = row_tokens(p, row, a), first = prefix ? wave : 0, step = prefix ? kWaves : 1;
    const int64_t from = prefix ? a.groups.bound(row + 1) : row, to = prefix ? a.groups.bound(row + 2) : row + 1, last = to * a.heads;
    const float* in = w.in[prefix];
    float* out = w.out[prefix];
    f32x4 before = {0.f, 0.f, 0.f, 0.f};
    if (in && first == 0)
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (t + e < len) before[e] = in[row * cap + t + e];
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
    if (t < len)          // scores are there up to the next multiple of 32 tokens, -inf past the length
        for (int64_t i = from * a.heads + first; i < last; i += step * kInFlight) {
            f32x4 z[kInFlight];
            float lse[kInFlight];
#pragma unroll
            for (int u = 0; u < kInFlight; ++u) {
                const int64_t j = i + u * step < last ? i + u * step : i;
                z[u] = *reinterpret_cast<const f32x4*>(p.scores + j * p.cap + t);
                lse[u] = a.lse2[j];
            }
#pragma unroll
            for (int u = 0; u < kInFlight; ++u)
#pragma unroll
                for (int e = 0; e < 4; ++e) sum[e] += i + u * step < last && z[u][e] != -INFINITY ? __builtin_amdgcn_exp2f(z[u][e] - lse[u]) : 0.f;
        }
    if (prefix) {         // the same for the whole workgroup
        parts[wave][lane] = sum;
        __syncthreads();
        if (wave != 0) return;
#pragma unroll
        for (int u = 1; u < kWaves; ++u) sum += parts[u][lane];
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (t + e < cap) out[row * cap + t + e] = t + e < len ? before[e] + sum[e] : 0.f;
}

constexpr int kMinRange = kWaves * kStep, kMaxRange = 1024, kMaxSplits = 128;

// Ranges of a row of `cap` tokens where `blocks` workgroups (of both kinds) would take whole rows: as many as give 2,048 workgroups.
void cut(int64_t cap, int64_t blocks, int& chunk, int& splits) {
    int64_t want = blocks <= 0 ? 1 : (2048 + blocks - 1) / blocks, c = (cap + want - 1) / want;
    if (c > kMaxRange) c = kMaxRange;
    if (c < kMinRange) c = kMinRange;
    if (c < (cap + kMaxSplits - 1) / kMaxSplits) c = (cap + kMaxSplits - 1) / kMaxSplits;
    c = (c + kMinRange - 1) / kMinRange * kMinRange;
    chunk = static_cast<int>(c);
    splits = static_cast<int>(cap <= 0 ? 0 : (cap + c - 1) / c);
}

size_t up(size_t bytes) { return (bytes + 255) / 256 * 256; }

struct Plan {
    int own_chunk, own_splits, pre_chunk, pre_splits;
    int64_t own_cap, pre_cap;
    size_t ml, o, lse2, own_scores, pre_scores, total;
};

// Blocks of 16 query rows a workgroup takes: one where neither a rollout's heads nor an average group's rows fill more.
int query_blocks(int64_t n, int heads, int kv_heads, int64_t n_groups) {
    const int64_t per = heads / kv_heads;
    return per > 16 || (n_groups > 0 && n * per > 16 * n_groups) ? 2 : 1;
}

Plan plan(int64_t n, int heads, int kv_heads, int hd, int page, int64_t own_pages, int64_t pre_pages, int64_t n_groups, bool weights) {
    Plan p{};
    const int64_t own = own_pages * page, pre = n_groups > 0 ? pre_pages * page : 0;
    const int64_t per = heads / kv_heads, rows_of = 16 * query_blocks(n, heads, kv_heads, n_groups);
    const int64_t blocks = n * kv_heads * ((per + rows_of - 1) / rows_of) + (pre > 0 ? (n * per / rows_of + n_groups) * kv_heads : 0);
    cut(own, blocks, p.own_chunk, p.own_splits);
    cut(pre, blocks, p.pre_chunk, p.pre_splits);
    p.own_cap = (own + kStep - 1) / kStep * kStep, p.pre_cap = (pre + kStep - 1) / kStep * kStep;
    const size_t rows = static_cast<size_t>(n) * heads, slots = p.own_splits + p.pre_splits;
    size_t at = 0;
    const auto take = [&](size_t bytes) {
        const size_t here = at;
        at += up(bytes);
        return here;
    };
    p.ml = take(rows * slots * 8);
    p.o = take(rows * slots * hd * 4);
    p.lse2 = take(weights ? rows * 4 : 0);
    p.own_scores = take(weights ? rows * p.own_cap * 4 : 0);
    p.pre_scores = take(weights ? rows * p.pre_cap * 4 : 0);
    p.total = at;
    return p;
}

bool shape_ok(int64_t n, int heads, int kv_heads, int hd, int page, int64_t own_pages, int64_t pre_pages, int64_t n_groups) {
    if (n < 0 || heads < 1 || kv_heads < 1 || heads % kv_heads || hd < 8 || hd > 128 || hd % 8 || page < 1 || own_pages < 1 || n_groups < 0) return false;
    if (n_groups > 0 && pre_pages < 1) return false;
    const int64_t most = 0x7fffffff - 64;
    return own_pages <= most / page && (n_groups == 0 || pre_pages <= most / page) && n <= most / heads;
}

template <int HD, int NQ, bool SCORES>
void launch(const Decode& a, hipStream_t st) {
    const int64_t per = a.heads / a.kv_heads;
    const int64_t prefix = a.pre.splits > 0 ? tile_bound(a.n * per, a.groups.n, 16 * NQ) * a.pre.splits * a.kv_heads : 0;
    const int64_t own = a.n * ((per + 16 * NQ - 1) / (16 * NQ)) * a.own.splits * a.kv_heads;
    arrol_launch(decode_kernel<HD, NQ, SCORES>, dim3(static_cast<unsigned>(prefix + own)), dim3(kThreads), 0, st, a, prefix);
}

}  // namespace

extern "C" size_t arrol_decode_attention_workspace_bytes(int32_t n, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, int32_t page_tokens,
                                                         int32_t max_pages_per_seq, int32_t max_pages_per_prefix, int32_t n_groups, int32_t want_weight) {
    if (n == 0 || !shape_ok(n, n_heads, n_kv_heads, head_dim, page_tokens, max_pages_per_seq, max_pages_per_prefix, n_groups)) return 0;
    return plan(n, n_heads, n_kv_heads, head_dim, page_tokens, max_pages_per_seq, max_pages_per_prefix, n_groups, want_weight != 0).total;
}

extern "C" int arrol_decode_attention(const void* q, int32_t n, int32_t n_heads, const void* kv, arrol_kv_layout layout, int32_t layer,
                                      const int32_t* block_table, const int32_t* seq_len, int32_t max_pages_per_seq, const int32_t* prefix_table,
                                      const int32_t* prefix_len, int32_t max_pages_per_prefix, const int64_t* group_offsets, int32_t n_groups, float scale,
                                      void* out, float* lse_out, const float* weight_in, const float* prefix_weight_in, float* weight_out,
                                      float* prefix_weight_out, void* workspace, size_t workspace_bytes, void* stream) {
    if (!shape_ok(n, n_heads, layout.n_kv_heads, layout.head_dim, layout.page_tokens, max_pages_per_seq, max_pages_per_prefix, n_groups)) return ARROL_EINVAL;
    if (layout.n_layers < 1 || layer < 0 || layer >= layout.n_layers || layout.n_pages < 0 || layout.n_pages > 0x7fffffff / layout.page_tokens) return ARROL_EINVAL;
    if (!(scale > 0.f) || scale > 3e38f) return ARROL_EINVAL;
    if (n == 0 && n_groups == 0) return ARROL_OK;
    const bool weights = weight_out || prefix_weight_out;
    if ((!weight_out && weight_in) || (!prefix_weight_out && prefix_weight_in) || (n_groups == 0 && prefix_weight_out)) return ARROL_EINVAL;
    if (n_groups > 0 && (!prefix_table || !prefix_len || !group_offsets || n_groups > (1 << 20))) return ARROL_EINVAL;
    if (n > 0 && (!q || !out || !block_table || !seq_len || !arrol_aligned16(q) || !arrol_aligned16(out))) return ARROL_EINVAL;
    if (layout.n_pages > 0 && (!kv || !arrol_aligned16(kv))) return ARROL_EINVAL;
    if (weights && (static_cast<int64_t>(n) * max_pages_per_seq + static_cast<int64_t>(n_groups) * max_pages_per_prefix) * layout.page_tokens >= int64_t{1} << 30) return ARROL_EINVAL;
    const Plan p = plan(n, n_heads, layout.n_kv_heads, layout.head_dim, layout.page_tokens, max_pages_per_seq, max_pages_per_prefix, n_groups, weights);
    if (n > 0 && (!workspace || !arrol_aligned16(workspace) || workspace_bytes < p.total)) return ARROL_EWORKSPACE;
    auto* ws = static_cast<unsigned char*>(workspace);
    Decode a;
    const int64_t slab = layout.n_pages * layout.page_tokens * layout.n_kv_heads * layout.head_dim;
    a.q = static_cast<const uint16_t*>(q);
    a.k = static_cast<const uint16_t*>(kv) + 2 * static_cast<int64_t>(layer) * slab, a.v = a.k + slab;
    a.n = n, a.heads = n_heads, a.kv_heads = layout.n_kv_heads, a.hd = layout.head_dim, a.page = layout.page_tokens, a.n_pages = layout.n_pages;
    a.slots = p.own_splits + p.pre_splits, a.c = scale * kLog2e;
    a.groups = {group_offsets, n, n_groups};
    a.part_ml = reinterpret_cast<float*>(ws + p.ml), a.part_o = reinterpret_cast<float*>(ws + p.o);
    a.lse2 = weights ? reinterpret_cast<float*>(ws + p.lse2) : nullptr;
    a.pre = {prefix_table, prefix_len, max_pages_per_prefix, p.pre_chunk, p.pre_splits, 0, weights ? reinterpret_cast<float*>(ws + p.pre_scores) : nullptr,
             static_cast<int>(p.pre_cap)};
    a.own = {block_table, seq_len, max_pages_per_seq, p.own_chunk, p.own_splits, p.pre_splits, weights ? reinterpret_cast<float*>(ws + p.own_scores) : nullptr,
             static_cast<int>(p.own_cap)};
    const int64_t tiles = 2 * static_cast<int64_t>(n) * (n_heads / a.kv_heads + 15) / 16 + n + n_groups + 2;      // of query rows, at most
    if (tiles * (a.slots + 1) * a.kv_heads >= (1 << 24)) return ARROL_EINVAL;      // lanes of a launch are counted in 32 bits
    const auto st = static_cast<hipStream_t>(stream);
    if (n > 0) {
        const bool two = query_blocks(n, n_heads, a.kv_heads, n_groups) > 1;
        if (weights) {
            if (a.hd <= 64) two ? launch<64, 2, true>(a, st) : launch<64, 1, true>(a, st);
            else two ? launch<128, 2, true>(a, st) : launch<128, 1, true>(a, st);
        } else {
            if (a.hd <= 64) two ? launch<64, 2, false>(a, st) : launch<64, 1, false>(a, st);
            else two ? launch<128, 2, false>(a, st) : launch<128, 1, false>(a, st);
        }
        const int64_t rows = static_cast<int64_t>(n) * n_heads;
        auto* o = static_cast<uint16_t*>(out);
        if (a.slots > 8) arrol_launch(decode_join_kernel<4>, dim3(static_cast<unsigned>(rows)), dim3(kThreads), 0, st, a, o, lse_out);
        else arrol_launch(decode_join_kernel<1>, dim3(static_cast<unsigned>((rows + kWaves - 1) / kWaves)), dim3(kThreads), 0, st, a, o, lse_out);
    }
    if (weights) {
        const auto blocks = [&](int64_t pages, int64_t tokens) { return (pages * a.page + tokens - 1) / tokens; };
        Weights w = {{weight_in, prefix_weight_in}, {weight_out, prefix_weight_out}, {weight_out ? n : 0, prefix_weight_out ? n_groups : 0}, 0, 0, 0};
        w.own_blocks = blocks(max_pages_per_seq, 256 * kWaves), w.own_total = w.own_blocks * w.rows[0];
        w.pre_blocks = w.rows[1] ? blocks(max_pages_per_prefix, 256) : 1;
        const int64_t total = w.own_total + w.pre_blocks * w.rows[1];
        if (total > 0) arrol_launch(decode_weight_kernel, dim3(static_cast<unsigned>(total)), dim3(kThreads), 0, st, a, w);
    }
    return arrol_launch_status();
}
