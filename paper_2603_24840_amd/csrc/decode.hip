// Attention of one new token per rollout over the paged KV pool.  The rollouts of a prompt share the prompt's pages: their
// queries are one matrix, and the prompt's keys and values are read once for all of them.
//
//   keys of rollout r: the prefix pages of its group, then its own pages;  one softmax over both
//   o = sum_t p_t v_t,  p_t = exp(z_t - lse),  z_t = scale <q, k_t>
//   weight of token t += sum of p_t over the query heads (for a prefix token: over the group's rollouts as well)
//
// Bound by reading the cache (2 flop per byte and query row), so the work is cut for bytes in flight: a workgroup takes a range of tokens for a kv
// head, and consecutive workgroups take consecutive kv heads, which together read whole pages.  Where up to 16 query rows read the tokens (a rollout's heads over
// its kv head, small groups) its four wavefronts take every fourth step of 32 tokens: K and V go, in whole rows of the head, through a part of the LDS
// that is the wavefront's own, and the next step's loads go out as soon as the registers are free, before the products - no barriers until the four
// are joined.  Where more do (large groups) the tokens' tile is the workgroup's and its wavefronts have 16 of the rows each.  Ranges are joined by a second
// launch; weights need the joined lse, so the scores are kept (4 bytes a query row and token against 4 head_dim of cache) and a third launch sums them.
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
    __device__ static __forceinline__ int swizzle(int r) { return HD == 128 ? r & 15 : (r >> 1) & 7; }
    __device__ static __forceinline__ int at(int r, int c) { return r * kRowBytes + ((c ^ swizzle(r)) << 4); }
    __device__ static __forceinline__ bf16x8 by_row(const unsigned char* tile, int block, int s, int lane) {
        return *reinterpret_cast<const bf16x8*>(tile + at(16 * block + (lane & 15), 4 * s + (lane >> 4)));
    }
};

// A tile of 32 rows of V for the transposing read of 16 head elements x 32 keys: the 8 keys x 32 bytes of a half-wavefront
// fall on all banks once.
template <int HD>
struct ValueTile {
    static constexpr int kRowBytes = 2 * HD, kChunks = HD / 8, kBytes = kStep * kRowBytes;
    __device__ static __forceinline__ int swizzle(int r) { return HD == 128 ? (r & 7) << 1 : ((r >> 1) & 3) << 1; }
    __device__ static __forceinline__ int at(int r, int c) { return r * kRowBytes + ((c ^ swizzle(r)) << 4); }
    __device__ static __forceinline__ bf16x8 by_column(const unsigned char* tile, int d, int lane) {
        const int row = 4 * (lane >> 4) + ((lane >> 2) & 3), chunk = 2 * d + ((lane >> 1) & 1), within = (lane & 1) * 8;
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t)(tile + at(row, chunk) + within));
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t)(tile + at(row + 16, chunk) + within));
        return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
};

// A wavefront's 16 query rows [first, first + 16) of a kv head (row = rollout * per + head of the kv head; past `end` the last one once
// more), lane = row lane % 16, and what it has gathered for them.
template <int HD>
struct Rows {
    static constexpr int KS = HD / 32, DB = HD / 16;
    bf16x8 q[KS];
    int64_t at;                       // this lane's row as a (rollout, head) index
    f32x4 o[DB];                      // head elements 16 d + 4 (lane / 16) + r
    float m, l;                       // maximum of z * log2 e; this lane's part of the sum
    __device__ __forceinline__ void load(const Decode& a, int kvh, int first, int end, int lane) {
        const int per = a.heads / a.kv_heads, r = first + (lane & 15) < end ? first + (lane & 15) : end - 1;
        at = static_cast<int64_t>(r / per) * a.heads + kvh * per + r % per;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            const int e = 32 * s + 8 * (lane >> 4);
            u32x4 x = {0, 0, 0, 0};
            if (e < a.hd) x = *reinterpret_cast<const u32x4*>(a.q + at * a.hd + e);
            q[s] = __builtin_bit_cast(bf16x8, x);
        }
        m = -INFINITY, l = 0.f;
#pragma unroll
        for (int d = 0; d < DB; ++d) o[d] = 0.f;
    }
    // 32 tokens whose keys and values lie in the LDS, of which those in `there` exist; `scores`: this row's of the first token.
    template <bool SCORES>
    __device__ __forceinline__ void step(const Decode& a, const unsigned char* keys, const unsigned char* values, uint32_t there, float* scores, int lane) {
        const int g = lane >> 4;
        f32x4 s[2];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            s[b] = 0.f;
#pragma unroll
            for (int e = 0; e < KS; ++e) s[b] = mfma16(KeyTile<HD>::by_row(keys, b, e, lane), q[e], s[b]);
        }
        float top = -INFINITY;
#pragma unroll
        for (int b = 0; b < 2; ++b) {
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                s[b][r] = there >> (16 * b + 4 * g + r) & 1 ? s[b][r] * a.c : -INFINITY;
                top = fmaxf(top, s[b][r]);
            }
            // Stored by every lane (rows past the end store the last one's once more): on a branch, the wait for the loads that are
            // under way would have to allow for fewer stores behind them than there are, and wait for those.
            if constexpr (SCORES) *reinterpret_cast<f32x4*>(scores + 16 * b + 4 * g) = s[b];
        }
        const auto larger = [](float x, float y) { return fmaxf(x, y); };
        top = wave_step<16>(wave_step<32>(top, larger), larger);
        if (__any(top > m + 8.f)) {      // as in the packed form: moved on only where it has grown by 2^8
            const float to = fmaxf(m, top), f = to == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - to);
            m = to;
            l *= f;
#pragma unroll
            for (int d = 0; d < DB; ++d) o[d] *= f;
        }
        const float base = m == -INFINITY ? 0.f : m;
        bf16x8 w;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float e = __builtin_amdgcn_exp2f(s[i >> 2][i & 3] - base);
            l += e;
            w[i] = static_cast<__bf16>(e);      // weights in bf16 for the product with V, their sum l in fp32 of the unrounded ones
        }
        if (there == ~0u) {
#pragma unroll
            for (int d = 0; d < DB; ++d) o[d] = mfma16(ValueTile<HD>::by_column(values, d, lane), w, o[d]);
        } else if (there) {      // what lies in the places of tokens that do not exist is another one's value: infinity, it would be NaN with their weight of 0
            u32x4 exists;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t two = there >> (16 * (i >> 1) + 4 * g + 2 * (i & 1));
                exists[i] = (two & 1 ? 0xffffu : 0u) | (two & 2 ? 0xffff0000u : 0u);
            }
#pragma unroll
            for (int d = 0; d < DB; ++d)
                o[d] = mfma16(__builtin_bit_cast(bf16x8, __builtin_bit_cast(u32x4, ValueTile<HD>::by_column(values, d, lane)) & exists), w, o[d]);
        }
    }
    __device__ __forceinline__ float sum() const {
        const auto add = [](float x, float y) { return x + y; };
        return wave_step<16>(wave_step<32>(l, add), add);
    }
};

// Where a step's 32 tokens lie: page id of token t + lane % 32, and its place in the pool.  A token that does not exist (past the range, or a page id out of
// range) takes the place of one of the step that does, so nothing else is read; its score and its value are put aside.  Of a step of none nothing is added.
struct Places {
    const int32_t* table;
    int t1, page;
    int64_t n_pages;
    uint32_t there;
    int place;
    __device__ __forceinline__ int page_of(int t, int lane) const {
        const int mine = t + (lane & 31);
        return mine < t1 ? table[mine / page] : -1;
    }
    __device__ __forceinline__ void resolve(int t, int id, int lane) {
        const bool exists = id >= 0 && id < n_pages;
        there = static_cast<uint32_t>(__ballot(exists));
        place = exists ? id * page + (t + (lane & 31)) % page : 0;
        const int other = there ? __builtin_amdgcn_readlane(place, uniform(__builtin_ctz(there))) : 0;
        place = exists ? place : other;
    }
};

// A workgroup with up to 16 query rows against tokens [t0, t1) of table row `row`: its wavefronts take every fourth step of 32 tokens, each with its own part of the
// LDS, and are joined at the end.
template <int HD, bool SCORES>
__device__ __forceinline__ void few_rows(const Decode& a, const Pages& p, int row, int kvh, int first, int end, int t0, int t1, int slot,
                                         unsigned char (*lds)[2 * ValueTile<HD>::kBytes], float (*stat)[2][16]) {
    constexpr int DB = HD / 16, VL = kStep * HD / 8 / 64;
    using VT = ValueTile<HD>;
    const int lane = threadIdx.x & 63, wave = uniform(static_cast<int>(threadIdx.x >> 6));
    const int per = a.heads / a.kv_heads, l15 = lane & 15, g = lane >> 4;
    unsigned char* tile = lds[wave];
    Rows<HD> rows;
    rows.load(a, kvh, first, end, lane);
    const int64_t token_stride = static_cast<int64_t>(a.kv_heads) * a.hd;
    // Chunks past the head are read as the head's last ones once more, but stay the zeros of clear_tiles in the LDS: Q is 0 there, and 0 times an infinity of the
    // head would be NaN in its score.
    const int last = a.hd / 8 - 1;
    const bool in_head = lane % VT::kChunks <= last;
    const int64_t in_row = static_cast<int64_t>(kvh) * a.hd + (lane % VT::kChunks < last ? lane % VT::kChunks : last) * 8;
    const uint16_t *k = a.k + in_row, *v = a.v + in_row;
    Places at = {p.table + static_cast<int64_t>(row) * p.per_row, t1, a.page, a.n_pages, 0, 0};
    u32x4 kx[VL], vx[VL];
    const auto load = [&]() {
#pragma unroll
        for (int i = 0; i < VL; ++i) {
            const int64_t row_at = __shfl(at.place, i * (64 / VT::kChunks) + lane / VT::kChunks) * token_stride;
            kx[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(k + row_at));      // read by this workgroup alone, as a rule
            vx[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(v + row_at));
        }
    };
    clear_tiles<HD>(&lds[0][0], kWaves * 2 * VT::kBytes, a.hd);
    constexpr int kStride = kWaves * kStep;
    int t = t0 + wave * kStep, id = -1;
    if (t < t1) {
        at.resolve(t, at.page_of(t, lane), lane);
        load();
        id = at.page_of(t + kStride, lane);
    }
    for (; t < t1; t += kStride) {
        const uint32_t now = at.there;
        wave_lds_exchange();               // the reads of the last step are done
        if (in_head)
#pragma unroll
            for (int i = 0; i < VL; ++i) {
                const int r = i * (64 / VT::kChunks) + lane / VT::kChunks, c = lane % VT::kChunks;
                *reinterpret_cast<u32x4*>(tile + KeyTile<HD>::at(r, c)) = kx[i];
                *reinterpret_cast<u32x4*>(tile + VT::kBytes + VT::at(r, c)) = vx[i];
            }
        wave_lds_exchange();
        if (t + kStride < t1) {
            at.resolve(t + kStride, id, lane);
            load();
            id = at.page_of(t + 2 * kStride, lane);
        }
        rows.template step<SCORES>(a, tile, tile + VT::kBytes, now, SCORES ? p.scores + rows.at * p.cap + t : nullptr, lane);
    }
    // The four wavefronts' parts, brought to one maximum and added in a fixed order.  A maximum takes no notice of NaN: where all scores are NaN it is -inf, as
    // where there are none, but the sums are NaN, so every part is multiplied, none left out (here and in the join).
    const float l = rows.sum();
    if (g == 0) stat[wave][0][l15] = rows.m, stat[wave][1][l15] = l;
    __syncthreads();
    const float top = fmaxf(fmaxf(stat[0][0][l15], stat[1][0][l15]), fmaxf(stat[2][0][l15], stat[3][0][l15]));
    const float f = rows.m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(rows.m - top);
    constexpr int kRowFloats = HD + 4;          // 16 rows x HD floats, padded against bank conflicts
    static_assert(2 * VT::kBytes >= 16 * kRowFloats * 4, "a wavefront's part");
    float* parts = reinterpret_cast<float*>(lds);
#pragma unroll
    for (int d = 0; d < DB; ++d) *reinterpret_cast<f32x4*>(parts + (wave * 16 + l15) * kRowFloats + 16 * d + 4 * g) = rows.o[d] * f;
    __syncthreads();
    for (int i = threadIdx.x; i < 16 * HD / 4; i += kThreads) {
        const int r = i / (HD / 4), e = i % (HD / 4) * 4, query = first + r;
        if (query >= end || e >= a.hd) continue;
        const int64_t out = (static_cast<int64_t>(query / per) * a.heads + kvh * per + query % per) * a.slots + slot;
        f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < kWaves; ++w) sum += *reinterpret_cast<const f32x4*>(parts + (w * 16 + r) * kRowFloats + e);
        *reinterpret_cast<f32x4*>(a.part_o + out * a.hd + e) = sum;
        if (e == 0) {
            const float mm = fmaxf(fmaxf(stat[0][0][r], stat[1][0][r]), fmaxf(stat[2][0][r], stat[3][0][r]));
            float ll = 0.f;
            for (int w = 0; w < kWaves; ++w) ll += stat[w][1][r] * (stat[w][0][r] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(stat[w][0][r] - mm));
            *reinterpret_cast<f32x2*>(a.part_ml + 2 * out) = f32x2{mm, ll};
        }
    }
}

// A workgroup with up to 64 query rows, 16 a wavefront: keys and values of 32 tokens are read once for all of them, straight into the LDS, three such steps ahead of
// the one that is worked on.  The tokens' places are looked up for up to kPlaces at a time, so that no load stands between those: the wait for it would be a
// wait for all of them.  4 prompts of 9,000 to 16,384 tokens, 16 rollouts of 32 heads over 8 each: the launch takes 112 us, without the products 72
// and without the loads 82 (one workgroup to a compute unit: they overlap little); with the scores stored 123.
constexpr int kPlaces = 2048, kAhead = 3;
template <int N>
__device__ __forceinline__ void steps_ready() { asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory"); }

template <int HD, bool SCORES>
__device__ __forceinline__ void many_rows(const Decode& a, const Pages& p, int row, int kvh, int first, int end, int t0, int t1, int slot, unsigned char* lds, int* places) {
    constexpr int DB = HD / 16, VL = kStep * HD / 8 / 64 / kWaves, kLoads = 2 * VL;       // a wavefront's instructions of a step: K and V
    using VT = ValueTile<HD>;
    const int lane = threadIdx.x & 63, wave = uniform(static_cast<int>(threadIdx.x >> 6)), g = lane >> 4;
    const bool working = first + 16 * wave < end;        // of the wavefront
    Rows<HD> rows;
    rows.load(a, kvh, working ? first + 16 * wave : first, end, lane);
    const int64_t token_stride = static_cast<int64_t>(a.kv_heads) * a.hd;
    const int last = a.hd / 8 - 1;
    const uint16_t *k = a.k + static_cast<int64_t>(kvh) * a.hd, *v = a.v + static_cast<int64_t>(kvh) * a.hd;
    const unsigned lds0 = lds_address(lds);
    const int32_t* table = p.table + static_cast<int64_t>(row) * p.per_row;
    // the chunks that a lane fetches: an instruction fills 1,024 bytes of a tile in order
    int from_k[VL], from_v[VL];
#pragma unroll
    for (int i = 0; i < VL; ++i) {
        const int r = (wave * VL + i) * (64 / VT::kChunks) + lane / VT::kChunks, c = lane % VT::kChunks, ck = c ^ KeyTile<HD>::swizzle(r), cv = c ^ VT::swizzle(r);
        from_k[i] = ck <= last ? ck * 8 : -1, from_v[i] = cv <= last ? cv * 8 : -1;        // -1: past the head, left as it is (as in few_rows).
        // (An instruction has every chunk of its rows, so none of them goes out without a lane, and the waits count them all.)
    }
    clear_tiles<HD>(lds, 4 * 2 * VT::kBytes, a.hd);
    for (int start = t0; start < t1; start += kPlaces) {
        const int count = t1 - start < kPlaces ? t1 - start : kPlaces, n = (count + kStep - 1) / kStep;
        __syncthreads();                                 // the last places and steps are read
        for (int i = threadIdx.x; i < n * kStep; i += kThreads) {
            const int t = start + i, id = t < t1 ? table[t / a.page] : -1;
            places[i] = id >= 0 && id < a.n_pages ? id * a.page + t % a.page : -1;
        }
        __syncthreads();
        const auto issue = [&](int step) {
            int place = places[step * kStep + (lane & 31)];
            const uint32_t there = static_cast<uint32_t>(__ballot(place >= 0));
            const int other = there ? __builtin_amdgcn_readlane(place, uniform(__builtin_ctz(there))) : 0;      // as in Places
            place = place < 0 ? other : place;
#pragma unroll
            for (int i = 0; i < VL; ++i) {
                const int64_t at = __shfl(place, (wave * VL + i) * (64 / VT::kChunks) + lane / VT::kChunks) * token_stride;
                const uint16_t *key = k + at + from_k[i], *value = v + at + from_v[i];
                const unsigned to = lds0 + (step & 3) * 2 * VT::kBytes + (wave * VL + i) * 1024;
                if (a.hd == HD || from_k[i] >= 0) asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(key), "s"(to) : "memory");
                if (a.hd == HD || from_v[i] >= 0) asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(value), "s"(to + VT::kBytes) : "memory");
            }
        };
        for (int i = 0; i < kAhead && i < n; ++i) issue(i);
        if (n >= kAhead) steps_ready<2 * kLoads>();
        else steps_ready<0>();
        for (int i = 0; i < n; ++i) {
            if (i + kAhead < n) issue(i + kAhead);
            if (working) {
                const uint32_t there = static_cast<uint32_t>(__ballot(places[i * kStep + (lane & 31)] >= 0));
                const unsigned char* keys = lds + (i & 3) * 2 * VT::kBytes;
                rows.template step<SCORES>(a, keys, keys + VT::kBytes, there, SCORES ? p.scores + rows.at * p.cap + start + i * kStep : nullptr, lane);
            }
            // the next step is there, the two behind it may be under way (stores, which count too, can only make this wait for more)
            if (i + kAhead >= n) steps_ready<0>();
            else steps_ready<2 * kLoads>();
        }
    }
    const float l = rows.sum();
    const int per = a.heads / a.kv_heads, query = first + 16 * wave + (lane & 15);
    if (query >= end) return;
    const int64_t out = (static_cast<int64_t>(query / per) * a.heads + kvh * per + query % per) * a.slots + slot;
    if (g == 0) *reinterpret_cast<f32x2*>(a.part_ml + 2 * out) = f32x2{rows.m, l};
#pragma unroll
    for (int d = 0; d < DB; ++d)
        if (16 * d + 4 * g < a.hd) *reinterpret_cast<f32x4*>(a.part_o + out * a.hd + 16 * d + 4 * g) = rows.o[d];
}

// Query rows that a workgroup takes, of the prefixes and of the rollouts' own tokens: 16 or 64.
struct Tiles {
    int64_t prefix_blocks, prefix_tiles;
    int prefix_rows, own_rows, own_tiles;
};

// Blocks: first the groups' prefixes - (range, tile of a group's query rows, kv head) - then the rollouts' own tokens -
// ((rollout, tile of query rows), range, kv head).
template <int HD, bool SCORES>
__global__ __launch_bounds__(kThreads, 2) void decode_kernel(Decode a, Tiles w) {
    __shared__ __align__(1024) unsigned char lds[kWaves][2 * ValueTile<HD>::kBytes];       // [wavefront][K, V] or [step % 4][K, V]
    __shared__ float stat[kWaves][2][16];
    __shared__ int places[kPlaces];
    const int lane = threadIdx.x & 63, per = a.heads / a.kv_heads;
    int64_t block = blockIdx.x;
    const bool prefix = block < w.prefix_blocks;
    block -= prefix ? 0 : w.prefix_blocks;
    const Pages& p = prefix ? a.pre : a.own;
    const int64_t rest = block / a.kv_heads;
    const int kvh = static_cast<int>(block % a.kv_heads), rows = prefix ? w.prefix_rows : w.own_rows;
    int row, split;
    int64_t first, begin, end;
    if (prefix) {
        split = static_cast<int>(rest / w.prefix_tiles);         // tiles of the same range lie next to each other
        const auto bound = [&](int s) { return a.groups.bound(s) * per; };
        int segment;
        const bool found = rows == 16 ? find_tile<16>(bound, a.groups.n + 2, rest % w.prefix_tiles, lane, segment, first, begin, end)
                                      : find_tile<64>(bound, a.groups.n + 2, rest % w.prefix_tiles, lane, segment, first, begin, end);
        if (!found || segment < 1 || segment > a.groups.n) return;
        row = segment - 1;
    } else {
        split = static_cast<int>(rest % p.splits);
        const int64_t which = rest / p.splits;
        row = static_cast<int>(which / w.own_tiles);
        first = static_cast<int64_t>(row) * per + which % w.own_tiles * rows;
        end = static_cast<int64_t>(row + 1) * per;
    }
    const int len = row_tokens(p, row, a), t0 = split * p.chunk;
    if (t0 >= len) return;
    const int t1 = len - t0 < p.chunk ? len : t0 + p.chunk, slot = p.first_slot + split, f = static_cast<int>(first), e = static_cast<int>(end);
    if (rows == 16) few_rows<HD, SCORES>(a, p, row, kvh, f, e, t0, t1, slot, lds, stat);
    else many_rows<HD, SCORES>(a, p, row, kvh, f, e, t0, t1, slot, &lds[0][0], places);
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
                const float f = __builtin_amdgcn_exp2f(s[u].x - base);
                if (i + u * WAVES < n) sum += f * s[u].y, x += f * v[u].x, y += f * v[u].y;
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

constexpr int kMinRange = kWaves * kStep, kMaxRange = 2048, kMaxSplits = 128;
// Tokens past a row's end that the kernels' 32-bit counters may reach: few_rows looks up pages two strides and a step ahead (2 * 128 + 32), many_rows goes in
// steps of kPlaces.
constexpr int kPastTheEnd = 4096;
static_assert(kPastTheEnd >= kPlaces + kStep && kPastTheEnd >= 3 * kWaves * kStep, "tokens are counted in 32 bits");

// Ranges of a row of `cap` tokens where `blocks` workgroups (of both kinds) would take whole rows: as many as give 2,048 workgroups, of at most
// 2,048 tokens (384 rollouts of up to 2,000 tokens: 356 us a call, in ranges of 1,024 404).
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
    Tiles tiles;
    int64_t blocks, join_blocks, own_weight_blocks, pre_weight_blocks;      // workgroups of the launches; of the weights', a row's
    bool fits;                      // lanes of a launch are counted in 32 bits
};
constexpr int64_t kMostBlocks = (int64_t{1} << 32) / kThreads;

// Query rows that a workgroup takes where a rollout's heads, or an average group, has `rows` of them and up to `tokens` tokens to read: 64 where 16
// would leave the same tokens to several, but not so few of them that four wavefronts side by side are done sooner (8 rollouts of 32 heads over 8 behind
// 200 tokens: 9.2 us, with 64 rows 10.9).
int rows_of(int64_t rows, int64_t tokens) { return rows > 16 && tokens > 512 ? 64 : 16; }
// Wavefronts that share a row's ranges in the join.
int join_waves(int slots) { return slots > 8 ? 4 : 1; }

Plan plan(int64_t n, int heads, int kv_heads, int hd, int page, int64_t own_pages, int64_t pre_pages, int64_t n_groups, bool weights) {
    Plan p{};
    const int64_t own = own_pages * page, pre = n_groups > 0 ? pre_pages * page : 0;
    const int64_t per = heads / kv_heads;
    Tiles& w = p.tiles;
    w.own_rows = rows_of(per, own), w.own_tiles = static_cast<int>((per + w.own_rows - 1) / w.own_rows);
    w.prefix_rows = n_groups > 0 ? rows_of(n * per / n_groups, pre) : 16;
    const int64_t blocks = n * kv_heads * w.own_tiles + (pre > 0 ? (n * per / w.prefix_rows + n_groups) * kv_heads : 0);
    cut(own, blocks, p.own_chunk, p.own_splits);
    cut(pre, blocks, p.pre_chunk, p.pre_splits);
    w.prefix_tiles = tile_bound(n * per, static_cast<int>(n_groups), w.prefix_rows);
    w.prefix_blocks = w.prefix_tiles * p.pre_splits * kv_heads;
    p.blocks = n > 0 ? w.prefix_blocks + n * w.own_tiles * p.own_splits * kv_heads : 0;
    p.join_blocks = join_waves(p.own_splits + p.pre_splits) > 1 ? n * heads : (n * heads + kWaves - 1) / kWaves;
    p.own_weight_blocks = (own + 256 * kWaves - 1) / (256 * kWaves), p.pre_weight_blocks = (pre + 255) / 256;
    p.fits = p.blocks < kMostBlocks && p.join_blocks < kMostBlocks &&
             (!weights || (n * own + n_groups * pre < int64_t{1} << 30 && n * p.own_weight_blocks + n_groups * p.pre_weight_blocks < kMostBlocks));
    p.own_cap = ((own + kStep - 1) / kStep | 1) * kStep, p.pre_cap = ((pre + kStep - 1) / kStep | 1) * kStep;      // odd, so that rows begin on all channels
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
    if (n < 0 || heads < 1 || kv_heads < 1 || heads % kv_heads || hd < 8 || hd > 128 || hd % 8 || page < 1 || own_pages < 1 || n_groups < 0 || n_groups > (1 << 20)) return false;
    if (n_groups > 0 && pre_pages < 1) return false;
    const int64_t most = 0x7fffffff - kPastTheEnd;
    return own_pages <= most / page && (n_groups == 0 || pre_pages <= most / page) && n <= most / heads;
}

template <int HD, bool SCORES>
void launch(const Decode& a, const Plan& p, hipStream_t st) {
    arrol_launch(decode_kernel<HD, SCORES>, dim3(static_cast<unsigned>(p.blocks)), dim3(kThreads), 0, st, a, p.tiles);
}

}  // namespace

extern "C" size_t arrol_decode_attention_workspace_bytes(int32_t n, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, int32_t page_tokens,
                                                         int32_t max_pages_per_seq, int32_t max_pages_per_prefix, int32_t n_groups, int32_t want_weight) {
    if (n == 0 || !shape_ok(n, n_heads, n_kv_heads, head_dim, page_tokens, max_pages_per_seq, max_pages_per_prefix, n_groups)) return 0;
    const Plan p = plan(n, n_heads, n_kv_heads, head_dim, page_tokens, max_pages_per_seq, max_pages_per_prefix, n_groups, want_weight != 0);
    return p.fits ? p.total : 0;
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
    if (n_groups > 0 && (!prefix_table || !prefix_len || !group_offsets)) return ARROL_EINVAL;
    if (n > 0 && (!q || !out || !block_table || !seq_len || !arrol_aligned16(q) || !arrol_aligned16(out))) return ARROL_EINVAL;
    if (layout.n_pages > 0 && (!kv || !arrol_aligned16(kv))) return ARROL_EINVAL;
    const Plan p = plan(n, n_heads, layout.n_kv_heads, layout.head_dim, layout.page_tokens, max_pages_per_seq, max_pages_per_prefix, n_groups, weights);
    if (!p.fits) return ARROL_EINVAL;
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
    const auto st = static_cast<hipStream_t>(stream);
    if (n > 0) {
        if (a.hd <= 64) weights ? launch<64, true>(a, p, st) : launch<64, false>(a, p, st);
        else weights ? launch<128, true>(a, p, st) : launch<128, false>(a, p, st);
        auto* o = static_cast<uint16_t*>(out);
        const dim3 grid(static_cast<unsigned>(p.join_blocks));
        if (join_waves(a.slots) > 1) arrol_launch(decode_join_kernel<4>, grid, dim3(kThreads), 0, st, a, o, lse_out);
        else arrol_launch(decode_join_kernel<1>, grid, dim3(kThreads), 0, st, a, o, lse_out);
    }
    if (weights) {
        Weights w = {{weight_in, prefix_weight_in}, {weight_out, prefix_weight_out}, {weight_out ? n : 0, prefix_weight_out ? n_groups : 0}, p.own_weight_blocks, 0, 1};
        w.own_total = w.own_blocks * w.rows[0];
        if (w.rows[1]) w.pre_blocks = p.pre_weight_blocks;
        const int64_t total = w.own_total + w.pre_blocks * w.rows[1];
        if (total > 0) arrol_launch(decode_weight_kernel, dim3(static_cast<unsigned>(total)), dim3(kThreads), 0, st, a, w);
    }
    return arrol_launch_status();
}
