// Attention of one new token per rollout over the paged KV pool.  The rollouts of a prompt share the prompt's pages: their
// queries are one matrix, and the prompt's keys and values are read once for all of them.
//
//   keys of rollout r: the prefix pages of its group, then its own pages;  one softmax over both
//   o = sum_t p_t v_t,  p_t = exp(z_t - lse),  z_t = scale <q, k_t>
//   weight of token t += sum of p_t over the query heads (for a prefix token: over the group's rollouts as well)
//
// Bound by reading the cache (2 flop per byte and query row), so the work is cut for bytes in flight: a wavefront takes one kv head's keys of a range of
// tokens, and consecutive wavefronts take consecutive kv heads, which together read whole pages.  K goes from memory straight into MFMA fragments,
// V through a part of the LDS that is the wavefront's own (transposing read), so there are no barriers.  Ranges are joined
// by a second launch; weights need the joined lse, so the scores are kept (4 bytes a query row and token against 4 head_dim of cache) and a third launch sums them.
#include "attention_tile.h"

namespace {
using namespace attention;

constexpr int kThreads = 256, kWaves = kThreads / ARROL_WAVE;
constexpr int kStep = 32;                  // tokens a wavefront takes at a time

__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

// Block tables of one kind of rows: the rollouts' own, or the groups' prefixes.
struct Pages {
    const int32_t *table, *len;
    int per_row, chunk, splits, first_slot;     // pages of a row; tokens of a range; ranges; the first one's slot among a query's partials
    float* scores;                              // [query rows][cap], or NULL
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

__device__ __forceinline__ int row_tokens(const Pages& p, int row, int page) {
    const int64_t cap = static_cast<int64_t>(p.per_row) * page;
    const int len = p.len[row];
    return len < 0 ? 0 : static_cast<int>(len < cap ? len : cap);
}

// A tile of 32 rows of V in the LDS for the transposing read of 16 head elements x 32 keys: the 8 keys x 32 bytes of a half-wavefront
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

// One wavefront: query rows [first, first + 16 NQ) of a kv head (row = rollout * per + head of the kv head; those from `end` on are
// padding) against tokens [t0, t1) of table row `row`.
template <int HD, int NQ>
__device__ __forceinline__ void decode_range(const Decode& a, const Pages& p, int row, int kvh, int64_t first, int64_t end, int t0, int t1, int slot,
                                             unsigned char* tile, int lane) {
    constexpr int KS = HD / 32, DB = HD / 16, VL = kStep * HD / 8 / 64;
    using VT = ValueTile<HD>;
    const int per = a.heads / a.kv_heads, l15 = lane & 15, g = lane >> 4;
    bf16x8 qf[NQ][KS];
    int64_t at[NQ];                        // this lane's query rows as (rollout, head) indices, -1 past the end
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
        const int64_t r = first + 16 * n + l15;
        at[n] = r < end ? r / per * a.heads + kvh * per + r % per : -1;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            const int e = 32 * s + 8 * g;
            u32x4 x = {0, 0, 0, 0};
            if (at[n] >= 0 && e < a.hd) x = *reinterpret_cast<const u32x4*>(a.q + at[n] * a.hd + e);
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
    const uint16_t *k = a.k + static_cast<int64_t>(kvh) * a.hd, *v = a.v + static_cast<int64_t>(kvh) * a.hd;
    for (int t = t0; t < t1; t += kStep) {
        // token t + (lane & 31): its place in the pool, -1 where there is none (past the range, or a page id out of range)
        const int mine = t + (lane & 31);
        int64_t place = -1;
        if (mine < t1) {
            const int id = table[mine / a.page];
            if (id >= 0 && id < a.n_pages) place = static_cast<int64_t>(id) * a.page + mine % a.page;
        }
        const uint32_t there = static_cast<uint32_t>(__ballot(place >= 0));
        u32x4 kx[2][KS], vx[VL];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            const int64_t at_k = __shfl(place, 16 * b + l15);
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                const int e = 32 * s + 8 * g;
                kx[b][s] = {0, 0, 0, 0};
                if (at_k >= 0 && e < a.hd) kx[b][s] = *reinterpret_cast<const u32x4*>(k + at_k * token_stride + e);
            }
        }
#pragma unroll
        for (int i = 0; i < VL; ++i) {
            const int j = i * (64 / VT::kChunks) + lane / VT::kChunks, c = lane % VT::kChunks;
            const int64_t at_v = __shfl(place, j);
            vx[i] = {0, 0, 0, 0};          // no token: zeros, whatever the page holds there (its weight is 0, and 0 * NaN is not)
            if (at_v >= 0 && c * 8 < a.hd) vx[i] = *reinterpret_cast<const u32x4*>(v + at_v * token_stride + c * 8);
        }
        f32x4 s[NQ][2];
#pragma unroll
        for (int n = 0; n < NQ; ++n)
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                s[n][b] = 0.f;
#pragma unroll
                for (int e = 0; e < KS; ++e) s[n][b] = mfma16(__builtin_bit_cast(bf16x8, kx[b][e]), qf[n][e], s[n][b]);
            }
        bf16x8 w[NQ];
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
            float top = -INFINITY;
#pragma unroll
            for (int b = 0; b < 2; ++b) {
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    s[n][b][r] = there >> (16 * b + 4 * g + r) & 1 ? s[n][b][r] * a.c : -INFINITY;
                    top = fmaxf(top, s[n][b][r]);
                }
                if (p.scores && at[n] >= 0) *reinterpret_cast<f32x4*>(p.scores + at[n] * p.cap + t + 16 * b + 4 * g) = s[n][b];
            }
            const auto larger = [](float x, float y) { return fmaxf(x, y); };
            top = wave_step<16>(wave_step<32>(top, larger), larger);
            if (__any(top > m[n] + 8.f)) {
                const float to = fmaxf(m[n], top), f = to == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m[n] - to);
                m[n] = to;
                l[n] *= f;
#pragma unroll
                for (int d = 0; d < DB; ++d) o[n][d] *= f;
            }
            const float base = m[n] == -INFINITY ? 0.f : m[n];
            float e[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                e[i] = __builtin_amdgcn_exp2f(s[n][i >> 2][i & 3] - base);
                l[n] += e[i];
                w[n][i] = static_cast<__bf16>(e[i]);      // weights in bf16 for the product with V, their sum l in fp32 of the unrounded ones
            }
        }
        wave_lds_exchange();               // the reads of the last round are done
#pragma unroll
        for (int i = 0; i < VL; ++i) *reinterpret_cast<u32x4*>(tile + VT::at(i * (64 / VT::kChunks) + lane / VT::kChunks, lane % VT::kChunks)) = vx[i];
        wave_lds_exchange();
#pragma unroll
        for (int d = 0; d < DB; ++d) {
            const bf16x8 x = VT::by_column(tile, d, lane);
#pragma unroll
            for (int n = 0; n < NQ; ++n) o[n][d] = mfma16(x, w[n], o[n][d]);
        }
    }
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
        const auto add = [](float x, float y) { return x + y; };
        const float sum = wave_step<16>(wave_step<32>(l[n], add), add);
        if (at[n] < 0) continue;
        const int64_t part = at[n] * a.slots + slot;
        if (g == 0) *reinterpret_cast<f32x2*>(a.part_ml + 2 * part) = f32x2{m[n], sum};
#pragma unroll
        for (int d = 0; d < DB; ++d)
            if (16 * d + 4 * g < a.hd) *reinterpret_cast<f32x4*>(a.part_o + part * a.hd + 16 * d + 4 * g) = o[n][d];
    }
}

// The rollouts' own tokens: unit = ((rollout, tile of query rows), range, kv head).
template <int HD, int NQ>
__global__ __launch_bounds__(kThreads) void decode_own_kernel(Decode a, int64_t units) {
    __shared__ __align__(16) unsigned char lds[kWaves][ValueTile<HD>::kBytes];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t unit = static_cast<int64_t>(blockIdx.x) * kWaves + wave;
    if (unit >= units) return;
    const int per = a.heads / a.kv_heads, tiles = (per + 16 * NQ - 1) / (16 * NQ);
    const int kvh = static_cast<int>(unit % a.kv_heads);
    int64_t rest = unit / a.kv_heads;
    const int split = static_cast<int>(rest % a.own.splits);
    rest /= a.own.splits;
    const int tile = static_cast<int>(rest % tiles), r = static_cast<int>(rest / tiles);
    const int len = row_tokens(a.own, r, a.page), t0 = split * a.own.chunk;
    if (t0 >= len) return;
    const int t1 = len - t0 < a.own.chunk ? len : t0 + a.own.chunk;
    decode_range<HD, NQ>(a, a.own, r, kvh, static_cast<int64_t>(r) * per + tile * 16 * NQ, static_cast<int64_t>(r + 1) * per, t0, t1, a.own.first_slot + split,
                         lds[wave], lane);
}

// The groups' prefixes: unit = (tile of a group's query rows, range, kv head).
template <int HD, int NQ>
__global__ __launch_bounds__(kThreads) void decode_prefix_kernel(Decode a, int64_t units) {
    __shared__ __align__(16) unsigned char lds[kWaves][ValueTile<HD>::kBytes];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t unit = static_cast<int64_t>(blockIdx.x) * kWaves + wave;
    if (unit >= units) return;
    const int per = a.heads / a.kv_heads;
    const int kvh = static_cast<int>(unit % a.kv_heads);
    const int64_t rest = unit / a.kv_heads;
    const int split = static_cast<int>(rest % a.pre.splits);
    int segment;
    int64_t first, end;
    if (!find_tile<16 * NQ>([&](int s) { return a.groups.bound(s) * per; }, a.groups.n + 2, rest / a.pre.splits, lane, segment, first, end)) return;
    if (segment < 1 || segment > a.groups.n) return;
    const int len = row_tokens(a.pre, segment - 1, a.page), t0 = split * a.pre.chunk;
    if (t0 >= len) return;
    const int t1 = len - t0 < a.pre.chunk ? len : t0 + a.pre.chunk;
    decode_range<HD, NQ>(a, a.pre, segment - 1, kvh, first, end, t0, t1, a.pre.first_slot + split, lds[wave], lane);
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

// Joins the ranges of a rollout's head: one wavefront each, lane = 2 head elements.
__global__ __launch_bounds__(kThreads) void decode_join_kernel(Decode a, uint16_t* __restrict__ out, float* __restrict__ lse_out) {
    const int lane = threadIdx.x & 63;
    const int64_t at = static_cast<int64_t>(blockIdx.x) * kWaves + (threadIdx.x >> 6);
    if (at >= static_cast<int64_t>(a.n) * a.heads) return;
    const int r = static_cast<int>(at / a.heads);
    const int n_own = (row_tokens(a.own, r, a.page) + a.own.chunk - 1) / a.own.chunk;
    const int group = group_of(a.groups, r, lane);
    const int n_pre = group < 0 ? 0 : (row_tokens(a.pre, group, a.page) + a.pre.chunk - 1) / a.pre.chunk;
    const float* ml = a.part_ml + 2 * at * a.slots;
    const int n = n_pre + n_own;
    const auto slot_of = [&](int i) { return i < n_pre ? a.pre.first_slot + i : a.own.first_slot + i - n_pre; };
    float top = -INFINITY;
    for (int i = lane; i < n; i += 64) top = fmaxf(top, ml[2 * slot_of(i)]);
    top = wave_reduce(top, [](float x, float y) { return fmaxf(x, y); });
    float sum = 0.f, x = 0.f, y = 0.f;
    const float base = top == -INFINITY ? 0.f : top;
    for (int i = 0; i < n; ++i) {
        const int slot = slot_of(i);
        const float f = __builtin_amdgcn_exp2f(ml[2 * slot] - base);
        sum += f * ml[2 * slot + 1];
        if (2 * lane < a.hd) {
            const f32x2 v = *reinterpret_cast<const f32x2*>(a.part_o + (at * a.slots + slot) * a.hd + 2 * lane);
            x += f * v.x, y += f * v.y;
        }
    }
    const float inverse = sum == 0.f ? 0.f : 1.f / sum;
    if (2 * lane < a.hd)
        *reinterpret_cast<uint32_t*>(out + at * a.hd + 2 * lane) = f32_to_bf16_rne(x * inverse) | static_cast<uint32_t>(f32_to_bf16_rne(y * inverse)) << 16;
    if (lane == 0) {
        const float lse2 = sum == 0.f ? -INFINITY : top + log2f(sum);
        if (lse_out) lse_out[at] = lse2 * kLn2;
        if (a.lse2) a.lse2[at] = lse2;
    }
}

// Weights of 64 tokens of a table row: the sum of exp2(score - lse) over the query rows that read them, four wavefronts a quarter each, added
// in a fixed order.
__global__ __launch_bounds__(kThreads) void decode_weight_kernel(Decode a, Pages p, int prefix, const float* __restrict__ in, float* __restrict__ out) {
    __shared__ float part[kWaves][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, row = blockIdx.y;
    const int64_t cap = static_cast<int64_t>(p.per_row) * a.page;
    const int len = row_tokens(p, row, a.page);
    const int64_t t = static_cast<int64_t>(blockIdx.x) * 64 + lane;
    const int64_t from = prefix ? a.groups.bound(row + 1) : row, to = prefix ? a.groups.bound(row + 2) : row + 1;
    float sum = 0.f;
    if (t < len)
        for (int64_t i = from * a.heads + wave; i < to * a.heads; i += kWaves) {
            const float z = p.scores[i * p.cap + t];
            sum += z == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(z - a.lse2[i]);
        }
    part[wave][lane] = sum;
    __syncthreads();
    if (wave == 0 && t < cap) {
        const int64_t at = row * cap + t;
        const float before = in && t < len ? in[at] : 0.f;
        out[at] = t < len ? before + ((part[0][lane] + part[1][lane]) + (part[2][lane] + part[3][lane])) : 0.f;
    }
}

constexpr int kMinRange = 64, kMaxRange = 512, kMaxSplits = 128;

// Ranges of a row of `cap` tokens where `rows` wavefronts would take whole rows: as many as give 4,096 wavefronts.
void cut(int64_t cap, int64_t rows, int& chunk, int& splits) {
    int64_t want = rows <= 0 ? 1 : (4096 + rows - 1) / rows, c = (cap + want - 1) / want;
    if (c > kMaxRange) c = kMaxRange;
    if (c < kMinRange) c = kMinRange;
    if (c < (cap + kMaxSplits - 1) / kMaxSplits) c = (cap + kMaxSplits - 1) / kMaxSplits;
    c = (c + kStep - 1) / kStep * kStep;
    chunk = static_cast<int>(c);
    splits = static_cast<int>(cap <= 0 ? 0 : (cap + c - 1) / c);
}

size_t up(size_t bytes) { return (bytes + 255) / 256 * 256; }

struct Plan {
    int own_chunk, own_splits, pre_chunk, pre_splits;
    int64_t own_cap, pre_cap;
    size_t ml, o, lse2, own_scores, pre_scores, total;
};

Plan plan(int64_t n, int heads, int kv_heads, int hd, int page, int64_t own_pages, int64_t pre_pages, int64_t n_groups, bool weights) {
    Plan p{};
    const int64_t own = own_pages * page, pre = n_groups > 0 ? pre_pages * page : 0;
    cut(own, n * kv_heads, p.own_chunk, p.own_splits);
    cut(pre, n_groups * kv_heads, p.pre_chunk, p.pre_splits);
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

template <int HD, int NQ>
void launch_prefix(const Decode& a, hipStream_t st) {
    const int64_t per = a.heads / a.kv_heads, units = tile_bound(a.n * per, a.groups.n, 16 * NQ) * a.pre.splits * a.kv_heads;
    arrol_launch(decode_prefix_kernel<HD, NQ>, dim3(static_cast<unsigned>((units + kWaves - 1) / kWaves)), dim3(kThreads), 0, st, a, units);
}
template <int HD, int NQ>
void launch_own(const Decode& a, hipStream_t st) {
    const int64_t per = a.heads / a.kv_heads, units = a.n * ((per + 16 * NQ - 1) / (16 * NQ)) * a.own.splits * a.kv_heads;
    arrol_launch(decode_own_kernel<HD, NQ>, dim3(static_cast<unsigned>((units + kWaves - 1) / kWaves)), dim3(kThreads), 0, st, a, units);
}
template <int HD>
void launch(const Decode& a, hipStream_t st) {
    const int64_t per = a.heads / a.kv_heads;
    if (a.pre.splits > 0) {
        const int64_t rows = a.n * per / a.groups.n;       // of an average group
        if (rows > 32) launch_prefix<HD, 4>(a, st);
        else if (rows > 16) launch_prefix<HD, 2>(a, st);
        else launch_prefix<HD, 1>(a, st);
    }
    if (per > 32) launch_own<HD, 4>(a, st);
    else if (per > 16) launch_own<HD, 2>(a, st);
    else launch_own<HD, 1>(a, st);
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
    if (layout.n_layers < 1 || layer < 0 || layer >= layout.n_layers || layout.n_pages < 0 || layout.n_pages > 0x7fffffff) return ARROL_EINVAL;
    if (!(scale > 0.f) || scale > 3e38f) return ARROL_EINVAL;
    if (n == 0 && n_groups == 0) return ARROL_OK;
    const bool weights = weight_out || prefix_weight_out;
    if ((!weight_out && weight_in) || (!prefix_weight_out && prefix_weight_in) || (n_groups == 0 && prefix_weight_out)) return ARROL_EINVAL;
    if (n_groups > 0 && (!prefix_table || !prefix_len || !group_offsets || n_groups > 65535)) return ARROL_EINVAL;
    if (n > 0 && (!q || !out || !block_table || !seq_len || !arrol_aligned16(q) || !arrol_aligned16(out))) return ARROL_EINVAL;
    if (layout.n_pages > 0 && (!kv || !arrol_aligned16(kv))) return ARROL_EINVAL;
    if (weights && n > 65535) return ARROL_EINVAL;
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
    a.pre = {prefix_table, prefix_len, max_pages_per_prefix, p.pre_chunk, p.pre_splits, 0, prefix_weight_out ? reinterpret_cast<float*>(ws + p.pre_scores) : nullptr,
             static_cast<int>(p.pre_cap)};
    a.own = {block_table, seq_len, max_pages_per_seq, p.own_chunk, p.own_splits, p.pre_splits, weight_out ? reinterpret_cast<float*>(ws + p.own_scores) : nullptr,
             static_cast<int>(p.own_cap)};
    const int64_t tiles = n + tile_bound(static_cast<int64_t>(n) * (n_heads / a.kv_heads), n_groups, 16);    // of either launch, at most
    if (tiles * (a.slots + 1) * a.kv_heads >= (1 << 26)) return ARROL_EINVAL;      // lanes of a launch are counted in 32 bits
    const auto st = static_cast<hipStream_t>(stream);
    if (n > 0) {
        if (a.hd <= 64) launch<64>(a, st);
        else launch<128>(a, st);
        const int64_t rows = static_cast<int64_t>(n) * n_heads;
        arrol_launch(decode_join_kernel, dim3(static_cast<unsigned>((rows + kWaves - 1) / kWaves)), dim3(kThreads), 0, st, a, static_cast<uint16_t*>(out), lse_out);
    }
    const auto blocks = [&](int pages) { return static_cast<unsigned>((static_cast<int64_t>(pages) * a.page + 63) / 64); };
    if (weight_out && n > 0) arrol_launch(decode_weight_kernel, dim3(blocks(max_pages_per_seq), n), dim3(kThreads), 0, st, a, a.own, 0, weight_in, weight_out);
    if (prefix_weight_out) arrol_launch(decode_weight_kernel, dim3(blocks(max_pages_per_prefix), n_groups), dim3(kThreads), 0, st, a, a.pre, 1, prefix_weight_in, prefix_weight_out);
    return arrol_launch_status();
}
