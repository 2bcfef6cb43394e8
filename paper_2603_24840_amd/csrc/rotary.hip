// Positions of queries and keys, and new tokens into the paged KV pool (gfx950, wave64).
//
// A head's elements below 2 * half are turned pair by pair by the angle position * inv_freq[pair]:
//   x' = m (x cos - y sin),  y' = m (x sin + y cos)        (m: magnitude; the inverse, which is the gradient, takes -sin)
// with pairs (i, i + half), or (2i, 2i + 1) where they are interleaved.  The angle is formed in turns and 64 bits and only what is left of it after
// whole turns is rounded to 32: at position 10^6 a 32-bit product is off by up to 0.03 radians.  Cosine and sine are those of the remaining half turns; a result is rounded once.
//
// A wavefront takes a token, or a part of its heads where tokens are few: it loads first, forms the cosines and sines of the token, one pair to a lane, while the loads are
// under way, hands them over through its own part of the LDS and stores.  No barrier.  What a lane holds is a unit: VEC elements and their partners, or 2 VEC
// elements side by side of the rest of the head or of an interleaved one, loaded and stored by that lane alone, so an output may be its input.
//
// Bound by memory: 11,136 tokens of 32 + 8 heads of 128 42.5 us (228 MB, 5.4 TB/s; torch's copy of 4 GiB 4.6 to 5.0), prompts into the pool with their keys kept 46.8 us (4.95 TB/s),
// 6,426 tokens with heads of 80, 40 of them turned, 21.1 us (3.9 TB/s: accesses of 8 bytes, of the part that is not turned, too).  Few tokens: one launch, 3.5 to 4.6 us.
#include "common.h"

namespace {

constexpr int kWaves = 4;                 // of a workgroup
// Units of a lane in flight, and wavefronts that a launch is cut into where tokens are fewer.  11,136 tokens, 32 + 8 heads of 128, from and to memory: 2 and 65,536 42.6 us
// (5.4 TB/s), 4 and 8,192 40.9, but half of the head turned, in pairs, 40.6 and 42.9; loads through the caches 46.4; stores past the caches too: 41.2, but the attention behind
// it 8 longer.  Into the pool, where every wavefront looks for its token's page: 6,426 tokens of 24 + 8 heads of 80, 3 and 8,192 21.1 us, 2 and 65,536 25.8, 4 and 65,536 32.8; prompts with their keys kept 46.9, 51.9 and 72.0.  Accesses of 16
// bytes at multiples of 8 where the second half begins there, with a short last unit, were a quarter slower (29.5 and 23.8 in a loop over one call).  Loads through the caches: the heads of
// 80 18.7 us, whose 8 bytes a lane share lines, but the prompts 52.9.
template <bool POOL> constexpr int kUnits = POOL ? 3 : 2;
template <bool POOL> constexpr int kWavefronts = POOL ? 8192 : 65536;
constexpr int kMaxHalf = 128;

struct Turn {
    const uint16_t *q, *k, *v;            // q, v may be NULL
    int64_t q_stride, k_stride, v_stride;
    uint16_t *q_out, *k_out;              // may be NULL where there is a pool
    int64_t q_out_stride, k_out_stride;
    const int32_t* position;              // NULL: the token's slot
    const double* inv_freq;
    int64_t T;
    int heads, kv_heads, hd, half;        // heads: 0 without q
    int units, groups;                    // of a head; parts of a token
    float magnitude, sign;
    // the pool
    const int64_t* cu;                    // NULL: a token a row of the table
    const int32_t *start, *table;
    uint16_t *pool_k, *pool_v;            // of the layer
    int64_t n_pages;
    int n_seq, page, width;
};

template <int N> struct Elements { typedef unsigned short type __attribute__((ext_vector_type(N))); };
template <> struct Elements<1> { typedef unsigned short type; };

__device__ __forceinline__ float widen(uint16_t x) { return __uint_as_float(static_cast<uint32_t>(x) << 16); }
__device__ __forceinline__ uint16_t narrow(float x) { return __builtin_bit_cast(uint16_t, static_cast<__bf16>(x)); }
template <int N> __device__ __forceinline__ uint16_t at(const typename Elements<N>::type& x, int i) { return x[i]; }
template <> __device__ __forceinline__ uint16_t at<1>(const uint16_t& x, int) { return x; }
template <int N> __device__ __forceinline__ void put(typename Elements<N>::type& x, int i, uint16_t v) { x[i] = v; }
template <> __device__ __forceinline__ void put<1>(uint16_t& x, int, uint16_t v) { x = v; }

// A value that is the same in all lanes and that no kernel of the call writes, by way of the scalar cache: its wait is not one for the vector loads under way.
template <class T>
__device__ __forceinline__ T fetch(const T* p) { return *(const __attribute__((address_space(4))) T*)p; }

// How many of cu[0..n] are at most t, 64 of them to a step: cu ascends, and whatever it holds the answer is in [0, n + 1].  first: cu[min(lane, n)], which
// is all there is to look at up to 63 sequences.
__device__ __forceinline__ int64_t offsets_up_to(const int64_t* cu, int n, int64_t t, int lane, int64_t first) {
    int64_t lo = 0, hi = static_cast<int64_t>(n) + 1;
    if (hi <= ARROL_WAVE) return __popcll(__ballot(lane < hi && first <= t));
    while (hi - lo > ARROL_WAVE) {
        const int64_t step = (hi - lo + ARROL_WAVE - 1) / ARROL_WAVE, i = lo + lane * step;
        const int below = __popcll(__ballot(i < hi && cu[i < hi ? i : lo] <= t));
        if (below == 0) return lo;
        const int64_t end = lo + below * step;
        lo = end - step + 1;
        hi = end < hi ? end : hi;
    }
    const int64_t i = lo + lane;
    return lo + __popcll(__ballot(i < hi && cu[i < hi ? i : 0] <= t));
}

template <int VEC, bool INTERLEAVED, bool POOL>
__global__ __launch_bounds__(kWaves * ARROL_WAVE) void rotary_kernel(Turn a) {
    typedef typename Elements<VEC>::type vec;
    constexpr int kInFlight = kUnits<POOL>;
    __shared__ float2 turns[kWaves][kMaxHalf];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t item = static_cast<int64_t>(blockIdx.x) * kWaves + wave;
    const int64_t t = item / a.groups;
    const int group = static_cast<int>(item - t * a.groups);
    if (t >= a.T) return;
    int64_t offset = 0;
    if (POOL && a.cu) offset = a.cu[lane < a.n_seq ? lane : a.n_seq];

    const int n_turned = INTERLEAVED ? 0 : a.half / VEC;      // units of two halves; interleaved ones see for themselves
    const uint16_t *q = a.q + t * a.q_stride, *k = a.k + t * a.k_stride;
    uint16_t *q_out = a.q_out + t * a.q_out_stride, *k_out = a.k_out ? a.k_out + t * a.k_out_stride : nullptr;
    const int total = (a.heads + a.kv_heads) * a.units;
    const int stride = ARROL_WAVE * a.groups, d_head = stride / a.units, d_unit = stride - d_head * a.units;
    int u = group * ARROL_WAVE + lane, head = u / a.units, unit = u - head * a.units;
    // where a unit's two parts lie in their head; the last unit of the rest may lack its second
    auto first_of = [&](int unit) { return INTERLEAVED ? 2 * VEC * unit : unit < n_turned ? VEC * unit : 2 * a.half + 2 * VEC * (unit - n_turned); };
    auto second_of = [&](int unit) { return INTERLEAVED || unit >= n_turned ? first_of(unit) + VEC : a.half + VEC * unit; };

    vec x[kInFlight], y[kInFlight];
    int of_head[kInFlight], of_unit[kInFlight];
    auto load = [&]() {
#pragma unroll
        for (int i = 0; i < kInFlight; ++i) {
            of_head[i] = u < total ? head : -1;
            of_unit[i] = unit;
            if (u < total) {
                const uint16_t* row = head < a.heads ? q + head * a.hd : k + (head - a.heads) * a.hd;
                const int second = second_of(unit);
                x[i] = __builtin_nontemporal_load(reinterpret_cast<const vec*>(row + first_of(unit)));
                if (second < a.hd) y[i] = __builtin_nontemporal_load(reinterpret_cast<const vec*>(row + second));
            }
            u += stride;
            head += d_head;
            unit += d_unit;
            if (unit >= a.units) { unit -= a.units; ++head; }
        }
    };
    load();
    u32x4 v[kInFlight];
    const int n_v = a.kv_heads * a.hd / 8, v0 = group * ARROL_WAVE + lane;
    const uint16_t* values = POOL ? a.v + t * a.v_stride : nullptr;
    if (POOL) {
#pragma unroll
        for (int i = 0; i < kInFlight; ++i)
            if (v0 + i * stride < n_v) v[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(values + (v0 + i * stride) * 8));
    }

    // where the token goes, and its position
    int64_t slot = 0, to = -1;            // to: token of the pool
    bool known = true;                    // a row of a sequence
    if (POOL) {
        int64_t of = t, j = 0;
        if (a.cu) {
            of = offsets_up_to(a.cu, a.n_seq, t, lane, offset) - 1;
            known = of >= 0 && of < a.n_seq;
        }
        const int s = __builtin_amdgcn_readfirstlane(static_cast<int>(of));
        if (known) {
            if (a.cu) {
                const int64_t begin = fetch(a.cu + s);
                j = t - (begin > 0 ? begin : 0);
            }
            slot = fetch(a.start + s) + j;
            const int64_t p = slot / a.page;
            if (slot >= 0 && p < a.width) {
                const int32_t id = fetch(a.table + static_cast<int64_t>(s) * a.width + p);
                if (id >= 0 && id < a.n_pages) to = static_cast<int64_t>(id) * a.page + (slot - p * a.page);
            }
        }
    }
    const int half = known ? a.half : 0;
    if (half > 0) {
        const double p = a.position ? static_cast<double>(fetch(a.position + t)) : static_cast<double>(slot);
        for (int i = lane; i < half; i += ARROL_WAVE) {
            const double full = p * (a.inv_freq[i] * 0.15915494309189533577);     // 1 / 2 pi
            float s, c;
            sincospif(static_cast<float>(2.0 * (full - rint(full))), &s, &c);
            turns[wave][i] = make_float2(c * a.magnitude, s * a.magnitude * a.sign);
        }
        wave_lds_exchange();
    }
    uint16_t* pool_k = POOL && to >= 0 ? a.pool_k + to * a.kv_heads * a.hd : nullptr;

    for (;;) {
#pragma unroll
        for (int i = 0; i < kInFlight; ++i) {
            if (of_head[i] < 0) continue;
            const int first = first_of(of_unit[i]), second = second_of(of_unit[i]);
            auto turn = [&](int pair, auto get, auto set) {
                const float2 cs = turns[wave][pair];
                const float p = widen(get(0)), r = widen(get(1));
                set(0, narrow(p * cs.x - r * cs.y));
                set(1, narrow(p * cs.y + r * cs.x));
            };
            if (INTERLEAVED) {
#pragma unroll
                for (int e = 0; e < VEC; ++e) {       // pairs of x, then of y
                    vec& z = e < VEC / 2 ? x[i] : y[i];
                    const int at0 = 2 * (e % (VEC / 2)), pair = of_unit[i] * VEC + e;
                    if (pair < half) turn(pair, [&](int w) { return at<VEC>(z, at0 + w); }, [&](int w, uint16_t b) { put<VEC>(z, at0 + w, b); });
                }
            } else if (of_unit[i] < n_turned && half > 0) {
#pragma unroll
                for (int e = 0; e < VEC; ++e)
                    turn(of_unit[i] * VEC + e, [&](int w) { return at<VEC>(w ? y[i] : x[i], e); }, [&](int w, uint16_t b) { put<VEC>(w ? y[i] : x[i], e, b); });
            }
            auto store = [&](uint16_t* row) {
                *reinterpret_cast<vec*>(row + first) = x[i];
                if (second < a.hd) *reinterpret_cast<vec*>(row + second) = y[i];
            };
            const int kv_head = of_head[i] - a.heads;
            if (kv_head < 0) {
                store(q_out + of_head[i] * a.hd);
            } else {
                if (k_out) store(k_out + kv_head * a.hd);
                if (POOL && pool_k) store(pool_k + kv_head * a.hd);
            }
        }
        if (u - lane >= total) break;     // the same in all lanes
        load();
    }

    if (POOL && to >= 0) {
        uint16_t* pool_v = a.pool_v + to * a.kv_heads * a.hd;
#pragma unroll
        for (int i = 0; i < kInFlight; ++i)
            if (v0 + i * stride < n_v) *reinterpret_cast<u32x4*>(pool_v + (v0 + i * stride) * 8) = v[i];
        for (int i = v0 + kInFlight * stride; i < n_v; i += stride)
            *reinterpret_cast<u32x4*>(pool_v + i * 8) = *reinterpret_cast<const u32x4*>(values + i * 8);
    }
}

template <bool POOL>
int turn(Turn& a, bool interleaved, hipStream_t st) {
    const int vec = interleaved || a.half % 8 == 0 ? 8 : a.half % 4 == 0 ? 4 : a.half % 2 == 0 ? 2 : 1;
    a.units = interleaved ? (a.hd + 15) / 16 : a.half / vec + (a.hd - 2 * a.half + 2 * vec - 1) / (2 * vec);
    const int64_t most = (static_cast<int64_t>(a.heads + a.kv_heads) * a.units + ARROL_WAVE - 1) / ARROL_WAVE;
    const int64_t want = kWavefronts<POOL> / a.T;
    a.groups = static_cast<int>(want < 1 ? 1 : want < most ? want : most);
    const dim3 grid(static_cast<unsigned>((a.T * a.groups + kWaves - 1) / kWaves)), block(kWaves * ARROL_WAVE);
    if (interleaved) arrol_launch(rotary_kernel<8, true, POOL>, grid, block, 0, st, a);
    else if (vec == 8) arrol_launch(rotary_kernel<8, false, POOL>, grid, block, 0, st, a);
    else if (vec == 4) arrol_launch(rotary_kernel<4, false, POOL>, grid, block, 0, st, a);
    else if (vec == 2) arrol_launch(rotary_kernel<2, false, POOL>, grid, block, 0, st, a);
    else arrol_launch(rotary_kernel<1, false, POOL>, grid, block, 0, st, a);
    return arrol_launch_status();
}

bool rows_ok(const void* p, int64_t stride, int64_t heads, int64_t hd) {
    return p && arrol_aligned16(p) && stride % 8 == 0 && stride >= heads * hd && stride <= (1 << 24);
}
bool sizes_ok(int64_t T, int32_t hd, int32_t rotary_dim) {
    return T >= 0 && T < (int64_t{1} << 25) && hd >= 8 && hd % 8 == 0 && hd <= 2 * kMaxHalf && rotary_dim >= 2 && rotary_dim % 2 == 0 && rotary_dim <= hd;
}

}  // namespace

extern "C" int arrol_rotary_frequencies(int32_t rotary_dim, double base, double factor, double original_context, double low, double high, double* inv_freq) {
    if (!inv_freq || rotary_dim < 2 || rotary_dim % 2 || rotary_dim > 2 * kMaxHalf) return ARROL_EINVAL;
    if (!(base > 0 && base <= 1e300) || !(factor > 0 && factor <= 1e300) || !(original_context >= 0 && original_context <= 1e300) || !(low <= high && low >= -1e300 && high <= 1e300)) return ARROL_EINVAL;
    for (int i = 0; i < rotary_dim / 2; ++i) {
        const double f = pow(base, -2.0 * i / rotary_dim), turns = original_context * f * 0.15915494309189533577;
        const double s = turns >= high ? 1.0 : turns <= low ? 0.0 : (turns - low) / (high - low);
        inv_freq[i] = f * (s + (1.0 - s) / factor);
    }
    return ARROL_OK;
}

extern "C" int arrol_rotary(const void* q, int64_t q_stride, const void* k, int64_t k_stride, const int32_t* position, const double* inv_freq, int64_t T,
                            int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, int32_t rotary_dim, int32_t interleaved, int32_t inverse, float magnitude,
                            void* q_out, int64_t q_out_stride, void* k_out, int64_t k_out_stride, void* stream) {
    if (!sizes_ok(T, head_dim, rotary_dim) || n_heads < 1 || n_kv_heads < 0 || (n_kv_heads == 0) != (k == nullptr) || (k == nullptr) != (k_out == nullptr)) return ARROL_EINVAL;
    if (T == 0) return ARROL_OK;
    if (!position || !inv_freq || !rows_ok(q, q_stride, n_heads, head_dim) || !rows_ok(q_out, q_out_stride, n_heads, head_dim)) return ARROL_EINVAL;
    if (k && (!rows_ok(k, k_stride, n_kv_heads, head_dim) || !rows_ok(k_out, k_out_stride, n_kv_heads, head_dim))) return ARROL_EINVAL;
    Turn a = {};
    a.q = static_cast<const uint16_t*>(q), a.q_stride = q_stride, a.q_out = static_cast<uint16_t*>(q_out), a.q_out_stride = q_out_stride;
    a.k = static_cast<const uint16_t*>(k), a.k_stride = k_stride, a.k_out = static_cast<uint16_t*>(k_out), a.k_out_stride = k_out_stride;
    a.position = position, a.inv_freq = inv_freq, a.T = T, a.heads = n_heads, a.kv_heads = n_kv_heads, a.hd = head_dim, a.half = rotary_dim / 2;
    a.magnitude = magnitude, a.sign = inverse ? -1.f : 1.f;
    return turn<false>(a, interleaved != 0, static_cast<hipStream_t>(stream));
}

extern "C" int arrol_append(const void* k, int64_t k_stride, const void* v, int64_t v_stride, const void* q, int64_t q_stride, const int64_t* cu_seqlens,
                            const int32_t* start, const int32_t* position, const double* inv_freq, int64_t T, int32_t n_seq, int32_t n_heads,
                            int32_t rotary_dim, int32_t interleaved, float magnitude, void* kv, arrol_kv_layout layout, int32_t layer,
                            const int32_t* block_table, int32_t max_pages_per_seq, void* q_out, int64_t q_out_stride, void* k_out,
                            int64_t k_out_stride, void* stream) {
    if (!inv_freq) rotary_dim = 2;        // of no meaning
    if (!sizes_ok(T, layout.head_dim, rotary_dim) || n_seq < 0 || (!cu_seqlens && T != n_seq) || max_pages_per_seq < 1) return ARROL_EINVAL;
    if (layout.n_kv_heads < 1 || layout.page_tokens < 1 || layout.n_pages < 0 || layout.n_pages > 0x7fffffff / layout.page_tokens) return ARROL_EINVAL;
    if (layer < 0 || layer >= layout.n_layers || n_heads < 0 || (n_heads == 0) != (q == nullptr) || (q == nullptr) != (q_out == nullptr)) return ARROL_EINVAL;
    if (T == 0) return ARROL_OK;
    if (!rows_ok(k, k_stride, layout.n_kv_heads, layout.head_dim) || !rows_ok(v, v_stride, layout.n_kv_heads, layout.head_dim)) return ARROL_EINVAL;
    if (k_out && !rows_ok(k_out, k_out_stride, layout.n_kv_heads, layout.head_dim)) return ARROL_EINVAL;
    if (q && (!rows_ok(q, q_stride, n_heads, layout.head_dim) || !rows_ok(q_out, q_out_stride, n_heads, layout.head_dim))) return ARROL_EINVAL;
    if ((n_seq > 0 && (!start || !block_table)) || (layout.n_pages > 0 && (!kv || !arrol_aligned16(kv)))) return ARROL_EINVAL;
    Turn a = {};
    a.q = static_cast<const uint16_t*>(q), a.q_stride = q_stride, a.q_out = static_cast<uint16_t*>(q_out), a.q_out_stride = q_out_stride;
    a.k = static_cast<const uint16_t*>(k), a.k_stride = k_stride, a.k_out = static_cast<uint16_t*>(k_out), a.k_out_stride = k_out_stride;
    a.v = static_cast<const uint16_t*>(v), a.v_stride = v_stride;
    a.position = position, a.inv_freq = inv_freq, a.T = T, a.heads = n_heads, a.kv_heads = layout.n_kv_heads, a.hd = layout.head_dim;
    a.half = inv_freq ? rotary_dim / 2 : 0;
    a.magnitude = magnitude, a.sign = 1.f;
    const int64_t slab = layout.n_pages * layout.page_tokens * layout.n_kv_heads * layout.head_dim;
    a.cu = cu_seqlens, a.start = start, a.table = block_table, a.n_seq = n_seq, a.page = layout.page_tokens, a.width = max_pages_per_seq, a.n_pages = layout.n_pages;
    a.pool_k = static_cast<uint16_t*>(kv) + 2 * static_cast<int64_t>(layer) * slab, a.pool_v = a.pool_k + slab;
    return turn<true>(a, interleaved != 0, static_cast<hipStream_t>(stream));
}
