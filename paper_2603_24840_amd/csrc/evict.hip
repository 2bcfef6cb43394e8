// Cuts rollouts' caches to a budget of tokens: the first and the most recent ones stay, and of those between them the ones that have
// gathered the most attention weight.
//
// Two launches.  plan: a workgroup a table row finds the smallest weight that stays (radix selection, 8 bits a pass over order-preserving integers, so
// the choice is exact and ties go to the lowest index), then, in index order, the kept tokens behind the cut and the freed slots before it;
// the k-th of the ones goes to the k-th of the others, so no token that lies right already is touched and no source is ever a
// destination.  copy: the moves, in every layer, K and V, 16 bytes a lane; bound by HBM.
#include "common.h"

namespace {

constexpr int kPlanThreads = 1024;       // of the larger form
constexpr int kCopyThreads = 256, kCopyMoves = 32, kInFlight = 8;

struct Move { int64_t from, to; };      // places (page * page_tokens + offset) of a token; -1: a page id out of range

struct Evict {
    const int32_t *table, *len, *position;
    const float* weight;
    int32_t *table_out, *len_out, *position_out;
    float* weight_out;
    Move* moves;
    int32_t *from, *to, *count;     // the same moves as token indices; how many
    int64_t n_pages;
    int per_row, page, budget, first, recent, most;
};

// Larger weights are larger integers; NaN lies below everything, -0 is 0.
__device__ __forceinline__ uint32_t order_of(float w) {
    if (w != w) return 0;
    const uint32_t u = __float_as_uint(w == 0.f ? 0.f : w);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// How many of the workgroup's threads before this one have `flag` set, and (in total) how many have it at all.
template <int WAVES>
__device__ __forceinline__ int rank_in_block(bool flag, int* totals, int& total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint64_t votes = __ballot(flag);
    __syncthreads();                       // totals of the last call are read
    if (lane == 0) totals[wave] = __popcll(votes);
    __syncthreads();
    int before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        before += w < wave ? totals[w] : 0;
        total += totals[w];
    }
    return before + __popcll(votes & ((uint64_t{1} << lane) - 1));
}

// THREADS: 256 for rows of up to 512 tokens, whose barriers are the time (32 rows of 64: 9.0 us a call, with 1,024 threads 9.5), 1,024 for longer ones
// (128 rows of 1,024: 225 us, with 256 threads 227.5).
template <int THREADS>
__global__ __launch_bounds__(THREADS) void evict_plan_kernel(Evict a) {
    constexpr int kWaves = THREADS / ARROL_WAVE;
    __shared__ int bins[256], totals[kWaves];
    __shared__ uint32_t digit_found;
    __shared__ int left_over;
    const int row = blockIdx.x, tid = threadIdx.x;
    const int cap = a.per_row * a.page;
    const int64_t base = static_cast<int64_t>(row) * cap;
    int len = a.len[row];
    len = len < 0 ? 0 : len < cap ? len : cap;
    const int left = len < a.budget ? len : a.budget;
    const float* weight = a.weight + base;
    const int32_t* table = a.table + static_cast<int64_t>(row) * a.per_row;
    const int lo = a.first, hi = len - a.recent;       // what is chosen from, where anything goes at all
    int moved = 0;
    if (left < len) {
        uint32_t prefix = 0, mask = 0;
        int need = left - a.first - a.recent;
        if (need > 0) {
            for (int shift = 24; shift >= 0; shift -= 8) {
                if (tid < 256) bins[tid] = 0;
                __syncthreads();
                for (int t = lo + tid; t < hi; t += THREADS) {
                    const uint32_t u = order_of(weight[t]);
                    if ((u & mask) == prefix) atomicAdd(&bins[u >> shift & 255], 1);
                }
                __syncthreads();
                if (tid < 64) {            // lane i has bins 255 - 4 i and the three below; how many lie above them
                    int mine[4], sum = 0;
#pragma unroll
                    for (int i = 0; i < 4; ++i) mine[i] = bins[255 - 4 * tid - i], sum += mine[i];
                    int above = static_cast<int>(wave_scan_sum(static_cast<int64_t>(sum))) - sum;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        if (above < need && above + mine[i] >= need) {
                            digit_found = 255 - 4 * tid - i;
                            left_over = need - above;
                        }
                        above += mine[i];
                    }
                }
                __syncthreads();
                prefix |= digit_found << shift;
                mask |= 0xffu << shift;
                need = left_over;
                __syncthreads();
            }
        } else {
            prefix = 0xffffffffu;          // above every weight
        }
        // what stays: larger than the smallest one that stays, and the first `need` of its equals
        int ties = 0, freed = 0;
        for (int start = 0; start < len; start += THREADS) {
            const int t = start + tid;
            const bool between = t >= lo && t < hi;
            const uint32_t u = between ? order_of(weight[t]) : 0;
            const bool tie = between && u == prefix;
            int total;
            const int rank = ties + rank_in_block<kWaves>(tie, totals, total);
            ties += total;
            const bool stays = t < len && (!between || u > prefix || (tie && rank < need));
            const bool mover = stays && t >= left, hole = !stays && t < left;
            const int place = rank_in_block<kWaves>(mover, totals, total) + moved;
            moved += total;
            const int slot = rank_in_block<kWaves>(hole, totals, total) + freed;
            freed += total;
            if (mover || hole) {
                const int id = table[t / a.page];
                const int64_t at = id >= 0 && id < a.n_pages ? static_cast<int64_t>(id) * a.page + t % a.page : -1;
                const int64_t k = static_cast<int64_t>(row) * a.most + (mover ? place : slot);
                if (mover) a.moves[k].from = at, a.from[k] = t;
                else a.moves[k].to = at, a.to[k] = t;
            }
        }
        __syncthreads();
    }
    if (tid == 0) a.count[row] = moved;
    // The outputs may be the inputs: what moves is read (behind the cut) before anything there is cleared.
    const int32_t* position = a.position ? a.position + base : nullptr;
    int32_t* position_out = a.position_out + base;
    float* weight_out = a.weight_out + base;
    for (int t = tid; t < left; t += THREADS) {
        weight_out[t] = weight[t];
        position_out[t] = position ? position[t] : t;
    }
    __syncthreads();
    for (int k = tid; k < moved; k += THREADS) {
        const int64_t at = static_cast<int64_t>(row) * a.most + k;
        const int from = a.from[at], to = a.to[at];
        weight_out[to] = weight[from];
        position_out[to] = position ? position[from] : from;
    }
    __syncthreads();
    for (int t = left + tid; t < cap; t += THREADS) {
        weight_out[t] = 0.f;
        position_out[t] = -1;
    }
    const int pages = (left + a.page - 1) / a.page;
    for (int p = tid; p < a.per_row; p += THREADS) a.table_out[static_cast<int64_t>(row) * a.per_row + p] = p < pages ? table[p] : -1;
    if (tid == 0) a.len_out[row] = left;
}

// The moves, 32 of a row to a workgroup and 8 loads of a lane in flight before its stores; consecutive workgroups take the same moves in every slab (layer, K or
// V), so the moves are read once and what is in flight lies far apart.  128 rows of 1 KiB tokens, 16 layers: 224 us a call; with a slab's moves one after the
// other 243, and with 16 moves and 4 loads 266.
__global__ __launch_bounds__(kCopyThreads) void evict_copy_kernel(unsigned char* __restrict__ kv, const Move* __restrict__ moves, const int32_t* __restrict__ count,
                                                                  int most, int groups, int slabs, int64_t blocks, int64_t slab_bytes, int vecs) {
    const int64_t token_bytes = static_cast<int64_t>(vecs) * 16;
    for (int64_t block = blockIdx.x; block < blocks; block += gridDim.x) {
        const int64_t which = block % slabs, rest = block / slabs;
        const int group = static_cast<int>(rest % groups), row = static_cast<int>(rest / groups);
        const int first = group * kCopyMoves, left = count[row] - first;
        if (left <= 0) continue;
        const int total = (left < kCopyMoves ? left : kCopyMoves) * vecs;
        const Move* mine = moves + static_cast<int64_t>(row) * most + first;
        unsigned char* slab = kv + which * slab_bytes;
        for (int base = threadIdx.x; base < total; base += kCopyThreads * kInFlight) {
            u32x4 x[kInFlight];
            int64_t to[kInFlight];
#pragma unroll
            for (int i = 0; i < kInFlight; ++i) {
                const int at = base + i * kCopyThreads;
                to[i] = -1;
                if (at < total) {
                    const Move m = mine[at / vecs];
                    if (m.from >= 0 && m.to >= 0) {
                        const int64_t within = at % vecs * 16;
                        x[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(slab + m.from * token_bytes + within));
                        to[i] = m.to * token_bytes + within;
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < kInFlight; ++i)
                if (to[i] >= 0) __builtin_nontemporal_store(x[i], reinterpret_cast<u32x4*>(slab + to[i]));
        }
    }
}

size_t up(size_t bytes) { return (bytes + 255) / 256 * 256; }

// Moves of a row at most: as many as slots before the cut, and as tokens behind it.
int64_t most_moves(int64_t cap, int64_t budget) { return cap <= budget ? 0 : cap - budget < budget ? cap - budget : budget; }

size_t workspace(int64_t rows, int64_t most) { return up(rows * most * sizeof(Move)) + 2 * up(rows * most * 4) + up(rows * 4); }

bool shape_ok(int64_t rows, int64_t per_row, int64_t page, int64_t budget) {
    return rows >= 0 && rows < (1 << 22) && per_row >= 1 && page >= 1 && budget >= 0 && per_row <= (0x7fffffff - kPlanThreads) / page;
}

}  // namespace

extern "C" size_t arrol_evict_workspace_bytes(int32_t n_rows, int32_t max_pages_per_seq, int32_t page_tokens, int32_t budget) {
    if (n_rows <= 0 || !shape_ok(n_rows, max_pages_per_seq, page_tokens, budget)) return 0;
    return workspace(n_rows, most_moves(static_cast<int64_t>(max_pages_per_seq) * page_tokens, budget));
}

extern "C" int arrol_evict(void* kv, arrol_kv_layout layout, const int32_t* block_table, const int32_t* seq_len, int32_t n_rows, int32_t max_pages_per_seq,
                           const float* weight, const int32_t* position, int32_t budget, int32_t n_first, int32_t n_recent, int32_t* block_table_out,
                           int32_t* seq_len_out, float* weight_out, int32_t* position_out, void* workspace_, size_t workspace_bytes, void* stream) {
    const int64_t token_bytes = static_cast<int64_t>(layout.n_kv_heads) * layout.head_dim * 2;
    if (!shape_ok(n_rows, max_pages_per_seq, layout.page_tokens, budget) || layout.n_layers < 1 || layout.n_layers > (1 << 24) || layout.n_kv_heads < 1 || layout.head_dim < 1 || layout.n_pages < 0) return ARROL_EINVAL;
    if (token_bytes % 16 || token_bytes > (1 << 24) || n_first < 0 || n_recent < 0 || static_cast<int64_t>(n_first) + n_recent > budget) return ARROL_EINVAL;
    if (n_rows == 0) return ARROL_OK;
    if (!block_table || !seq_len || !weight || !block_table_out || !seq_len_out || !weight_out || !position_out) return ARROL_EINVAL;
    if (layout.n_pages > 0 && (!kv || !arrol_aligned16(kv))) return ARROL_EINVAL;
    const int64_t cap = static_cast<int64_t>(max_pages_per_seq) * layout.page_tokens, most = most_moves(cap, budget);
    if (!workspace_ || !arrol_aligned16(workspace_) || workspace_bytes < workspace(n_rows, most)) return ARROL_EWORKSPACE;
    auto* ws = static_cast<unsigned char*>(workspace_);
    Evict a;
    a.moves = reinterpret_cast<Move*>(ws), ws += up(n_rows * most * sizeof(Move));
    a.from = reinterpret_cast<int32_t*>(ws), ws += up(n_rows * most * 4);
    a.to = reinterpret_cast<int32_t*>(ws), ws += up(n_rows * most * 4);
    a.count = reinterpret_cast<int32_t*>(ws);
    a.table = block_table, a.len = seq_len, a.position = position, a.weight = weight;
    a.table_out = block_table_out, a.len_out = seq_len_out, a.position_out = position_out, a.weight_out = weight_out;
    a.n_pages = layout.n_pages, a.per_row = max_pages_per_seq, a.page = layout.page_tokens;
    a.budget = budget, a.first = n_first, a.recent = n_recent, a.most = static_cast<int>(most);
    const auto st = static_cast<hipStream_t>(stream);
    if (cap <= 512) arrol_launch(evict_plan_kernel<256>, dim3(n_rows), dim3(256), 0, st, a);
    else arrol_launch(evict_plan_kernel<kPlanThreads>, dim3(n_rows), dim3(kPlanThreads), 0, st, a);
    if (most > 0) {
        const int64_t groups = (most + kCopyMoves - 1) / kCopyMoves, blocks = groups * n_rows * layout.n_layers * 2;
        const int64_t slab = layout.n_pages * layout.page_tokens * token_bytes;
        const unsigned grid = static_cast<unsigned>(blocks < (1 << 23) ? blocks : (1 << 23));
        arrol_launch(evict_copy_kernel, dim3(grid), dim3(kCopyThreads), 0, st, static_cast<unsigned char*>(kv), a.moves, a.count, a.most, static_cast<int>(groups),
                     2 * layout.n_layers, blocks, slab, static_cast<int>(token_bytes / 16));
    }
    return arrol_launch_status();
}
