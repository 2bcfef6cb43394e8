// What a call of the log-prob gradient takes (host code alone, without a GPU or its headers): pieces of tokens and vocabulary, tiles, parts of K extents, and the workspace
// that holds them.
#pragma once
#include <cstddef>
#include <cstdint>

namespace logprob_grad {

constexpr int64_t kPieceRows = 16384;              // tokens of a piece
constexpr int64_t kPieceElements = int64_t{1} << 28;     // of dz
constexpr int kFoundTokens = 1024;                 // of a piece, that the workgroups of the first product look through by themselves
// An LM head of more elements than these is more than the 256 MiB cache holds, and so is its gradient: that goes past the caches, where its lines would have to be written back
// while the next call reads (16 x 151,936 x 2048, calls one after the other: dz 191 us, so 132; the call 532 and 491.  128 tokens: 608 and 551).
constexpr int64_t kCachedElements = int64_t{1} << 27;
constexpr int kResidentSteps = 5, kResidentTokens = kResidentSteps * 64;

inline size_t up(size_t bytes) { return (bytes + 255) / 256 * 256; }
inline int64_t up256(int64_t n) { return (n + 255) / 256 * 256; }

// Which forms a piece takes, of dz and of the products: those whose estimated times are the smallest.  Measured, microseconds: what a tile costs beside its K64
// steps, a step where the chip is full (of every one of the `per_unit` workgroups that a compute unit has at a time) and a step where it is not.  1,024 x 32,000 x 2048:
// dz 111 / 154 / 148 / 197 / 220, products 245 / 249 / 246 / 293 / 446; 640 tokens of it: 103 / 91 / 107 / 122 / 137 and 175 / 158 / 166 / 193 / 276; 318 x 4,096 x 256:
// 14.9 / 11.4 / 9.7 / 7.9 / 7.4 and 19.4 / 10.0 / 9.3 / 9.2 / 6.8; 16 x 151,936 x 2048 (LM head from memory, and its gradient to it): dz in 128 x 160 150, 128 x 64 132, 64 x 64 135.
// Next to the edges of the forms, whole calls with d = 2048, as chosen and with another form taken out: 321 x 128,256 749 and 740 (without 128 x 128), 321 x 151,936 882 and 878 .. 886,
// 384 x 32,000 187 and 187 .. 202, 384 x 151,936 905 and 881 (without 128 x 128), 311 x 128,256 612 and 660 (without 128 x 160); not at 192 tokens, where dL/dh in 128 x 64 costs 7 %
// (192 x 128,256 510 and 474 without it, 192 x 151,936 611 and 576).
enum Form { kRing, kMid160, kMid128, kMidFew, kMid64, kForms };
struct Size {
    int bm, bn, bm_w, bn_w;         // of dz and dL/dh, and of dL/dW
    int per_unit;
    double tile, step, lone, tile_w, step_w, lone_w;
};
constexpr Size kSize[kForms] = {{256, 256, 256, 256, 1, 8.7, 1.45, 1.1, 10.0, 1.55, 1.1}, {128, 160, 128, 128, 2, 5.5, 1.07, 0.6, 4.2, 0.95, 0.53}, {128, 128, 128, 128, 2, 4.8, 0.95, 0.53, 4.2, 0.95, 0.53},
                                {128, 64, 128, 128, 2, 1.7, 0.66, 0.33, 4.2, 0.95, 0.53}, {64, 64, 64, 64, 3, 1.4, 0.57, 0.2, 2.0, 0.6, 0.2}};

constexpr int kMaxSlabs = 32, kSlabTiles = 512;     // of 256 x 256
constexpr int64_t kSlabFloats = kSlabTiles * int64_t{65536};
static_assert(kSlabFloats / 2 <= kCachedElements, "a gradient that goes past the caches has no parts");
// From so many blocks of 64 x 256 on, seven to a compute unit, the hidden states' way into the registers is worth it.  The launch of the products, resident and in tiles: 311 x 151,936 x 2048
// (19,000 blocks) 457 us and 600, 16 tokens 260 and 335, 110 x 79,125 x 3264 228 and 272, 300 x 32,000 x 1024 (2,000) 54 and 61; 250 x 20,000 x 1000 (1,252) 38.4 and 34.8, 320 x 16,384 x 512
// (512) 22.7 and 19.8.  Whole calls of 320 tokens, as many as there are registers for: x 128,256 x 2048 610 and 699, x 151,936 x 2048 711 and 845; of 192 608 and 700.
constexpr int kResidentBlocks = 1792;
constexpr double kJoin = 3.5, kJoinBytes = 3e6;      // microseconds; bytes a microsecond

struct Pieces {
    int64_t rows, n_rows;           // tokens of a piece, pieces
    int64_t v, n_v;                 // vocabulary rows of a piece (a multiple of 256), pieces: as many as kPieceElements allow
    Form dz, products;
    int slabs, k64_per_slab;        // parts of the vocabulary piece that dL/dh's K extent is cut into, and their steps
    int parts;                      // of the tokens that dL/dW's is
    int blocks;                     // of 64 vocabulary rows to a workgroup of the resident form of dL/dW, 0: the tiles of `products`
};
inline int64_t tiles_of(int64_t n, int64_t m, int bn, int bm) { return ((n + bn - 1) / bn) * ((m + bm - 1) / bm); }

inline double dz_time(const Size& f, int64_t rows, int64_t v, int64_t d) {
    const double steps = static_cast<double>((d + 63) / 64), r = static_cast<double>(tiles_of(rows, v, f.bn, f.bm)) / (256 * f.per_unit);
    if (r <= 1) return f.tile + steps * (f.lone > f.step * r ? f.lone : f.step * r);
    const double up = static_cast<double>(static_cast<int64_t>(r + 0.999));
    return (up < r + 0.5 ? up : r + 0.5) * (f.tile + steps * f.step);       // of many rounds the last one's workgroups start early
}
// blocks: of the resident form of dL/dW, 0: tiles.  The resident form, two workgroups to a compute unit: 3.0 + 2.0 for every 64 tokens to fetch the hidden states, 3.0 + 0.5 a block; alone on
// it 2.0 + 1.0 and 1.2 + 0.2.
inline double products_time(const Size& f, int64_t rows, int64_t v, int64_t d, int slabs, int parts, int blocks) {
    const double n_h = static_cast<double>(tiles_of(rows, d, f.bn, f.bm) * slabs), n_w = static_cast<double>(blocks ? tiles_of(v, d, 64 * blocks, 256) : tiles_of(v, d, f.bn_w, f.bm_w) * parts);
    const double k_h = static_cast<double>((v / 64 + slabs - 1) / slabs), k_w = static_cast<double>(((rows + 63) / 64 + parts - 1) / parts), places = 256.0 * (blocks ? 2 : f.per_unit);
    const double each_w = blocks ? 3.0 + 2.0 * k_w + blocks * (3.0 + 0.5 * k_w) : f.tile_w + k_w * f.step_w;
    const double lone_h = f.tile + k_h * f.lone, lone_w = blocks ? 2.0 + k_w + blocks * (1.2 + 0.2 * k_w) : f.tile_w + k_w * f.lone_w, longest = lone_h > lone_w ? lone_h : lone_w;
    const double all = (n_h * (f.tile + k_h * f.step) + n_w * each_w) / places;
    return n_h + n_w <= places ? (all > longest ? all : longest) : all + longest / 2;
}
// fp32 values kept for the sums of dL/dW's parts: parts are taken only where there are some, so where two whole gradients fit, whatever the pieces and the estimates.
inline int64_t part_floats(int64_t T, int64_t V, int64_t d) {
    const int64_t head = up256(V) * d;
    if (T <= 256 || 2 * head > kSlabFloats) return 0;
    return kMaxSlabs * head < kSlabFloats ? kMaxSlabs * head : kSlabFloats;
}
inline void choose_forms(Pieces& p, int64_t T, int64_t V, int64_t d, const Size* sizes) {
    double best_dz = 1e30, best = 1e30;
    const int64_t floats = part_floats(T, V, d);
    for (int f = 0; f < kForms; ++f) {
        const Size& size = sizes[f];
        const double dz = f == kRing && d % 64 ? 1e30 : dz_time(size, p.rows, p.v, d);
        if (dz < best_dz) best_dz = dz, p.dz = static_cast<Form>(f);
        // parts of dL/dW's K extent where that is long and its tiles are few: as many as fill the chip, of 8 steps at least
        const int64_t tiles_w = tiles_of(p.v, d, size.bn_w, size.bm_w), k_w = (p.rows + 63) / 64;
        int64_t parts = f != kRing && k_w >= 32 && tiles_w < 256 ? 512 / tiles_w : 1;
        parts = parts < k_w / 8 ? parts : k_w / 8;
        parts = parts < kMaxSlabs ? parts : kMaxSlabs;
        if (parts * p.v * d > floats) parts = floats / (p.v * d);
        const int64_t tile = static_cast<int64_t>(size.bm) * size.bn, tiles = tiles_of(p.rows, d, size.bn, size.bm), k64 = p.v / 64;
        const bool resident = f != kRing && p.rows <= kResidentTokens && tiles_of(p.v, d, 64, 256) >= kResidentBlocks;
        for (int with = 0; with < 5; ++with) {          // 0: one part, 1: those parts, 2 ..: resident hidden states and 4, 8 or 16 blocks
            if ((with == 1 && parts < 2) || (with > 1 && !resident)) continue;
            const int n = with == 1 ? static_cast<int>(parts) : 1, blocks = with > 1 ? 1 << with : 0;
            for (int s = 1; s <= kMaxSlabs; s += s < 4 ? 1 : s / 4) {
                if (s > 1 && (s > k64 / 2 || s * tiles * tile > kSlabFloats)) break;
                const bool join_h = s > 1 || p.n_v > 1;
                const double join = join_h || with == 1 ? kJoin + ((join_h ? 4.0 * s * p.rows * d : 0.0) + (with == 1 ? 4.0 * n * p.v * d : 0.0)) / kJoinBytes : 0.0;
                const double t = products_time(size, p.rows, p.v, d, s, n, blocks) + join;
                if (t < best) best = t, p.products = static_cast<Form>(f), p.slabs = s, p.parts = n, p.blocks = blocks;
            }
        }
    }
}
inline Pieces pieces(int64_t T, int64_t V, int64_t d, const Size* sizes = kSize) {
    Pieces p;
    p.n_rows = (T + kPieceRows - 1) / kPieceRows;
    p.rows = (T + p.n_rows - 1) / p.n_rows;
    const int64_t most = kPieceElements / up256(p.rows) / 256 * 256, all = up256(V);
    p.n_v = (all + most - 1) / most;
    p.v = up256((all + p.n_v - 1) / p.n_v);
    p.n_v = (all + p.v - 1) / p.v;
    choose_forms(p, T, V, d, sizes);
    const int64_t k64 = ((V < p.v ? V : p.v) + 63) / 64;      // of the first piece, no part of which may be empty
    p.k64_per_slab = static_cast<int>((k64 + p.slabs - 1) / p.slabs);
    p.slabs = static_cast<int>((k64 + p.k64_per_slab - 1) / p.k64_per_slab);
    return p;
}

inline bool found_by_dz(const Pieces& p, int64_t rows) { return p.dz != kRing && rows <= kFoundTokens && p.n_v == 1; }

struct Workspace {
    size_t H, g, lse, target, row, rest, n_active, dz, slabs, slabs_w, sum, bytes;
};
// Sizes that no smaller batch exceeds.
inline Workspace workspace(int64_t T, int64_t V, int64_t d, bool lm_head) {
    Workspace w;
    const int64_t rows = T < kPieceRows ? T : kPieceRows, all = up256(rows) * up256(V);
    const int64_t one = rows * d, many = kMaxSlabs * one < kSlabFloats ? kMaxSlabs * one : kSlabFloats;      // one slab, or kSlabTiles tiles at most
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t was = at; at += up(bytes); return was; };
    w.n_active = take(4);
    w.g = take(rows * 4), w.lse = take(rows * 4), w.target = take(rows * 4), w.row = take(rows * 4), w.rest = take(rows * 4);
    w.H = take(up256(rows) * d * 2);
    w.dz = take((all < kPieceElements ? all : kPieceElements) * 2);
    w.slabs = take((one > many ? one : many) * 4);
    w.slabs_w = take(part_floats(T, V, d) * 4);
    w.sum = take(lm_head && T > kPieceRows ? V * d * 4 : 0);
    w.bytes = at;
    return w;
}

inline bool sizes_ok(int64_t T, int64_t V, int64_t d) { return T >= 0 && T < (int64_t{1} << 40) && V >= 1 && V <= (1 << 24) && d >= 8 && d % 8 == 0 && d <= 16384; }

}  // namespace logprob_grad
