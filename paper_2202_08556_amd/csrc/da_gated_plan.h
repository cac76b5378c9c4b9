// Products of the gated feed-forward block, how each is cut into tiles and parts, and the scratch memory that this takes.
// Host code without device code: what a call reports and what it launches come from the same products here.
#pragma once
#include <algorithm>
#include <stddef.h>
#include <stdint.h>

namespace daspmm {

int compute_units() noexcept;

struct GatedShape {
    int64_t rows, d, h, dout;
};

enum { kStore = 0, kGate = 1, kGateGrad = 2 };   // what becomes of a product's sums
constexpr int kLineBytes = 128;  // of the inner axis in a tile
constexpr int kWideColumns = 256;

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline size_t round16(size_t n) { return (n + 15) & ~(size_t)15; }

// M x N numbers (kGate: two of each), sums over `segments` pairs of operands with an inner axis of K; `batches` of them.
// few: the outer positions are rows of the input, not a weight's.
struct Product {
    int64_t M, N, K;
    int segments, batches, epi;
    bool few;
};

inline Product gate_product(const GatedShape& s) { return {s.rows, s.h, s.d, 1, 1, kGate, true}; }
inline Product down_product(const GatedShape& s) { return {s.rows, s.dout, s.h, 1, 1, kStore, true}; }
inline Product hidden_grad_product(const GatedShape& s) { return {s.rows, s.h, s.dout, 1, 1, kGateGrad, true}; }
inline Product input_grad_product(const GatedShape& s) { return {s.rows, s.d, s.h, 2, 1, kStore, true}; }
// both weights' gradients, or one of them
inline Product up_grad_product(const GatedShape& s, int batches) { return {s.d, s.h, s.rows, 1, batches, kStore, false}; }
inline Product down_grad_product(const GatedShape& s) { return {s.h, s.dout, s.rows, 1, 1, kStore, false}; }

// Tile of a product, and how its sum is cut.  A tile of 128 x 128 has the most products for what it reads; tiles of 64 x 64
// are taken where the larger ones would leave much of the chip idle in their last turn (1531 x 602 out of 1187 float32: 60
// large tiles, 240 small ones), and no more rows or columns than there are.  Where even these are fewer than the units, the
// inner axis is cut, in parts of at least eight tiles of it (sixteen where it makes two parts at most).
struct GemmPlan {
    int BM, BN;
    int splits, per;
};

// size: bytes of a number
inline GemmPlan gemm_plan(const Product& g, int size) {
    GemmPlan p{};
    const int64_t width = g.epi == kGate ? 2 * g.N : g.N, cus = compute_units();
    auto tiles = [&](int64_t bm, int64_t bn) { return ceil_div(g.M, bm) * ceil_div(width, bn) * g.batches; };
    p.BM = g.M <= 16 ? 16 : g.M <= 32 ? 32 : g.M <= 64 ? 64 : 128;
    p.BN = 128;
    if (p.BM == 128) {
        if (width <= 64 && g.epi != kGate) p.BN = 64;
        else if (10 * ceil_div(tiles(128, 128), cus) > 3 * ceil_div(tiles(64, 64), cus)) p.BM = p.BN = 64;
    } else if (p.BM == 64 && tiles(64, 128) < cus) {
        p.BN = 64;
    }
    const int64_t count = tiles(p.BM, p.BN), inner = ceil_div(g.K, kLineBytes / size) * g.segments;
    int64_t splits = 1;
    if (count <= cus) splits = std::min(2 * cus / std::max<int64_t>(count, 1), std::max<int64_t>(1, inner / (2 * count <= cus ? 8 : 16)));
    p.per = (int)std::max<int64_t>(1, ceil_div(inner, std::max<int64_t>(splits, 1)));
    p.splits = (int)std::max<int64_t>(1, ceil_div(inner, p.per));
    return p;
}

// bfloat16, where the tiles' loads may be of whole pieces: 256 x 256 where there are enough tiles of it, otherwise 128 x 256,
// two blocks to a compute unit, where these are enough (33558 x 216 x 984 forward: 134 us with the smaller tiles, 107 so).
// Up to 128 rows the weights' stream is the bound: the inner axis is cut in parts of 512 positions and more until the chip
// is full (79 x 2168 x 9560 forward: 102 and 66 us).  Cutting other products cost more than it gave (backward of 1024 x 1024 x
// 4096: 200 and 248 us both ways).
struct WidePlan {
    int rows;                    // 256, 128; 0: not taken
    int splits;
};

inline WidePlan wide_plan(const Product& g) {
    const int64_t width = g.epi == kGate ? 2 * g.N : g.N, cus = compute_units();
    auto tiles = [&](int64_t rows) { return ceil_div(g.M, rows) * ceil_div(width, kWideColumns) * g.batches; };
    if (tiles(256) >= cus) return WidePlan{256, 1};
    const int64_t count = tiles(128);
    if (count >= cus) return WidePlan{128, 1};
    const int64_t splits = std::max<int64_t>(1, std::min(2 * cus / count, g.K * g.segments / 512));
    return g.few && g.M > 16 && g.M <= 128 && count * splits >= cus ? WidePlan{128, (int)splits} : WidePlan{0, 1};
}

// Threads side by side in a launch of a product, whichever kernels take it
inline int64_t launch_threads(const Product& g, int size) {
    if (g.M == 0 || g.N == 0) return 0;
    const int64_t width = g.epi == kGate ? 2 * g.N : g.N;
    const GemmPlan p = gemm_plan(g, size);
    const int64_t threads = ceil_div(g.M, p.BM) * ceil_div(width, p.BN) * (p.BM == 128 && p.BN == 128 ? 512 : 256);
    const WidePlan w = size == 2 ? wide_plan(g) : WidePlan{0, 1};
    return w.rows ? std::max(threads, ceil_div(g.M, w.rows) * ceil_div(width, kWideColumns) * 2 * w.rows) : threads;
}

// Whether every launch can be counted: of 2^32 threads and more the high bits are lost
inline bool gated_fits(const GatedShape& s, int size) {
    if (std::max({s.rows, s.d, s.h, s.dout}) <= 1 << 17) return true;    // 2^11 x 2^12 tiles at most, of 256 threads
    for (const Product& g : {gate_product(s), down_product(s), hidden_grad_product(s), input_grad_product(s), up_grad_product(s, 1),
                             up_grad_product(s, 2), down_grad_product(s)})
        if (launch_threads(g, size) >= 1LL << 32) return false;
    return true;
}

// Scratch of a product: its parts, whichever kernels take it
inline size_t part_bytes(const Product& g, int size) {
    if (g.M == 0 || g.N == 0) return 0;
    int splits = gemm_plan(g, size).splits;
    if (size == 2) splits = std::max(splits, wide_plan(g).splits);
    return splits > 1 ? (size_t)g.batches * splits * g.M * g.N * (g.epi == kGate ? 2 : 1) * sizeof(float) : 0;
}

// Parts of a backward pass, one product's at a time.  One weight's gradient alone is half the tiles of both and may be cut
// further: neither covers the other.
inline size_t backward_part_bytes(const GatedShape& s, int size) {
    return std::max({part_bytes(hidden_grad_product(s), size), part_bytes(input_grad_product(s), size), part_bytes(up_grad_product(s, 1), size),
                     part_bytes(up_grad_product(s, 2), size), part_bytes(down_grad_product(s), size)});
}

}  // namespace daspmm
