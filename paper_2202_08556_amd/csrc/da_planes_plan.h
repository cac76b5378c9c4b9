// How a product of packed matrices is cut into tiles and parts.  Host code without device code.
#pragma once
#include "da_gated_plan.h"

namespace daspmm {

constexpr int kMostParted = 1024;            // tiles whose sums are in parts

struct PlanePlan {
    int shape;                   // 0 large, 1 middle, 2 small
    int tiles_m, tiles_n;
    int64_t tiles;               // of a batch
    int splits, per;
};

// What tiles of a size cost, in us, as measured on products of 200 to 8192: a step of a block where at most half of the units have one,
// where each has at most one, and where they have two (the large tiles: one after the other), and what a block needs beside its steps.
struct PlaneCost {
    int64_t side, threads;
    double few, one, two, more;
};
constexpr PlaneCost kPlaneCost[2][3] = {
    {{256, 512, 1.2, 1.65, 1.65, 12.0}, {128, 256, 0.55, 0.7, 0.9, 6.0}, {64, 256, 0.24, 0.28, 0.32, 4.0}},         // One
    {{256, 512, 1.65, 2.35, 2.35, 13.0}, {128, 256, 0.72, 0.95, 1.2, 6.0}, {64, 256, 0.28, 0.32, 0.36, 4.0}}};      // Halves

// The tile, and the number of parts of the inner axis, whose turns on the chip take the least time: large tiles read least for what
// they compute, small ones and parts keep all units busy, and a tile's parts go to memory and are read by one block (22 KB/us).
// Blocks of 128 x 128 whose results leave (all but those of logits, whose sums may not be cut) need 2 us more: with and without them 12 updates of 256 x
// 1024 take 196 and 217 us and dx of 1000000 x 32 x 200 in bfloat16 186 and 271; but logits of 4096 x 407 x 856 in bfloat16 38 and 33, of 6633 x 253 x
// 1287 in float32 78 and 75.
// 1024 x 4096 times its transpose, one after the other in tiles of 256, 128 and 64 with the best number of parts: 131, 34 and 27 us;
// 2048 x 2048 . 2048 x 8192: 159, 175 and 240.
inline PlanePlan plane_plan(int64_t Ma, int64_t Nb, int64_t steps, int64_t batches, bool symmetric, bool may_split, int halves) {
    PlanePlan best{};
    const int64_t cus = compute_units();
    double least = 0.0;
    for (int shape = 0; shape < 3; ++shape) {
        const PlaneCost& c = kPlaneCost[halves][shape];
        PlanePlan p{};
        p.shape = shape;
        p.tiles_m = (int)ceil_div(Ma, c.side);
        p.tiles_n = (int)ceil_div(Nb, c.side);
        p.tiles = symmetric ? (int64_t)p.tiles_m * (p.tiles_m + 1) / 2 : (int64_t)p.tiles_m * p.tiles_n;
        // a launch counts its threads in 32 bits; whoever has checked that the large tiles are few enough finds a plan
        if (shape > 0 && p.tiles * c.threads >= 1LL << 32) continue;
        const bool parts = may_split && p.tiles * batches <= kMostParted;
        for (int64_t splits = 1; splits <= 1024 && (splits == 1 || (parts && steps / splits >= 4)); splits += std::max<int64_t>(1, splits / 2)) {
            const int64_t per = std::max<int64_t>(1, ceil_div(steps, splits)), real = std::max<int64_t>(1, ceil_div(steps, per));
            const int64_t blocks = p.tiles * batches * real, slots = shape == 0 ? cus : 2 * cus;
            const double more = c.more + (shape == 1 && may_split ? 2.0 : 0.0);
            const double turn = (double)per * (blocks > cus ? c.two : 2 * blocks > cus ? c.one : c.few) + more;
            const double join = real > 1 ? 2.0 + (double)(real * c.side * c.side * 4) / 22e3 : 0.0;
            const double time = (double)ceil_div(std::max<int64_t>(blocks, 1), slots) * turn + join;
            if ((shape == 0 && splits == 1) || time < least) {
                least = time;
                best = p;
                best.splits = (int)real;
                best.per = (int)per;
            }
        }
    }
    return best;
}
inline size_t plane_part_bytes(const PlanePlan& p, int64_t batches) {
    const size_t side = kPlaneCost[0][p.shape].side;
    return p.splits > 1 ? (size_t)batches * p.tiles * p.splits * side * side * sizeof(float) : 0;
}

}  // namespace daspmm
