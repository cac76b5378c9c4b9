// Products of packed matrices: how one is cut into tiles and parts, and its launch.
#pragma once
#include "da_internal.h"
#include "da_planes.h"

#include <algorithm>
#include <atomic>

namespace daspmm {
namespace {

typedef PlaneShape<256, 256, 2, 4, 2> PlaneLarge;
typedef PlaneShape<128, 128, 2, 2, 2> PlaneMiddle;
typedef PlaneShape<64, 64, 2, 2, 4> PlaneSmall;

struct PlanePlan {
    int shape;                   // 0 large, 1 middle, 2 small
    int tiles_m, tiles_n;
    int64_t tiles;               // of a batch
    int splits, per;
};

// The largest tiles of which there is one for every unit; fewer than two of the smallest to a unit: the inner axis is cut, in
// parts of at least eight steps.
inline PlanePlan plane_plan(int64_t Ma, int64_t Nb, int64_t steps, int64_t batches, bool symmetric, bool may_split) {
    PlanePlan p{};
    const int64_t cus = compute_units();
    auto set = [&](int shape, int64_t bm, int64_t bn) {
        p.shape = shape;
        p.tiles_m = (int)ceil_div(Ma, bm);
        p.tiles_n = (int)ceil_div(Nb, bn);
        p.tiles = symmetric ? (int64_t)p.tiles_m * (p.tiles_m + 1) / 2 : (int64_t)p.tiles_m * p.tiles_n;
        return p.tiles * batches >= cus;
    };
    if (!set(0, 256, 256) && !set(1, 128, 128)) set(2, 64, 64);
    p.splits = 1;
    p.per = (int)std::max<int64_t>(steps, 1);
    if (may_split && p.tiles * batches < cus) {
        const int64_t splits = std::max<int64_t>(1, std::min<int64_t>(2 * cus / std::max<int64_t>(1, p.tiles * batches), steps / 8));
        p.per = (int)std::max<int64_t>(1, ceil_div(steps, splits));
        p.splits = (int)std::max<int64_t>(1, ceil_div(steps, p.per));
    }
    return p;
}
inline size_t plane_part_bytes(const PlanePlan& p, int64_t Ma, int64_t Nb, int64_t batches) {
    return p.splits > 1 ? (size_t)batches * p.splits * Ma * Nb * sizeof(float) : 0;
}

template <class P, class S, int ALAY, int BLAY, int BOUND, class E>
void plane_launch(const PlaneArgs& g, const E& epi, const PlanePlan& p, int batches, hipStream_t s) {
    auto kernel = plane_kernel<P, S, ALAY, BLAY, BOUND, E>;
    static std::atomic<uint64_t> allowed{0};                 // devices that know how much LDS the kernel takes
    int device = 0;
    (void)hipGetDevice(&device);
    const uint64_t bit = 1ull << (device & 63);
    if (!(allowed.load(std::memory_order_relaxed) & bit) &&
        hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, S::LDS) == hipSuccess)
        allowed.fetch_or(bit, std::memory_order_relaxed);
    hipLaunchKernelGGL(kernel, dim3((unsigned)p.tiles, (unsigned)p.splits, (unsigned)batches), dim3(S::THREADS), S::LDS, s, g, epi);
    if constexpr (!E::kWhole) {
        if (p.splits > 1) {
            const int64_t blocks = std::min<int64_t>(ceil_div((int64_t)g.Ma * g.Nb / 4, 256), 8192);
            hipLaunchKernelGGL((plane_join_kernel<S::BM, S::BN, E>), dim3((unsigned)blocks, 1, (unsigned)batches), dim3(256), 0, s, g, epi);
        }
    }
}

// `p` is plane_plan's for the same sizes; `part` holds plane_part_bytes.
template <class P, int ALAY, int BLAY, int BOUND, class E>
void plane_product(PlaneArgs g, const E& epi, const PlanePlan& p, int batches, float* part, hipStream_t s) {
    if (p.tiles == 0 || batches == 0) return;
    g.tiles_m = p.tiles_m;
    g.tiles_n = p.tiles_n;
    g.splits = p.splits;
    g.per = p.per;
    g.part = part;
    if (p.shape == 0) plane_launch<P, PlaneLarge, ALAY, BLAY, BOUND, E>(g, epi, p, batches, s);
    else if (p.shape == 1) plane_launch<P, PlaneMiddle, ALAY, BLAY, BOUND, E>(g, epi, p, batches, s);
    else plane_launch<P, PlaneSmall, ALAY, BLAY, BOUND, E>(g, epi, p, batches, s);
}

}  // namespace
}  // namespace daspmm
