// Products of packed matrices: their launch.
#pragma once
#include "da_internal.h"
#include "da_planes.h"

#include <algorithm>

namespace daspmm {
namespace {

typedef PlaneShape<256, 256, 2, 4, 2, false> PlaneLarge;
typedef PlaneShape<128, 128, 2, 2, 2, true> PlaneMiddle;
typedef PlaneShape<64, 64, 2, 2, 4, true> PlaneSmall;

static_assert(PlaneLarge::THREADS == kPlaneCost[0][0].threads && PlaneMiddle::THREADS == kPlaneCost[0][1].threads &&
              PlaneSmall::THREADS == kPlaneCost[0][2].threads && PlaneLarge::BM == kPlaneCost[0][0].side &&
              PlaneMiddle::BM == kPlaneCost[0][1].side && PlaneSmall::BM == kPlaneCost[0][2].side, "the tiles that are planned with");

template <class P, class S, int ALAY, int BLAY, int BOUND, class E>
void plane_launch(const PlaneArgs& g, const E& epi, const PlanePlan& p, int batches, hipStream_t s) {
    constexpr auto kernel = plane_kernel<P, S, ALAY, BLAY, BOUND, E>;
    allow_lds<kernel>(S::LDS);
    hipLaunchKernelGGL(kernel, dim3((unsigned)p.tiles, (unsigned)p.splits, (unsigned)batches), dim3(S::THREADS), S::LDS, s, g, epi);
}

// `p` is plane_plan's for the same sizes; `part` holds plane_part_bytes, `arrived` kMostParted numbers that are 0 and are left so.
template <class P, int ALAY, int BLAY, int BOUND, class E>
void plane_product(PlaneArgs g, const E& epi, const PlanePlan& p, int batches, float* part, int* arrived, hipStream_t s) {
    if (p.tiles == 0 || batches == 0) return;
    g.tiles_m = p.tiles_m;
    g.tiles_n = p.tiles_n;
    g.splits = p.splits;
    g.per = p.per;
    g.part = part;
    g.arrived = arrived;
    if (p.shape == 0) plane_launch<P, PlaneLarge, ALAY, BLAY, BOUND, E>(g, epi, p, batches, s);
    else if (p.shape == 1) plane_launch<P, PlaneMiddle, ALAY, BLAY, BOUND, E>(g, epi, p, batches, s);
    else plane_launch<P, PlaneSmall, ALAY, BLAY, BOUND, E>(g, epi, p, batches, s);
}

}  // namespace
}  // namespace daspmm
