// The gated feed-forward block between its translation units: one for each type, and the C entry points.
#pragma once
#include "da_gated_plan.h"

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace daspmm {

// Everything of one call; what a direction does not use is null.
struct GatedCall {
    GatedShape s;
    const void *x, *dy, *wg, *wu, *wd;
    int64_t ldx, ldy;
    int act;
    float *u, *v;                // dense rows x h
    void* a;                     // dense rows x h
    void *y, *dx, *dwg, *dwu, *dwd;
    char* workspace;
    hipStream_t stream;
};

template <class T> size_t gated_forward_bytes(const GatedShape& s);
template <class T> size_t gated_backward_bytes(const GatedShape& s);
template <class T> void gated_forward(const GatedCall& c);
template <class T> void gated_backward(const GatedCall& c);

}  // namespace daspmm
