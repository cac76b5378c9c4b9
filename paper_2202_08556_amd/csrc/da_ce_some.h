// Cross entropy of a linear layer for 5 to 64 rows of float32, or 5 to 32 of bfloat16: the weight is still what has to be read, and
// packing it reads and writes it once more than a product does.  The fp32 matrix cores take it as it comes; with 64 rows they are as
// busy as memory (16 x 16 x 4 products for every 16 rows of 64 bytes).  Forward and backward by rows, against packing the weight:
//   4096 x 32000 float32   5: 464   32: 510   64: 680   65, packed: 1340 us      1000 x 100000   5: 363   32: 447   64: 653   65: 1046
//   ... bfloat16           5: 270   16: 280   32: 403   33, packed: 460; 40 here: 520            5: 278   16: 293   32: 403   33: 583, 40 here 502
// (forward and backward; forward alone, whose weight needs no packing where its sizes are whole, 32 rows of bfloat16 take 96 here and 60 packed).
// 64 rows of float32 are what the registers hold; packing would be the better way from some 140 on.
// The logits of 64 rows take 177 us of the matrix cores' 109, the other products 400 of 218.
//
// Logits: a block of four waves has 64 classes, a wave every fourth 16 of its lines; a lane loads 16 bytes of four lines, which are the
// second operand of 16 products for every 16 rows.  Backward, a wave has 16 lines and goes along the classes, 64 at a time: the
// weight's numbers times dz for dx, then x times dz for dw.  dz is in LDS, once for four waves.
#pragma once
#include "da_ce_few.h"
#include "da_ce_narrow.h"

namespace daspmm {

template <class T> constexpr int some_rows = sizeof(T) == 4 ? kSomeRows : 32;
constexpr int kSomeStep = 64, kSomePitch = kSomeStep + 4;      // classes of a step

// Blocks to a unit whose registers there have to be, backward and for logits
constexpr int some_blocks(int RF) { return RF == 1 ? 4 : RF <= 3 ? 3 : 2; }
constexpr int some_logit_blocks(int RF) { return RF <= 2 ? 4 : 3; }

// Loads above are asked for before anything below: left alone, the compiler moves each to just before its use
__device__ __forceinline__ void some_ask() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

// Four neighbouring numbers
template <class T> __device__ __forceinline__ f32x4 some_four(const T* __restrict__ p) {
    float v[4];
    load_floats<4>(p, v);
    return f32x4{v[0], v[1], v[2], v[3]};
}

// RF: 16 rows each
template <class T, int RF, bool BWD> __global__ __launch_bounds__(kFewBlock, some_logit_blocks(RF)) void ce_some_logits_kernel(FewArgs a)
{
    __shared__ __attribute__((aligned(16))) f32x4 others[3][4][64];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, i16 = lane & 15, h = lane >> 4;
    if (!BWD && blockIdx.x == 0 && blockIdx.y == 0 && tid <= kSomeRows) a.arrived[tid * kFewApart] = 0;
    const long n = (long)blockIdx.x * kSomeStep + 4 * i16, left = a.V - n;
    const int k1 = min((int)(blockIdx.y + 1) * a.per, a.d);
    const T* __restrict__ W = static_cast<const T*>(a.w) + n;
    const T* __restrict__ X = static_cast<const T*>(a.x);
    bool there[RF];
    const T* row[RF];                                        // one that is not there is the first, and its numbers are dropped
#pragma unroll
    for (int f = 0; f < RF; ++f) {
        there[f] = few_target(a, f * 16 + i16, BWD) >= 0;
        row[f] = X + (there[f] ? f * 16 + i16 : 0) * a.ldx;
    }
    f32x4 acc[RF][4];
#pragma unroll
    for (int f = 0; f < RF; ++f)
#pragma unroll
        for (int c = 0; c < 4; ++c) acc[f][c] = f32x4{0.f, 0.f, 0.f, 0.f};
    struct Lines {
        f32x4 w[4], x[RF];
    };
    auto get = [&](int k, Lines& g) {                        // lines k to k + 15
#pragma unroll
        for (int u = 0; u < 4; ++u) g.w[u] = some_four(W + (long)(k + 4 * h + u) * a.V);
#pragma unroll
        for (int f = 0; f < RF; ++f) g.x[f] = some_four(row[f] + k + 4 * h);
    };
    auto get_some = [&](int k, Lines& g) {                   // ... of which those below k1 are there
#pragma unroll
        for (int u = 0; u < 4; ++u) g.w[u] = narrow_four(W + (long)(k + 4 * h + u) * a.V, k + 4 * h + u < k1 ? (int)min(left, 4l) : 0);
#pragma unroll
        for (int f = 0; f < RF; ++f) g.x[f] = narrow_four(row[f] + k + 4 * h, k1 - k - 4 * h);
    };
    auto add = [&](Lines& g) {
#pragma unroll
        for (int f = 0; f < RF; ++f)
#pragma unroll
            for (int u = 0; u < 4; ++u) g.x[f][u] = there[f] ? g.x[f][u] : 0.f;
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int f = 0; f < RF; ++f)
#pragma unroll
                for (int c = 0; c < 4; ++c) acc[f][c] = __builtin_amdgcn_mfma_f32_16x16x4f32(g.x[f][u], g.w[u][c], acc[f][c], 0, 0, 0);
    };
    // Whole ones first, the next of which are always asked for, at worst once more: the wait in front of the products can leave them out
    int k = blockIdx.y * a.per + 16 * wave;
    const int many = (long)(blockIdx.x + 1) * kSomeStep <= a.V ? max(0, (k1 - k + 48) / 64) : 0, last = k + 64 * (many - 1);
    Lines one, two;
    if (many > 0) {
        get(k, one);
        for (;;) {
            get(min(k + 64, last), two);
            some_ask();
            add(one);
            k += 64;
            if (k > last) break;
            get(min(k + 64, last), one);
            some_ask();
            add(two);
            k += 64;
            if (k > last) break;
        }
    }
    for (; k < k1; k += 64) {
        get_some(k, one);
        add(one);
    }
#pragma unroll
    for (int f = 0; f < RF; ++f) {
        __syncthreads();
        if (wave > 0)
#pragma unroll
            for (int c = 0; c < 4; ++c) others[wave - 1][c][lane] = acc[f][c];
        __syncthreads();
        if (wave == 0 && n < a.Vp) {
#pragma unroll
            for (int c = 0; c < 4; ++c) acc[f][c] = (acc[f][c] + others[0][c][lane]) + (others[1][c][lane] + others[2][c][lane]);
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int r = f * 16 + 4 * h + q;
                const float s[4] = {acc[f][0][q], acc[f][1][q], acc[f][2][q], acc[f][3][q]};
                if (r < a.rows) store_floats<4>(a.part + ((long)blockIdx.y * a.rows + r) * a.Vp + n, s);
            }
        }
    }
}

// dz: a class of a row to a thread
__global__ __launch_bounds__(kFewBlock) void ce_some_grad_kernel(FewArgs a)
{
    const long v = (long)blockIdx.x * kFewBlock + threadIdx.x;
    if (v >= a.Vp) return;
    const int r = blockIdx.y, t = a.kept_target[r];
    float dz = 0.f;
    if (t >= 0 && v < a.V) {
        const float g = a.reduction == DA_LOSS_ROWS ? a.dloss[r * a.stride] : a.reduction == DA_LOSS_MEAN ? a.dloss[0] / (float)max(1, *a.count) : a.dloss[0];
        const float p = exp2_hw((few_logit(a, r, v) - a.lse[r]) * 1.44269504088896f);
        dz = g * (v == t ? p - 1.f : p);
    }
    a.dz[r * a.Vp + v] = dz;
}

template <class T, int RF> __global__ __launch_bounds__(kFewBlock, some_blocks(RF)) void ce_some_products_kernel(FewArgs a)
{
    __shared__ __attribute__((aligned(16))) float tiles[2][RF * 16][kSomePitch];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, i16 = lane & 15, h = lane >> 4;
    const int k = blockIdx.x * 64 + wave * 16;               // the wave's lines
    const bool mine = k + i16 < a.d;
    const T* __restrict__ W = static_cast<const T*>(a.w) + (long)(k + i16) * a.V;
    const bool whole = k + 16 <= a.d;
    float x[RF * 4];                                         // of row 4 s + h, line i16
#pragma unroll
    for (int s = 0; s < RF * 4; ++s) {
        const int r = 4 * s + h;
        float one[1] = {0.f};
        if (mine && a.dw && few_target(a, r, true) >= 0) load_floats<1>(static_cast<const T*>(a.x) + (long)r * a.ldx + k + i16, one);
        x[s] = one[0];
    }
    f32x4 dx[RF][4];
#pragma unroll
    for (int f = 0; f < RF; ++f) dx[f][0] = dx[f][1] = dx[f][2] = dx[f][3] = f32x4{0.f, 0.f, 0.f, 0.f};
    f32x4 w[4], then[4], dz[RF];
    auto get = [&](long v) {
        if (a.dx && whole && v + kSomeStep <= a.V) {
#pragma unroll
            for (int u = 0; u < 4; ++u) then[u] = some_four(W + v + 16 * u + 4 * h);
        } else if (a.dx) {
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const long at = v + 16 * u + 4 * h;
                then[u] = narrow_four(W + at, mine ? (int)max(min(a.V - at, 4l), 0l) : 0);
            }
        }
#pragma unroll
        for (int f = 0; f < RF; ++f) {
            const int r = f * 16 + tid / 16;
            dz[f] = some_four(a.dz + min(r, a.rows - 1) * a.Vp + v + tid % 16 * 4);
        }
    };
    const long step = (long)gridDim.y * kSomeStep;
    int buf = 0;
    long v = (long)blockIdx.y * kSomeStep;
    if (v < a.V) get(v);
    for (; v < a.V; v += step, buf ^= 1) {
        float (*const tile)[kSomePitch] = tiles[buf];        // its readers of two steps ago are behind the last step's barrier
#pragma unroll
        for (int f = 0; f < RF; ++f)
            *reinterpret_cast<f32x4*>(&tile[f * 16 + tid / 16][tid % 16 * 4]) = f * 16 + tid / 16 < a.rows ? dz[f] : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int u = 0; u < 4; ++u) w[u] = then[u];
        __syncthreads();
        if (v + step < a.V) get(v + step);
        if (a.db && blockIdx.x == 0 && tid < kSomeStep && v + tid < a.V) {
            float s[4] = {};
#pragma unroll
            for (int r = 0; r < RF * 16; ++r) s[r & 3] += tile[r][tid];
            store_param(a.db, a.param_type, v + tid, (s[0] + s[1]) + (s[2] + s[3]));
        }
        if (a.dx)
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                f32x4 z[RF];
#pragma unroll
                for (int f = 0; f < RF; ++f) z[f] = *reinterpret_cast<const f32x4*>(&tile[f * 16 + i16][16 * u + 4 * h]);
#pragma unroll
                for (int c = 0; c < 4; ++c)
#pragma unroll
                    for (int f = 0; f < RF; ++f) dx[f][u] = __builtin_amdgcn_mfma_f32_16x16x4f32(z[f][c], w[u][c], dx[f][u], 0, 0, 0);
            }
        if (a.dw) {
            f32x4 dw[4];
#pragma unroll
            for (int c = 0; c < 4; ++c) dw[c] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int s = 0; s < RF * 4; ++s) {
                const f32x4 z = *reinterpret_cast<const f32x4*>(&tile[4 * s + h][4 * i16]);
#pragma unroll
                for (int c = 0; c < 4; ++c) dw[c] = __builtin_amdgcn_mfma_f32_16x16x4f32(x[s], z[c], dw[c], 0, 0, 0);
            }
            const long n = v + 4 * i16, left = a.V - n;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int line = k + 4 * h + q;
                if (line >= a.d) break;
                T* __restrict__ p = static_cast<T*>(a.dw) + (long)line * a.V + n;
                const float s[4] = {dw[0][q], dw[1][q], dw[2][q], dw[3][q]};
                if (left >= 4) {
                    store_floats<4>(p, s);
                } else {
#pragma unroll
                    for (int i = 0; i < 3; ++i) {
                        const float one[1] = {s[i]};
                        if (i < left) store_floats<1>(p + i, one);
                    }
                }
            }
        }
    }
    if (!a.dx || !mine) return;
#pragma unroll
    for (int f = 0; f < RF; ++f)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int r = f * 16 + 4 * h + q;
            if (r >= a.rows) break;
            // without a target 0, also where the weight holds infinities
            const float one[1] = {a.kept_target[r] >= 0 ? (dx[f][0][q] + dx[f][1][q]) + (dx[f][2][q] + dx[f][3][q]) : 0.f};
            if (gridDim.y > 1) a.dx_part[((long)blockIdx.y * a.rows + r) * a.d + k + i16] = one[0];
            else store_floats<1>(static_cast<T*>(a.dx) + (long)r * a.d + k + i16, one);
        }
}

}  // namespace daspmm
