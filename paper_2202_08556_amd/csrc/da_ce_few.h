// Cross entropy of a linear layer for up to 4 rows (single tokens): every number of the weight is read for a handful of products, so
// memory bounds it and the vector units do the arithmetic, in 32 bits for both types.  Packing the weight for the matrix cores would
// read and write it once more than the products themselves (3 rows of 1208 x 11583 float32, forward: 67 us,
// so 22; the weight's 56 MB are 11 of them).
//
// Logits: a lane owns 16 bytes of a line of the weight and goes down the lines, four waves of a block and the blocks of a column of
// the grid share them; the parts of the sums pass through memory.  Backward, a block owns four lines of the weight and of its gradient:
// one walk along them gives dw and the block's numbers of dx.
#pragma once
#include "da_layer_common.h"

namespace daspmm {

constexpr int kFewRows = 4, kSomeRows = 64;  // here, and of da_ce_some.h
constexpr int kFewBlock = 256, kFewLines = 256, kFewDown = 4;        // threads; lines whose factors are in LDS; lines of a block backward
constexpr int kFewApart = 32;                // counts lie in lines of their own

struct FewArgs {
    const void *x, *w, *b, *target;
    long ldx, V, Vp;             // classes, padded
    int rows, d, param_type, target64, reduction;
    int splits, per;             // of the lines, lines of one
    float* part;                 // [split][row][Vp]
    float2* sums;                // [row][block]
    int each;                    // classes of a thread in that
    float* at_target;            // [row]
    uint32_t* arrived;           // [kSomeRows + 1][kFewApart]: blocks of a row, rows
    double* losses;              // [row]
    int* count;
    int* kept_target;            // [row]: the class, or -1
    float *lse, *loss;
    const float* dloss;
    long stride;
    float* dz;                   // [row][Vp]
    float* dx_part;              // [part of the classes][row][d], where there are several
    void *dx, *dw, *db;
};

__device__ __forceinline__ int few_target(const FewArgs& a, int r, bool backward) {
    if (r >= a.rows) return -1;
    if (backward) return a.kept_target[r];
    const long t = a.target64 ? static_cast<const int64_t*>(a.target)[r] : (long)static_cast<const int32_t*>(a.target)[r];
    return t >= 0 && t < a.V ? (int)t : -1;
}

template <class T, int R, bool BWD> __global__ __launch_bounds__(kFewBlock) void ce_few_logits_kernel(FewArgs a)
{
    constexpr int V = 16 / sizeof(T), U = 4;
    __shared__ __attribute__((aligned(16))) float factor[kFewLines][R];
    __shared__ float others[3][64][V * R];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    if (!BWD && blockIdx.x == 0 && blockIdx.y == 0 && tid <= kSomeRows) a.arrived[tid * kFewApart] = 0;
    const long n = ((long)blockIdx.x * 64 + lane) * V;
    const long left = a.V - n;
    const int k0 = blockIdx.y * a.per, k1 = min(k0 + a.per, a.d);
    const T* __restrict__ W = static_cast<const T*>(a.w);
    const T* __restrict__ X = static_cast<const T*>(a.x);
    float acc[R][V];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int i = 0; i < V; ++i) acc[r][i] = 0.f;
    auto line = [&](int k, float (&w)[V]) {
        const T* __restrict__ p = W + (long)k * a.V + n;
        if (left >= V) {
            load_floats<V>(p, w);
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                float one[1] = {0.f};
                if (i < left) load_floats<1>(p + i, one);
                w[i] = one[0];
            }
        }
    };
    for (int c0 = k0; c0 < k1; c0 += kFewLines) {
        const int lines = min(kFewLines, k1 - c0);
        __syncthreads();
        for (int k = tid; k < kFewLines * R; k += kFewBlock) {
            const int r = k / kFewLines, l = k % kFewLines;
            float one[1] = {0.f};
            if (l < lines && few_target(a, r, BWD) >= 0) load_floats<1>(X + (long)r * a.ldx + c0 + l, one);
            factor[l][r] = one[0];
        }
        __syncthreads();
        auto add = [&](int l, const float (&w)[V]) {
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int i = 0; i < V; ++i) acc[r][i] += factor[l][r] * w[i];
        };
        int l = wave;
        for (; l + 4 * (U - 1) < lines; l += 4 * U) {
            float w[U][V];
#pragma unroll
            for (int u = 0; u < U; ++u) line(c0 + l + 4 * u, w[u]);
#pragma unroll
            for (int u = 0; u < U; ++u) add(l + 4 * u, w[u]);
        }
        for (; l < lines; l += 4) {
            float w[V];
            line(c0 + l, w);
            add(l, w);
        }
    }
    if (wave > 0)
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int i = 0; i < V; ++i) others[wave - 1][lane][r * V + i] = acc[r][i];
    __syncthreads();
    if (wave == 0 && n < a.Vp)
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if (r >= a.rows) break;
            float s[V];
#pragma unroll
            for (int i = 0; i < V; ++i) s[i] = (acc[r][i] + others[0][lane][r * V + i]) + (others[1][lane][r * V + i] + others[2][lane][r * V + i]);
            store_floats<V>(a.part + ((long)blockIdx.y * a.rows + r) * a.Vp + n, s);
        }
}

// A logit from its parts
__device__ __forceinline__ float few_logit(const FewArgs& a, int r, long v) {
    const float* __restrict__ p = a.part + r * a.Vp + v;
    const long step = a.rows * a.Vp;
    float s[4] = {};
    int k = 0;
    for (; k + 4 <= a.splits; k += 4)
#pragma unroll
        for (int u = 0; u < 4; ++u) s[u] += p[(k + u) * step];
    for (; k < a.splits; ++k) s[0] += p[k * step];
    const float z = (s[0] + s[1]) + (s[2] + s[3]);
    return a.b ? z + load_param(a.b, a.param_type, v) : z;
}

// Maxima and sums of 256 x each classes of a row; the block that comes last at a row makes its loss of them, the last of those their sum
__global__ __launch_bounds__(kFewBlock) void ce_few_sums_kernel(FewArgs a)
{
    __shared__ float red[4];
    __shared__ int last;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, r = blockIdx.y, t = few_target(a, r, false);
    auto largest = [&](float x) {
        for (int d = 1; d < 64; d <<= 1) x = fmaxf(x, __shfl_xor(x, d, 64));
        if (lane == 0) red[wave] = x;
        __syncthreads();
        x = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
        __syncthreads();
        return x;
    };
    auto total = [&](float x) {
        x = wave_sum(x, 64);
        if (lane == 0) red[wave] = x;
        __syncthreads();
        x = (red[0] + red[1]) + (red[2] + red[3]);
        __syncthreads();
        return x;
    };
    auto comes_last = [&](uint32_t* count, uint32_t of) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");     // what this wave has stored is there
        __syncthreads();
        if (tid == 0) last = __hip_atomic_fetch_add(count, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == of - 1;
        __syncthreads();
        return last;
    };
    uint64_t* const sums = reinterpret_cast<uint64_t*>(a.sums + (long)r * gridDim.x);
    auto above = [](float m) { return m == -INFINITY ? 0.f : m; };
    if (t >= 0) {
        constexpr int U = 4;
        float own = -INFINITY, own_sum = 0.f;                // of the thread's
        for (int i = 0; i < a.each; i += U) {
            float z[U], m = own;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const long v = ((long)blockIdx.x * a.each + i + u) * kFewBlock + tid;
                z[u] = i + u < a.each && v < a.V ? few_logit(a, r, v) : -INFINITY;
                if (i + u < a.each && v == t) __hip_atomic_store(a.at_target + r, z[u], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                m = fmaxf(m, z[u]);
            }
            own_sum *= exp2_hw((own - above(m)) * 1.44269504088896f);
#pragma unroll
            for (int u = 0; u < U; ++u) own_sum += exp2_hw((z[u] - above(m)) * 1.44269504088896f);
            own = m;
        }
        const float most = largest(own);
        const float sum = total(own_sum * exp2_hw((own - above(most)) * 1.44269504088896f));
        if (tid == 0)
            __hip_atomic_store(sums + blockIdx.x, (uint64_t)__float_as_uint(most) | (uint64_t)__float_as_uint(sum) << 32, __ATOMIC_RELAXED,
                               __HIP_MEMORY_SCOPE_AGENT);
    }
    if (!comes_last(a.arrived + r * kFewApart, gridDim.x)) return;
    double loss = 0.0;
    if (t >= 0) {
        auto get = [&](int c) { return __hip_atomic_load(sums + c, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); };
        float most = -INFINITY, sum = 0.f;
        for (int c = tid; c < (int)gridDim.x; c += kFewBlock) most = fmaxf(most, __uint_as_float((uint32_t)get(c)));
        most = largest(most);
        const float from = above(most);
        for (int c = tid; c < (int)gridDim.x; c += kFewBlock) {
            const uint64_t e = get(c);
            sum += __uint_as_float((uint32_t)(e >> 32)) * exp2_hw((__uint_as_float((uint32_t)e) - from) * 1.44269504088896f);
        }
        const float lse = most + logf(total(sum));
        loss = lse - __hip_atomic_load(a.at_target + r, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        if (tid == 0) a.lse[r] = lse;
    }
    if (tid == 0) {
        a.kept_target[r] = t;
        if (a.reduction == DA_LOSS_ROWS) a.loss[r] = (float)loss;
        __hip_atomic_store(reinterpret_cast<uint64_t*>(a.losses) + r, (uint64_t)__double_as_longlong(loss), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    if (!comes_last(a.arrived + kSomeRows * kFewApart, a.rows) || wave > 0) return;
    static_assert(kSomeRows == 64, "a row to a lane");
    double all = lane < a.rows ? __longlong_as_double((long long)__hip_atomic_load(reinterpret_cast<uint64_t*>(a.losses) + lane, __ATOMIC_RELAXED,
                                                                                  __HIP_MEMORY_SCOPE_AGENT))
                               : 0.0;
    for (int d = 1; d < 64; d <<= 1) all += __shfl_xor(all, d, 64);
    const int many = __popcll(__ballot(few_target(a, lane, false) >= 0));
    if (lane == 0) {
        *a.count = many;
        if (a.reduction != DA_LOSS_ROWS) *a.loss = (float)(a.reduction == DA_LOSS_MEAN ? all / max(1, many) : all);
    }
}

// dz and db: a class to a thread
__global__ __launch_bounds__(kFewBlock) void ce_few_grad_kernel(FewArgs a)
{
    const long v = (long)blockIdx.x * kFewBlock + threadIdx.x;
    if (v >= a.Vp) return;
    const float all = a.reduction == DA_LOSS_MEAN ? a.dloss[0] / (float)max(1, *a.count) : a.dloss[0];
    float db = 0.f;
    for (int r = 0; r < a.rows; ++r) {
        const int t = a.kept_target[r];
        float dz = 0.f;
        if (t >= 0 && v < a.V) {
            const float g = a.reduction == DA_LOSS_ROWS ? a.dloss[r * a.stride] : all;
            const float p = exp2_hw((few_logit(a, r, v) - a.lse[r]) * 1.44269504088896f);
            dz = g * (v == t ? p - 1.f : p);
        }
        a.dz[r * a.Vp + v] = dz;
        db += dz;
    }
    if (a.db && v < a.V) store_param(a.db, a.param_type, v, db);
}

// Four lines of the weight, four neighbouring classes to a lane and step
template <class T, int R> __global__ __launch_bounds__(kFewBlock) void ce_few_products_kernel(FewArgs a)
{
    constexpr int K = kFewDown;
    __shared__ float x[K][R];
    __shared__ float sums[4][K * R];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, k0 = blockIdx.x * K;
    for (int i = tid; i < K * R; i += kFewBlock) {
        const int k = i / R, r = i % R;
        float one[1] = {0.f};
        if (k0 + k < a.d && r < a.rows && a.kept_target[r] >= 0) load_floats<1>(static_cast<const T*>(a.x) + (long)r * a.ldx + k0 + k, one);
        x[k][r] = one[0];
    }
    __syncthreads();
    const T* __restrict__ W = static_cast<const T*>(a.w);
    float acc[K][R];
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int r = 0; r < R; ++r) acc[k][r] = 0.f;
    for (long v = ((long)blockIdx.y * kFewBlock + tid) * 4; v < a.V; v += (long)gridDim.y * kFewBlock * 4) {
        const long left = a.V - v;
        float w[K][4], dz[R][4];
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i) w[k][i] = 0.f;
        if (a.dx)
#pragma unroll
            for (int k = 0; k < K; ++k) {
                if (k0 + k >= a.d) break;
                const T* __restrict__ p = W + (long)(k0 + k) * a.V + v;
                if (left >= 4) {
                    load_floats<4>(p, w[k]);
                } else {
#pragma unroll
                    for (int i = 0; i < 3; ++i)
                        if (i < left) {
                            float one[1];
                            load_floats<1>(p + i, one);
                            w[k][i] = one[0];
                        }
                }
            }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if (r < a.rows) {
                load_floats<4>(a.dz + r * a.Vp + v, dz[r]);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) dz[r][i] = 0.f;
            }
        }
#pragma unroll
        for (int k = 0; k < K; ++k) {
            float dw[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const float f = x[k][r];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    acc[k][r] += w[k][i] * dz[r][i];
                    dw[i] += f * dz[r][i];
                }
            }
            if (a.dw && k0 + k < a.d) {
                T* __restrict__ p = static_cast<T*>(a.dw) + (long)(k0 + k) * a.V + v;
                if (left >= 4) {
                    store_floats<4>(p, dw);
                } else {
#pragma unroll
                    for (int i = 0; i < 3; ++i) {
                        const float one[1] = {dw[i]};
                        if (i < left) store_floats<1>(p + i, one);
                    }
                }
            }
        }
    }
    if (!a.dx) return;
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const float s = wave_sum(acc[k][r], 64);
            if (lane == 0) sums[wave][k * R + r] = s;
        }
    __syncthreads();
    for (int i = tid; i < K * R; i += kFewBlock) {
        const int k = k0 + i / R, r = i % R;
        if (k >= a.d || r >= a.rows) continue;
        // without a target 0, also where the weight holds infinities
        const float one[1] = {a.kept_target[r] >= 0 ? (sums[0][i] + sums[1][i]) + (sums[2][i] + sums[3][i]) : 0.f};
        if (gridDim.y > 1) a.dx_part[((long)blockIdx.y * a.rows + r) * a.d + k] = one[0];
        else store_floats<1>(static_cast<T*>(a.dx) + (long)r * a.d + k, one);
    }
}
template <class T> __global__ __launch_bounds__(kFewBlock) void ce_few_join_kernel(FewArgs a, int parts)
{
    const int i = blockIdx.x * kFewBlock + threadIdx.x, all = a.rows * a.d;
    if (i >= all) return;
    float s[4] = {};
    int k = 0;
    for (; k + 4 <= parts; k += 4)
#pragma unroll
        for (int u = 0; u < 4; ++u) s[u] += a.dx_part[(long)(k + u) * all + i];
    for (; k < parts; ++k) s[0] += a.dx_part[(long)k * all + i];
    const float one[1] = {(s[0] + s[1]) + (s[2] + s[3])};
    store_floats<1>(static_cast<T*>(a.dx) + i, one);
}

}  // namespace daspmm
