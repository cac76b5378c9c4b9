// Cross entropy of a linear layer with few classes and more inner positions than da_ce_narrow.h holds: 64 positions of the weight
// at a time are in LDS, two steps of them, and x passes from memory to the matrix cores (float32 for both types).  A block takes 128
// rows that have a target at a time, 32 to a wave.  Backward, the same walk gives the logits again and a second one dx; dz, a few
// numbers a row, goes to memory for another kernel, whose blocks own 64 inner positions of dw over a part of the rows.
// (Packed for the 16-bit matrix cores, 100000 rows of 700 with 10 classes took 800 us, 290 of them in packing x; so 64 forward and 263 backward.)
#pragma once
#include "da_ce_narrow.h"

namespace daspmm {

constexpr int kTallClasses = 64, kTallStep = 64, kTallPitch = kTallStep + 4, kTallRows = 128;

struct TallArgs : NarrowArgs {
    float* dz;                   // [row][16 NF], of the rows with a target
    long per;                    // rows of a part of dw
};

// 64 inner positions of the weight from k0 on, [class][position]: a thread's numbers on their way, and their place
template <class T, int NF> struct TallWeight {
    static constexpr int EACH = NF * 16 * kTallStep / kNarrowBlock;
    float v[EACH];
    __device__ __forceinline__ void load(const T* __restrict__ W, int k0, int d, int V) {
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const int at = threadIdx.x + i * kNarrowBlock, p = k0 + at / (NF * 16), n = at % (NF * 16);
            float one[1] = {0.f};
            if (p < d && n < V) load_floats<1>(W + (long)p * V + n, one);
            v[i] = one[0];
        }
    }
    __device__ __forceinline__ void put(float* __restrict__ w) const {
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const int at = threadIdx.x + i * kNarrowBlock;
            w[at % (NF * 16) * kTallPitch + at / (NF * 16)] = v[i];
        }
    }
};

template <class T, int NF, bool BWD>
__global__ __launch_bounds__(kNarrowBlock) void ce_tall_kernel(TallArgs a)
{
    constexpr int RF = kTallRows / 64, STEP = kTallStep, FRAGS = STEP / 16;
    __shared__ __attribute__((aligned(16))) float w[2][NF * 16 * kTallPitch];
    __shared__ int list[kNarrowChunk];
    __shared__ int counts[4];
    __shared__ double totals[4];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, i16 = lane & 15, h = lane >> 4;
    const int steps = (a.d + STEP - 1) / STEP;
    const T* __restrict__ W = static_cast<const T*>(a.w);
    const T* __restrict__ X = static_cast<const T*>(a.x);
    float bias[NF][4];
#pragma unroll
    for (int j = 0; j < NF; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int n = j * 16 + 4 * h + q;
            bias[j][q] = n >= a.V ? -INFINITY : a.b ? load_param(a.b, a.param_type, n) : 0.f;
        }
    const int* const kept = a.kept_target;
    float factor = 0.f;
    if constexpr (BWD) factor = a.reduction == DA_LOSS_MEAN ? a.dloss[0] / (float)max(1, *a.count) : a.reduction == DA_LOSS_SUM ? a.dloss[0] : 0.f;
    double total = 0.0;
    long many = 0;

    for (long first = (long)blockIdx.x * a.chunk; first < a.rows; first += (long)gridDim.x * a.chunk) {
        __syncthreads();                                     // the list before has been read
        const int here = (int)min((long)a.chunk, a.rows - first);
        int n = 0;
        for (int k = 0; k < here; k += kNarrowBlock) {
            const long r = first + k + tid;
            long t = -1;
            if (k + tid < here) {
                if constexpr (BWD) t = kept[r];
                else t = a.target64 ? static_cast<const int64_t*>(a.target)[r] : (long)static_cast<const int32_t*>(a.target)[r];
                if (t >= a.V) t = -1;
                if constexpr (!BWD) {
                    a.kept_target[r] = t < 0 ? -1 : (int)t;
                    if (t < 0 && a.reduction == DA_LOSS_ROWS) a.loss[r] = 0.f;
                }
            }
            const uint64_t mask = __ballot(t >= 0);
            if (lane == 0) counts[wave] = __popcll(mask);
            __syncthreads();
            int at = n;
            for (int v = 0; v < wave; ++v) at += counts[v];
            at += __popcll(mask & ((1ull << lane) - 1));     // rows before this one that have a target; of k + tid
            if (t >= 0) list[at] = (k + tid) | (int)t << 16;
            else if (k + tid < here) list[kNarrowChunk - 1 - (k + tid - at)] = k + tid;      // the others from the end
            n += counts[0] + counts[1] + counts[2] + counts[3];
            __syncthreads();
        }
        many += n;
        if constexpr (BWD) {
            if (a.dx)                                        // rows without a target
                for (int k = wave; k < here - n; k += 4) {
                    T* __restrict__ p = static_cast<T*>(a.dx) + (first + list[kNarrowChunk - 1 - k]) * a.d;
                    const float zero[4] = {0.f, 0.f, 0.f, 0.f}, one[1] = {0.f};
                    for (int c = 4 * lane; c < a.d; c += 256) {
                        if (c + 4 <= a.d) {
                            store_floats<4>(p + c, zero);
                        } else {
                            for (int q = c; q < a.d; ++q) store_floats<1>(p + q, one);
                        }
                    }
                }
        }
        for (int g0 = 0; g0 < n; g0 += kTallRows) {
            bool there[RF];
            long row[RF];
            int t[RF];
            f32x4 z[RF][NF];
#pragma unroll
            for (int f = 0; f < RF; ++f) {
                const int mine = g0 + (wave * RF + f) * 16 + i16;            // of the list
                there[f] = mine < n;
                const int entry = there[f] ? list[mine] : -0x10000;
                t[f] = entry >> 16;
                row[f] = first + (entry & 0xffff);
#pragma unroll
                for (int j = 0; j < NF; ++j) z[f][j] = f32x4{0.f, 0.f, 0.f, 0.f};
            }
            // logits: the next step's numbers are on their way while this one's are multiplied
            f32x4 x[RF][FRAGS];
            TallWeight<T, NF> next;
            auto load = [&](int s) {
#pragma unroll
                for (int f = 0; f < RF; ++f)
#pragma unroll
                    for (int u = 0; u < FRAGS; ++u) {
                        const int c = s * STEP + u * 16 + 4 * h;
                        x[f][u] = narrow_four(X + row[f] * a.ldx + c, there[f] ? a.d - c : 0);
                    }
            };
            next.load(W, 0, a.d, a.V);
            load(0);
            __syncthreads();                                 // both places of the weight are free
            next.put(w[0]);
            for (int s = 0; s < steps; ++s) {
                f32x4 now[RF][FRAGS];
#pragma unroll
                for (int f = 0; f < RF; ++f)
#pragma unroll
                    for (int u = 0; u < FRAGS; ++u) now[f][u] = x[f][u];
                if (s + 1 < steps) {
                    next.load(W, (s + 1) * STEP, a.d, a.V);
                    load(s + 1);
                }
                __syncthreads();                             // this step's weight is there; the step before has been multiplied
                const float* const here_w = w[s & 1];
#pragma unroll
                for (int u = 0; u < FRAGS; ++u)
#pragma unroll
                    for (int j = 0; j < NF; ++j) {
                        const f32x4 wf = *reinterpret_cast<const f32x4*>(here_w + (j * 16 + i16) * kTallPitch + u * 16 + 4 * h);
#pragma unroll
                        for (int q = 0; q < 4; ++q)
#pragma unroll
                            for (int f = 0; f < RF; ++f) z[f][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(wf[q], now[f][u][q], z[f][j], 0, 0, 0);
                    }
                if (s + 1 < steps) next.put(w[(s + 1) & 1]);
            }
#pragma unroll
            for (int f = 0; f < RF; ++f)
#pragma unroll
                for (int j = 0; j < NF; ++j)
#pragma unroll
                    for (int q = 0; q < 4; ++q) z[f][j][q] += bias[j][q];
            if constexpr (!BWD) {
#pragma unroll
                for (int f = 0; f < RF; ++f) {
                    float most = -INFINITY, at_target = 0.f, sum = 0.f;
#pragma unroll
                    for (int j = 0; j < NF; ++j)
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            most = fmaxf(most, z[f][j][q]);
                            if (j * 16 + 4 * h + q == t[f]) at_target = z[f][j][q];
                        }
                    most = fmaxf(most, __shfl_xor(most, 16, 64));
                    most = fmaxf(most, __shfl_xor(most, 32, 64));
                    const float from = most == -INFINITY ? 0.f : most;
#pragma unroll
                    for (int j = 0; j < NF; ++j)
#pragma unroll
                        for (int q = 0; q < 4; ++q) sum += exp2_hw((z[f][j][q] - from) * 1.44269504088896f);
                    sum += __shfl_xor(sum, 16, 64);
                    sum += __shfl_xor(sum, 32, 64);
                    at_target += __shfl_xor(at_target, 16, 64);
                    at_target += __shfl_xor(at_target, 32, 64);
                    const float lse = most + logf(sum), loss = lse - at_target;
                    if (there[f] && h == 0) {
                        a.lse[row[f]] = lse;
                        if (a.reduction == DA_LOSS_ROWS) a.loss[row[f]] = loss;
                        total += loss;
                    }
                }
            } else {
#pragma unroll
                for (int f = 0; f < RF; ++f) {
                    const float lse = there[f] ? a.lse[row[f]] : 0.f;
                    const float g = a.reduction == DA_LOSS_ROWS ? (there[f] ? a.dloss[row[f] * a.stride] : 0.f) : factor;
#pragma unroll
                    for (int j = 0; j < NF; ++j) {
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            const int c = j * 16 + 4 * h + q;
                            const float p = exp2_hw((z[f][j][q] - lse) * 1.44269504088896f);
                            z[f][j][q] = there[f] && c < a.V ? g * (c == t[f] ? p - 1.f : p) : 0.f;
                        }
                        if (there[f]) *reinterpret_cast<f32x4*>(a.dz + row[f] * (NF * 16) + j * 16 + 4 * h) = z[f][j];
                    }
                }
                if (!a.dx) continue;
                next.load(W, 0, a.d, a.V);
                __syncthreads();                             // the logits' last step has been multiplied
                next.put(w[0]);
                for (int s = 0; s < steps; ++s) {
                    if (s + 1 < steps) next.load(W, (s + 1) * STEP, a.d, a.V);
                    __syncthreads();
                    const float* const here_w = w[s & 1];
#pragma unroll
                    for (int u = 0; u < FRAGS; ++u) {
                        f32x4 sum[RF];
#pragma unroll
                        for (int f = 0; f < RF; ++f) sum[f] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                        for (int j = 0; j < NF; ++j)
#pragma unroll
                            for (int q = 0; q < 4; ++q) {
                                const float wt = here_w[(j * 16 + 4 * h + q) * kTallPitch + u * 16 + i16];
#pragma unroll
                                for (int f = 0; f < RF; ++f) sum[f] = __builtin_amdgcn_mfma_f32_16x16x4f32(wt, z[f][j][q], sum[f], 0, 0, 0);
                            }
                        const int c = s * STEP + u * 16 + 4 * h, left = a.d - c;
#pragma unroll
                        for (int f = 0; f < RF; ++f) {
                            if (!there[f]) continue;
                            T* __restrict__ out = static_cast<T*>(a.dx) + row[f] * a.d + c;
                            const float v[4] = {sum[f][0], sum[f][1], sum[f][2], sum[f][3]};
                            if (left >= 4) {
                                store_floats<4>(out, v);
                            } else {
#pragma unroll
                                for (int q = 0; q < 3; ++q) {
                                    const float one[1] = {v[q]};
                                    if (q < left) store_floats<1>(out + q, one);
                                }
                            }
                        }
                    }
                    if (s + 1 < steps) next.put(w[(s + 1) & 1]);
                }
            }
        }
    }
    if constexpr (!BWD) {
        total = wave_sum(total, 64);
        if (lane == 0) totals[wave] = total;
        __syncthreads();
        if (tid == 0) {
            const double sum = (totals[0] + totals[1]) + (totals[2] + totals[3]);
            if (gridDim.x > 1) {
                a.sums[2 * blockIdx.x] = sum;
                a.sums[2 * blockIdx.x + 1] = (double)many;
            } else {
                *a.count = (int)many;
                if (a.reduction != DA_LOSS_ROWS) *a.loss = (float)(a.reduction == DA_LOSS_MEAN ? sum / (double)max(1L, many) : sum);
            }
        }
    }
}

// dw = x^T dz over the rows of a part, 64 inner positions to a block, 16 to a wave; the first block of a part makes its db, too
template <class T, int NF> __global__ __launch_bounds__(kNarrowBlock) void ce_tall_weight_kernel(TallArgs a)
{
    constexpr int ROWS = 64, PK = 64 + 4, PV = NF * 16 + 4;
    __shared__ __attribute__((aligned(16))) float xs[ROWS * PK];
    __shared__ __attribute__((aligned(16))) float ds[ROWS * PV];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, i16 = lane & 15, h = lane >> 4, k0 = blockIdx.x * 64;
    const T* __restrict__ X = static_cast<const T*>(a.x);
    const long r0 = blockIdx.y * a.per, r1 = min(r0 + a.per, a.rows);
    f32x4 dw[NF];
#pragma unroll
    for (int j = 0; j < NF; ++j) dw[j] = f32x4{0.f, 0.f, 0.f, 0.f};
    float db = 0.f;
    const bool sums = a.db && blockIdx.x == 0;
    f32x4 x[4], z[NF];
    const int line = tid / 16, at = tid % 16 * 4;            // 16 rows at a time
    auto load = [&](long r) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const long m = r + i * 16 + line;
            const bool there = m < r1 && a.kept_target[m] >= 0;
            x[i] = narrow_four(X + m * a.ldx + k0 + at, there ? a.d - k0 - at : 0);
        }
#pragma unroll
        for (int i = 0; i < NF; ++i) {
            const int k = tid + i * kNarrowBlock, l = k / (NF * 4);
            const long m = r + l;
            const bool there = m < r1 && a.kept_target[m] >= 0;
            z[i] = there ? *reinterpret_cast<const f32x4*>(a.dz + m * (NF * 16) + k % (NF * 4) * 4) : f32x4{0.f, 0.f, 0.f, 0.f};
        }
    };
    if (r0 < r1) load(r0);
    for (long r = r0; r < r1; r += ROWS) {
        __syncthreads();                                     // the rows before have been multiplied
#pragma unroll
        for (int i = 0; i < 4; ++i) *reinterpret_cast<f32x4*>(xs + (i * 16 + line) * PK + at) = x[i];
#pragma unroll
        for (int i = 0; i < NF; ++i) {
            const int k = tid + i * kNarrowBlock;
            *reinterpret_cast<f32x4*>(ds + k / (NF * 4) * PV + k % (NF * 4) * 4) = z[i];
        }
        __syncthreads();
        if (r + ROWS < r1) load(r + ROWS);
        if (a.dw)
#pragma unroll
            for (int m = 0; m < ROWS; m += 16) {
                float xt[4];
#pragma unroll
                for (int q = 0; q < 4; ++q) xt[q] = xs[(m + 4 * h + q) * PK + wave * 16 + i16];
#pragma unroll
                for (int j = 0; j < NF; ++j)
#pragma unroll
                    for (int q = 0; q < 4; ++q) dw[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(ds[(m + 4 * h + q) * PV + j * 16 + i16], xt[q], dw[j], 0, 0, 0);
            }
        if (sums && tid < NF * 16) {
            float s[4] = {};
            for (int m = 0; m < ROWS; m += 4)
#pragma unroll
                for (int u = 0; u < 4; ++u) s[u] += ds[(m + u) * PV + tid];
            db += (s[0] + s[1]) + (s[2] + s[3]);
        }
    }
    float* __restrict__ part = a.part + (long)blockIdx.y * (a.d + 1) * a.V;
    const int p = k0 + wave * 16 + i16;
    if (a.dw && p < a.d)
#pragma unroll
        for (int j = 0; j < NF; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int n = j * 16 + 4 * h + q;
                if (n < a.V) part[(long)p * a.V + n] = dw[j][q];
            }
    if (sums && tid < a.V) part[(long)a.d * a.V + tid] = db;
}

}  // namespace daspmm
