// Cross entropy of a linear layer with few classes and inner positions (node classification): the weight fits in LDS, a row's
// classes in the registers of a few lanes, and a block does everything for 64 rows at a time.  float32 matrix cores for both
// types: nothing is rounded between the products.
//
// A block goes through chunks of rows, lists those that have a target and takes them 64 at a time, 16 to a wave.  Forward, a wave
// multiplies its rows, as they come from memory, with the weight in LDS, and has the rows' logits whole.  Backward it does so again,
// and the lanes that hold dz hold it as the operand of dz w^T; dz and x go to LDS for x^T dz, of which each wave owns some inner
// positions over all of the block's rows.  The blocks' parts of dw and db are added in one order.
// 262144 x 128 x 41 float32, half of the rows labelled: 34 us forward and 86 backward (by the packed products 340 and 490).
#pragma once
#include "da_layer_common.h"

namespace daspmm {

typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kNarrowClasses = 128, kNarrowInner = 256, kNarrowBlock = 256, kNarrowRows = 64, kNarrowChunk = 1024;
constexpr int kNarrowLds = 156 * 1024;

struct NarrowArgs {
    const void *x, *w, *b, *target;
    long ldx, rows;
    int d, V;                    // inner positions, classes
    int param_type, target64, reduction;
    int chunk;
    int* count;                  // of all rows with a target
    int* kept_target;            // [row]: the class, or -1
    float* lse;                  // [row]
    float* loss;
    double* sums;                // forward, several blocks: [block][2], their losses and rows
    const float* dloss;
    long stride;
    void *dx, *dw, *db;
    float* part;                 // backward, several blocks: [block][d + 1][V], of dw and db
};

constexpr int narrow_pitch(int n) { return n + 4; }                          // numbers; four lines lie in different banks
inline int narrow_inner(int64_t d) { return (int)((d + 15) / 16 * 16); }
inline size_t narrow_lds(int fragments, int inner, bool backward) {
    const size_t w = (size_t)fragments * 16 * narrow_pitch(inner), list = kNarrowChunk;
    return 4 * (w + list + (backward ? (size_t)kNarrowRows * (narrow_pitch(inner) + narrow_pitch(fragments * 16)) : 0));
}

// Four numbers of a row from column c on, of which `left` are there
template <class T> __device__ __forceinline__ f32x4 narrow_four(const T* __restrict__ p, int left) {
    float v[4] = {0.f, 0.f, 0.f, 0.f};
    if (left >= 4) {
        load_floats<4>(p, v);
    } else {
#pragma unroll
        for (int i = 0; i < 3; ++i)
            if (i < left) {
                float one[1];
                load_floats<1>(p + i, one);
                v[i] = one[0];
            }
    }
    return f32x4{v[0], v[1], v[2], v[3]};
}

// NF fragments of 16 classes; KW fragments of 16 inner positions of dw to a wave
template <class T, int NF, int KW, bool BWD>
__global__ __launch_bounds__(kNarrowBlock) void ce_narrow_kernel(NarrowArgs a)
{
    extern __shared__ __attribute__((aligned(16))) float room[];
    __shared__ int counts[4];
    __shared__ double totals[4][2];
    const int inner = (a.d + 15) / 16 * 16, PK = narrow_pitch(inner), PV = narrow_pitch(NF * 16);
    float* const w = room;                                   // [class][inner position]
    int* const list = reinterpret_cast<int*>(w + NF * 16 * PK);              // rows of the chunk that have a target, their classes from bit 16 on; the others from the end
    float* const xs = reinterpret_cast<float*>(list + kNarrowChunk);     // [row][inner position]
    float* const ds = xs + kNarrowRows * PK;                 // [row][class]
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, i16 = lane & 15, h = lane >> 4;
    const T* __restrict__ W = static_cast<const T*>(a.w);
    const T* __restrict__ X = static_cast<const T*>(a.x);

    constexpr int W_AT_ONCE = 8;
    for (int k0 = tid; k0 < inner * NF * 16; k0 += W_AT_ONCE * kNarrowBlock) {
        float one[W_AT_ONCE][1];
#pragma unroll
        for (int u = 0; u < W_AT_ONCE; ++u) {                // what is not there is some other number until it is put down
            const int k = k0 + u * kNarrowBlock, p = k / (NF * 16), n = k % (NF * 16);
            load_floats<1>(W + (long)min(p, a.d - 1) * a.V + min(n, a.V - 1), one[u]);
        }
#pragma unroll
        for (int u = 0; u < W_AT_ONCE; ++u) {
            const int k = k0 + u * kNarrowBlock, p = k / (NF * 16), n = k % (NF * 16);
            if (p < inner) w[n * PK + p] = p < a.d && n < a.V ? one[u][0] : 0.f;
        }
    }
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
    f32x4 dw[KW][NF];
    float db[NF][4];
#pragma unroll
    for (int j = 0; j < NF; ++j) {
#pragma unroll
        for (int k = 0; k < KW; ++k) dw[k][j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int q = 0; q < 4; ++q) db[j][q] = 0.f;
    }

    for (long first = (long)blockIdx.x * a.chunk; first < a.rows; first += (long)gridDim.x * a.chunk) {
        __syncthreads();                                     // the list before has been read; w is there
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
            else if (k + tid < here) list[kNarrowChunk - 1 - (k + tid - at)] = k + tid;
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
        for (int g0 = 0; g0 < n; g0 += kNarrowRows) {
            const int mine = g0 + wave * 16 + i16;           // this lane's row of the list
            const bool there = mine < n;
            const int entry = there ? list[mine] : -0x10000, t = entry >> 16;
            const long row = first + (entry & 0xffff);
            const T* __restrict__ x = X + (there ? row : first) * a.ldx;
            f32x4 z[NF];
#pragma unroll
            for (int j = 0; j < NF; ++j) z[j] = f32x4{0.f, 0.f, 0.f, 0.f};
            constexpr int AT_ONCE = 8;
            for (int k0 = 0; k0 < inner; k0 += 16 * AT_ONCE) {
                f32x4 xf[AT_ONCE];
                if (a.d == inner && k0 + 16 * AT_ONCE <= inner) {            // all at once, with nothing to decide by lane
#pragma unroll
                    for (int u = 0; u < AT_ONCE; ++u) {
                        float v[4];
                        load_floats<4>(x + k0 + u * 16 + 4 * h, v);
                        xf[u] = f32x4{v[0], v[1], v[2], v[3]};
                    }
#pragma unroll
                    for (int u = 0; u < AT_ONCE; ++u)
#pragma unroll
                        for (int q = 0; q < 4; ++q) xf[u][q] = there ? xf[u][q] : 0.f;
                } else {
#pragma unroll
                    for (int u = 0; u < AT_ONCE; ++u) {
                        const int c = k0 + u * 16 + 4 * h;
                        xf[u] = narrow_four(x + c, there ? a.d - c : 0);
                    }
                }
#pragma unroll
                for (int u = 0; u < AT_ONCE; ++u) {
                    const int c = k0 + u * 16 + 4 * h;
                    if (k0 + u * 16 >= inner) break;
                    if constexpr (BWD) *reinterpret_cast<f32x4*>(xs + (wave * 16 + i16) * PK + c) = xf[u];
#pragma unroll
                    for (int j = 0; j < NF; ++j) {
                        const f32x4 wf = *reinterpret_cast<const f32x4*>(w + (j * 16 + i16) * PK + c);
#pragma unroll
                        for (int q = 0; q < 4; ++q) z[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(wf[q], xf[u][q], z[j], 0, 0, 0);
                    }
                }
            }
#pragma unroll
            for (int j = 0; j < NF; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) z[j][q] += bias[j][q];
            if constexpr (!BWD) {
                float most = -INFINITY, at_target = 0.f, sum = 0.f;
#pragma unroll
                for (int j = 0; j < NF; ++j)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        most = fmaxf(most, z[j][q]);
                        if (j * 16 + 4 * h + q == t) at_target = z[j][q];
                    }
                most = fmaxf(most, __shfl_xor(most, 16, 64));
                most = fmaxf(most, __shfl_xor(most, 32, 64));
                const float from = most == -INFINITY ? 0.f : most;
#pragma unroll
                for (int j = 0; j < NF; ++j)
#pragma unroll
                    for (int q = 0; q < 4; ++q) sum += exp2_hw((z[j][q] - from) * 1.44269504088896f);
                sum += __shfl_xor(sum, 16, 64);
                sum += __shfl_xor(sum, 32, 64);
                at_target += __shfl_xor(at_target, 16, 64);
                at_target += __shfl_xor(at_target, 32, 64);
                const float lse = most + logf(sum), loss = lse - at_target;
                if (there && h == 0) {
                    a.lse[row] = lse;
                    if (a.reduction == DA_LOSS_ROWS) a.loss[row] = loss;
                    total += loss;
                }
            } else {
                const float lse = there ? a.lse[row] : 0.f;
                const float g = a.reduction == DA_LOSS_ROWS ? (there ? a.dloss[row * a.stride] : 0.f) : factor;
#pragma unroll
                for (int j = 0; j < NF; ++j) {
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const int c = j * 16 + 4 * h + q;
                        const float p = exp2_hw((z[j][q] - lse) * 1.44269504088896f);
                        z[j][q] = there && c < a.V ? g * (c == t ? p - 1.f : p) : 0.f;
                        db[j][q] += z[j][q];
                    }
                    *reinterpret_cast<f32x4*>(ds + (wave * 16 + i16) * PV + j * 16 + 4 * h) = z[j];
                }
                if (a.dx) {
                    T* __restrict__ out = static_cast<T*>(a.dx) + row * a.d;
                    for (int k0 = 0; k0 < inner; k0 += 16) {
                        f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                        for (int j = 0; j < NF; ++j)
#pragma unroll
                            for (int q = 0; q < 4; ++q)
                                s = __builtin_amdgcn_mfma_f32_16x16x4f32(w[(j * 16 + 4 * h + q) * PK + k0 + i16], z[j][q], s, 0, 0, 0);
                        const int c = k0 + 4 * h, left = a.d - c;
                        if (there) {
                            const float v[4] = {s[0], s[1], s[2], s[3]};
                            if (left >= 4) {
                                store_floats<4>(out + c, v);
                            } else {
#pragma unroll
                                for (int q = 0; q < 3; ++q) {
                                    const float one[1] = {v[q]};
                                    if (q < left) store_floats<1>(out + c + q, one);
                                }
                            }
                        }
                    }
                }
                __syncthreads();
                if (a.dw)
#pragma unroll
                    for (int k = 0; k < KW; ++k) {
                        const int k0 = (wave + 4 * k) * 16;
                        if (k0 >= inner) break;
#pragma unroll
                        for (int r = 0; r < kNarrowRows; r += 16) {
                            if (g0 + r >= n) break;
                            float xt[4];
#pragma unroll
                            for (int q = 0; q < 4; ++q) xt[q] = xs[(r + 4 * h + q) * PK + k0 + i16];
#pragma unroll
                            for (int j = 0; j < NF; ++j)
#pragma unroll
                                for (int q = 0; q < 4; ++q)
                                    dw[k][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(ds[(r + 4 * h + q) * PV + j * 16 + i16], xt[q], dw[k][j], 0, 0, 0);
                        }
                    }
                __syncthreads();                             // before the next rows
            }
        }
    }

    if constexpr (!BWD) {
        total = wave_sum(total, 64);
        if (lane == 0) totals[wave][0] = total;
        __syncthreads();
        if (tid == 0) {
            const double sum = (totals[0][0] + totals[1][0]) + (totals[2][0] + totals[3][0]);
            if (gridDim.x > 1) {
                a.sums[2 * blockIdx.x] = sum;
                a.sums[2 * blockIdx.x + 1] = (double)many;
            } else {
                *a.count = (int)many;
                if (a.reduction != DA_LOSS_ROWS) *a.loss = (float)(a.reduction == DA_LOSS_MEAN ? sum / (double)max(1L, many) : sum);
            }
        }
    } else {
        const bool alone = gridDim.x == 1;
        float* __restrict__ part = a.part + (long)blockIdx.x * (a.d + 1) * a.V;
        if (a.dw)
#pragma unroll
            for (int k = 0; k < KW; ++k) {
                const int p = (wave + 4 * k) * 16 + i16;
                if (p >= a.d) continue;
#pragma unroll
                for (int j = 0; j < NF; ++j)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const int n = j * 16 + 4 * h + q;
                        if (n >= a.V) continue;
                        if (alone) {
                            const float one[1] = {dw[k][j][q]};
                            store_floats<1>(static_cast<T*>(a.dw) + (long)p * a.V + n, one);
                        } else {
                            part[(long)p * a.V + n] = dw[k][j][q];
                        }
                    }
            }
        if (a.db) {
            __syncthreads();
#pragma unroll
            for (int j = 0; j < NF; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    float s = db[j][q];
                    for (int m = 1; m < 16; m <<= 1) s += __shfl_xor(s, m, 64);
                    if (i16 == 0) ds[wave * PV + j * 16 + 4 * h + q] = s;
                }
            __syncthreads();
            if (tid < a.V) {
                const float s = (ds[tid] + ds[PV + tid]) + (ds[2 * PV + tid] + ds[3 * PV + tid]);
                if (alone) store_param(a.db, a.param_type, tid, s);
                else part[(long)a.d * a.V + tid] = s;
            }
        }
    }
}

// The number of rows with a target and, but for DA_LOSS_ROWS, the loss
__global__ __launch_bounds__(256) void ce_narrow_total_kernel(NarrowArgs a, int blocks)
{
    __shared__ double red[4][2];
    double s = 0.0, n = 0.0;
    for (int k = threadIdx.x; k < blocks; k += 256) {
        s += a.sums[2 * k];
        n += a.sums[2 * k + 1];
    }
    s = wave_sum(s, 64);
    n = wave_sum(n, 64);
    if ((threadIdx.x & 63) == 0) {
        red[threadIdx.x >> 6][0] = s;
        red[threadIdx.x >> 6][1] = n;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        s = (red[0][0] + red[1][0]) + (red[2][0] + red[3][0]);
        n = (red[0][1] + red[1][1]) + (red[2][1] + red[3][1]);
        *a.count = (int)n;
        if (a.reduction != DA_LOSS_ROWS) *a.loss = (float)(a.reduction == DA_LOSS_MEAN ? s / (n > 0.0 ? n : 1.0) : s);
    }
}

// dw and db from the blocks' parts: 16 numbers and 16 parts at once to a block
template <class T> __global__ __launch_bounds__(256) void ce_narrow_join_kernel(NarrowArgs a, int blocks)
{
    __shared__ float red[16][17];
    const long all = (long)(a.d + 1) * a.V, from = a.dw ? 0 : (long)a.d * a.V;
    const int k0 = threadIdx.x >> 4;
    for (long c0 = from + (long)blockIdx.x * 16; c0 < all; c0 += (long)gridDim.x * 16) {
        const long c = c0 + (threadIdx.x & 15);
        const bool take = c < (long)a.d * a.V || (c < all && a.db);
        float s[4] = {};
        if (take) {
            int k = k0;
            for (; k + 48 < blocks; k += 64)
#pragma unroll
                for (int u = 0; u < 4; ++u) s[u] += a.part[(k + u * 16) * all + c];
            for (; k < blocks; k += 16) s[0] += a.part[k * all + c];
        }
        red[k0][threadIdx.x & 15] = (s[0] + s[1]) + (s[2] + s[3]);
        __syncthreads();
        if (threadIdx.x < 16 && take) {
            float one[1] = {0.f};
            for (int i = 0; i < 16; ++i) one[0] += red[i][threadIdx.x];
            if (c < (long)a.d * a.V) store_floats<1>(static_cast<T*>(a.dw) + c, one);
            else store_param(a.db, a.param_type, c - (long)a.d * a.V, one[0]);
        }
        __syncthreads();                                     // before the next numbers
    }
}
// blocks of it; a launch has fewer than 2^32 threads
inline unsigned narrow_join_blocks(int64_t numbers) {
    const int64_t most = 1 << 20, blocks = (numbers + 15) / 16;
    return (unsigned)(blocks < most ? blocks : most);
}

}  // namespace daspmm
