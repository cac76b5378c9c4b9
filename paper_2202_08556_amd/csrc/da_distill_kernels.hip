// Distillation from a teacher's best classes, forward and backward.
//
//   p = softmax(t / T) over a row's entries, q = softmax(z / T) over all classes
//   loss = T^2 sum_k p_k (log p_k - log q_k),  dz_j = dloss T (q_j - sum of p over the entries of class j)
//
// Memory bounds it: z in once forward, z in and dz out backward; the entries are few beside that.  All logits are
// taken relative to the row's largest before they are scaled, and the backward pass gets the largest and the sum
// apart: as one number, their logarithm's rounding would be that of the logits' size, not of their spread.
//
//   narrow rows  P lanes hold a row in registers
//   wide rows    one block walks a row with a running maximum and sum; few rows are cut into pieces, a block each,
//                joined by distill_join_kernel
// 262144 x 41 float32 with 8 entries: 20 us forward, 37 backward (3 TB/s: rows of 164 bytes, a sixth of the bytes are entries).
// 2048 x 65536 bf16: 79 us forward, 109 backward (3.4 and 4.9 TB/s; a copy 5.2).
#pragma once
#include "da_layer_common.h"

#include <type_traits>

namespace daspmm {

constexpr int kDistillBlock = 256;
constexpr int kDistillMaxBest = 1024;

struct Teacher {
    long classes, best;
    const void* index;
    const void* top;
    int index64, top_dtype;
    float scale;                 // log2(e) / temperature

    __device__ long cls(long at) const {
        return index64 ? static_cast<const int64_t*>(index)[at] : (long)static_cast<const int32_t*>(index)[at];
    }
    __device__ bool has(long c) const { return c >= 0 && c < classes; }
    __device__ float logit(long at) const { return load_param(top, top_dtype, at); }
};

// An entry as the others of its row see it: its class, -1 where it is missing, and exp((t - largest) / T)
struct Entry { int cls; float p; };

// V logits from column c on, those past the end as -inf
template <class T, int V> __device__ __forceinline__ void load_logits(const T* __restrict__ row, long c, long end, float (&x)[V]) {
    if (c + V <= end) {
        load_floats<V>(row + c, x);
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            float one[1] = {-INFINITY};
            if (c + i < end) load_floats<1>(row + c + i, one);
            x[i] = one[0];
        }
    }
}
template <class T, int V> __device__ __forceinline__ void store_grads(T* __restrict__ row, long c, long end, const float (&x)[V]) {
    if (c + V <= end) {
        store_floats<V>(row + c, x);
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float one[1] = {x[i]};
            if (c + i < end) store_floats<1>(row + c + i, one);
        }
    }
}

// The larger one; NaN if one is.  A teacher's NaN would otherwise be a missing entry.
__device__ __forceinline__ float larger(float x, float o) { return o > x || o != o ? o : x; }

__device__ __forceinline__ float wave_max(float x, int lanes) {
    for (int d = 1; d < lanes; d <<= 1) x = larger(x, __shfl_xor(x, d, 64));
    return x;
}

// exp((x - largest) / T); scale = log2(e) / T.  The difference comes first: scaled, large logits would lose it.
__device__ __forceinline__ float shifted_exp(float x, float largest, float scale) { return exp2_hw((x - largest) * scale); }

// ------------------------------------------------------------------------------------------
// narrow rows: E accesses of V logits a lane.  BWD: a lane group's entries go through LDS, `best` slots of class and
// p for each, so that entries of one class are found; the first of them writes the gradient of its class over the
// one that its row's lanes wrote (the same wave, later).
// ------------------------------------------------------------------------------------------
template <class T, int V, int E, bool BWD>
__global__ __launch_bounds__(kDistillBlock) void distill_narrow_kernel(
    long rows, int P, Teacher te, const T* __restrict__ z, long ldz, float temperature, float* __restrict__ loss,
    float* __restrict__ stats, const float* __restrict__ dloss, long dloss_stride, T* __restrict__ dz)
{
    extern __shared__ Entry entries[];
    const int lane = threadIdx.x & (P - 1), per_block = kDistillBlock / P;
    Entry* mine = entries + (threadIdx.x / P) * te.best;
    const float inv_t = 1.f / temperature;
    for (long row = (long)blockIdx.x * per_block + threadIdx.x / P; row < rows; row += (long)gridDim.x * per_block) {
        const T* __restrict__ zp = z + row * ldz;
        float x[E][V];
#pragma unroll
        for (int e = 0; e < E; ++e) load_logits<T, V>(zp, (long)(lane + P * e) * V, te.classes, x[e]);
        // the teacher's entries
        float tmax = -INFINITY;
        for (long k = lane; k < te.best; k += P)
            if (te.has(te.cls(row * te.best + k))) tmax = larger(tmax, te.logit(row * te.best + k));
        tmax = wave_max(tmax, P);
        if constexpr (!BWD) {
            float m = -INFINITY, s = 0.f;
#pragma unroll
            for (int e = 0; e < E; ++e)
#pragma unroll
                for (int i = 0; i < V; ++i) m = fmaxf(m, x[e][i]);
            m = wave_max(m, P);
#pragma unroll
            for (int e = 0; e < E; ++e)
#pragma unroll
                for (int i = 0; i < V; ++i)
                    s += (lane + P * e) * V + i < te.classes ? shifted_exp(x[e][i], m, te.scale) : 0.f;
            s = wave_sum(s, P);
            float ps = 0.f, a = 0.f;
            for (long k = lane; k < te.best; k += P) {
                const long c = te.cls(row * te.best + k);
                if (!te.has(c)) continue;
                const float t = te.logit(row * te.best + k) - tmax;
                const float p = exp2_hw(t * te.scale);
                float zc[1];
                load_floats<1>(zp + c, zc);
                ps += p;
                if (p != 0.f) a += p * ((t - (zc[0] - m)) * inv_t);
            }
            ps = wave_sum(ps, P);
            a = wave_sum(a, P);
            if (lane == 0) {
                loss[row] = tmax == -INFINITY ? 0.f : temperature * temperature * (a / ps - logf(ps) + logf(s));
                if (stats) { stats[2 * row] = m; stats[2 * row + 1] = 1.f / s; }
            }
        } else {
            const float m = stats[2 * row], inv = stats[2 * row + 1];
            const float grad = tmax == -INFINITY ? 0.f : dloss[row * dloss_stride] * temperature;
            T* __restrict__ dp = dz + row * te.classes;
            float ps = 0.f;
            for (long k = lane; k < te.best; k += P) {
                const long c = te.cls(row * te.best + k);
                const float p = te.has(c) ? shifted_exp(te.logit(row * te.best + k), tmax, te.scale) : 0.f;
                ps += p;
                mine[k] = Entry{te.has(c) ? (int)c : -1, p};
            }
            ps = 1.f / wave_sum(ps, P);
#pragma unroll
            for (int e = 0; e < E; ++e) {
#pragma unroll
                for (int i = 0; i < V; ++i) x[e][i] = tmax == -INFINITY ? 0.f : grad * (shifted_exp(x[e][i], m, te.scale) * inv);
                store_grads<T, V>(dp, (long)(lane + P * e) * V, te.classes, x[e]);
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
            if (tmax != -INFINITY) {
                for (long k = lane; k < te.best; k += P) {
                    const int c = mine[k].cls;
                    if (c < 0) continue;
                    float p = 0.f;
                    bool first = true;
                    for (long j = 0; j < te.best; ++j) {
                        const Entry o = mine[j];
                        if (o.cls == c) {
                            p += o.p;
                            if (j < k) first = false;
                        }
                    }
                    if (!first) continue;
                    float zc[1];
                    load_floats<1>(zp + c, zc);
                    const float d[1] = {grad * (shifted_exp(zc[0], m, te.scale) * inv - p * ps)};
                    store_floats<1>(dp + c, d);
                }
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        }
    }
}

// ------------------------------------------------------------------------------------------
// wide rows
// ------------------------------------------------------------------------------------------
constexpr int kWideBlock = 512;

__device__ __forceinline__ void join_max_sum(float& m, float& s, float om, float os, float scale) {
    const float top = fmaxf(m, om);
    if (top != -INFINITY) {                                  // nothing but -inf so far: the sum stays as it is
        s = s * shifted_exp(m, top, scale) + os * shifted_exp(om, top, scale);
        m = top;
    } else {
        s += os;
    }
}

// Largest of a block's values, and their sum, for every thread
template <int BLOCK> __device__ __forceinline__ float block_max(float x, float* red) {
    x = wave_max(x, 64);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = x;
    __syncthreads();
    x = red[0];
    for (int w = 1; w < BLOCK / 64; ++w) x = larger(x, red[w]);
    return x;
}
template <int BLOCK> __device__ __forceinline__ float block_sum(float x, float* red) {
    x = wave_sum(x, 64);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = x;
    __syncthreads();
    x = red[0];
    for (int w = 1; w < BLOCK / 64; ++w) x += red[w];
    return x;
}

// A thread's first entry, asked for before the row's logits
struct FirstEntry {
    long cls = -1;
    float t = 0.f;
    __device__ void load(long row, const Teacher& te) {
        if (threadIdx.x < te.best) {
            cls = te.cls(row * te.best + threadIdx.x);
            t = te.logit(row * te.best + threadIdx.x);
            if (!te.has(cls)) cls = -1;
        }
    }
};

// loss of a row from its largest logit and sum, by all threads of a block
template <class T, int BLOCK>
__device__ __forceinline__ void row_loss(long row, const Teacher& te, const FirstEntry& first, const T* __restrict__ zp, float m,
                                         float s, float temperature, float* __restrict__ loss, float* __restrict__ stats, float* red)
{
    float tmax = first.cls >= 0 ? first.t : -INFINITY;
    for (long k = threadIdx.x + BLOCK; k < te.best; k += BLOCK)
        if (te.has(te.cls(row * te.best + k))) tmax = larger(tmax, te.logit(row * te.best + k));
    tmax = block_max<BLOCK>(tmax, red);
    const float inv_t = 1.f / temperature;
    float ps = 0.f, a = 0.f;
    auto add = [&](long c, float logit) {
        float zc[1];
        load_floats<1>(zp + c, zc);
        const float t = logit - tmax, p = exp2_hw(t * te.scale);
        ps += p;
        if (p != 0.f) a += p * ((t - (zc[0] - m)) * inv_t);
    };
    if (first.cls >= 0) add(first.cls, first.t);
    for (long k = threadIdx.x + BLOCK; k < te.best; k += BLOCK) {
        const long c = te.cls(row * te.best + k);
        if (te.has(c)) add(c, te.logit(row * te.best + k));
    }
    ps = block_sum<BLOCK>(ps, red);
    a = block_sum<BLOCK>(a, red);
    if (threadIdx.x == 0) {
        loss[row] = tmax == -INFINITY ? 0.f : temperature * temperature * (a / ps - logf(ps) + logf(s));
        if (stats) { stats[2 * row] = m; stats[2 * row + 1] = 1.f / s; }
    }
}

// A thread's logits of a turn of a block, U accesses of V, as they come from memory.  The next turn's are asked for before
// this one's are used: converted at once, they would be waited for.
template <class T, int V, int U> struct Turn {
    typedef typename std::conditional<sizeof(T) == 2, uint16_t, float>::type Raw;
    typename Pack<Raw, V>::type x[U];

    static __device__ __forceinline__ Raw none() {
        if constexpr (sizeof(T) == 2) return 0xff80u;        // -inf
        else return -INFINITY;
    }
    // from column c on; `whole`: the block's turn ends before `end`
    __device__ __forceinline__ void load(const T* __restrict__ row, long c, long end, bool whole) {
        const Raw* __restrict__ p = reinterpret_cast<const Raw*>(row);
        if (whole) {
#pragma unroll
            for (int u = 0; u < U; ++u) x[u] = *reinterpret_cast<const typename Pack<Raw, V>::type*>(p + c + (long)u * kWideBlock * V);
        } else {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const long at = c + (long)u * kWideBlock * V;
#pragma unroll
                for (int i = 0; i < V; ++i) x[u][i] = none();
                if (at + V <= end) x[u] = *reinterpret_cast<const typename Pack<Raw, V>::type*>(p + at);
                else
#pragma unroll
                    for (int i = 0; i < V - 1; ++i)
                        if (at + i < end) x[u][i] = p[at + i];
            }
        }
    }
    __device__ __forceinline__ float get(int u, int i) const {
        if constexpr (sizeof(T) == 2) return __uint_as_float((uint32_t)x[u][i] << 16);
        else return x[u][i];
    }
};
constexpr int kWideTurns = 4, kWideForwardTurns = 2;          // forward the logits are wanted twice, as floats: 4 cost half of the waves

// blockIdx.x: piece of `piece` columns; rows over blockIdx.y
template <class T, int V>
__global__ __launch_bounds__(kWideBlock) void distill_wide_kernel(long rows, long piece, Teacher te, const T* __restrict__ z,
                                                                  long ldz, float temperature, float* __restrict__ loss,
                                                                  float* __restrict__ stats, float2* __restrict__ part)
{
    __shared__ float red[kWideBlock / 64];
    constexpr int U = kWideForwardTurns;
    constexpr long TURN = (long)U * kWideBlock * V;
    for (long row = blockIdx.y; row < rows; row += gridDim.y) {
        const T* __restrict__ zp = z + row * ldz;
        const long c0 = blockIdx.x * piece, c1 = min(c0 + piece, te.classes);
        FirstEntry first;
        if (gridDim.x == 1) first.load(row, te);
        float m = -INFINITY, s = 0.f;
        Turn<T, V, U> next;
        next.load(zp, c0 + threadIdx.x * V, c1, c0 + TURN <= c1);
        for (long c = c0; c < c1; c += TURN) {
            const Turn<T, V, U> now = next;
            if (c + TURN < c1) next.load(zp, c + TURN + threadIdx.x * V, c1, c + 2 * TURN <= c1);
            float top = m;
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int i = 0; i < V; ++i) top = fmaxf(top, now.get(u, i));
            // nothing but -inf (or NaN) so far: taken relative to 0, where -inf adds nothing and NaN shows
            const float from = top == -INFINITY ? 0.f : top;
            s = m == -INFINITY ? s : s * shifted_exp(m, from, te.scale);
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int i = 0; i < V; ++i) s += shifted_exp(now.get(u, i), from, te.scale);
            m = top;
        }
        const float top = block_max<kWideBlock>(m, red);
        if (top != -INFINITY) s = m == -INFINITY ? s : s * shifted_exp(m, top, te.scale);
        s = block_sum<kWideBlock>(s, red);
        if (gridDim.x == 1) row_loss<T, kWideBlock>(row, te, first, zp, top, s, temperature, loss, stats, red);
        else if (threadIdx.x == 0) part[row * gridDim.x + blockIdx.x] = make_float2(top, s);
        __syncthreads();
    }
}

template <class T>
__global__ __launch_bounds__(256) void distill_join_kernel(long rows, int pieces, Teacher te, const T* __restrict__ z, long ldz,
                                                           float temperature, float* __restrict__ loss,
                                                           float* __restrict__ stats, const float2* __restrict__ part)
{
    __shared__ float red[4];
    for (long row = blockIdx.x; row < rows; row += gridDim.x) {
        FirstEntry first;
        first.load(row, te);
        float m = -INFINITY, s = 0.f;
        for (int k = 0; k < pieces; ++k) {                   // the same order for every thread
            const float2 p = part[row * pieces + k];
            join_max_sum(m, s, p.x, p.y, te.scale);
        }
        row_loss<T, 256>(row, te, first, z + row * ldz, m, s, temperature, loss, stats, red);
        __syncthreads();
    }
}

template <class T, int V>
__global__ __launch_bounds__(kWideBlock) void distill_wide_grad_kernel(
    long rows, long piece, Teacher te, const T* __restrict__ z, long ldz, float temperature, const float* __restrict__ stats,
    const float* __restrict__ dloss, long dloss_stride, T* __restrict__ dz)
{
    __shared__ float red[kWideBlock / 64];
    __shared__ Entry entries[kDistillMaxBest];
    constexpr int U = kWideTurns;
    constexpr long TURN = (long)U * kWideBlock * V;
    for (long row = blockIdx.y; row < rows; row += gridDim.y) {
        const T* __restrict__ zp = z + row * ldz;
        T* __restrict__ dp = dz + row * te.classes;
        const long c0 = blockIdx.x * piece, c1 = min(c0 + piece, te.classes);
        Turn<T, V, U> next;
        next.load(zp, c0 + threadIdx.x * V, c1, c0 + TURN <= c1);
        float tmax = -INFINITY, ps = 0.f;
        for (long k = threadIdx.x; k < te.best; k += kWideBlock)
            if (te.has(te.cls(row * te.best + k))) tmax = larger(tmax, te.logit(row * te.best + k));
        tmax = block_max<kWideBlock>(tmax, red);
        for (long k = threadIdx.x; k < te.best; k += kWideBlock) {
            const long c = te.cls(row * te.best + k);
            const float p = te.has(c) ? shifted_exp(te.logit(row * te.best + k), tmax, te.scale) : 0.f;
            ps += p;
            entries[k] = Entry{te.has(c) ? (int)c : -1, p};
        }
        ps = 1.f / block_sum<kWideBlock>(ps, red);
        const float m = stats[2 * row], inv = stats[2 * row + 1];
        const bool none = tmax == -INFINITY;
        const float grad = none ? 0.f : dloss[row * dloss_stride] * temperature;
        const float ginv = grad * inv;
        for (long c = c0; c < c1; c += TURN) {
            const Turn<T, V, U> now = next;
            if (c + TURN < c1) next.load(zp, c + TURN + threadIdx.x * V, c1, c + 2 * TURN <= c1);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                float x[V];
#pragma unroll
                for (int i = 0; i < V; ++i) x[i] = none ? 0.f : ginv * shifted_exp(now.get(u, i), m, te.scale);
                store_grads<T, V>(dp, c + threadIdx.x * V + (long)u * kWideBlock * V, c1, x);
            }
        }
        __syncthreads();                                     // the gradients of the entries' classes come over the others
        if (!none) {
            for (long k = threadIdx.x; k < te.best; k += kWideBlock) {
                const int c = entries[k].cls;
                if (c < c0 || c >= c1) continue;
                float p = 0.f;
                bool first = true;
                for (long j = 0; j < te.best; ++j) {
                    const Entry o = entries[j];
                    if (o.cls == c) {
                        p += o.p;
                        if (j < k) first = false;
                    }
                }
                if (!first) continue;
                float zc[1];
                load_floats<1>(zp + c, zc);
                const float d[1] = {grad * (shifted_exp(zc[0], m, te.scale) * inv - p * ps)};
                store_floats<1>(dp + c, d);
            }
        }
        __syncthreads();
    }
}

}  // namespace daspmm
