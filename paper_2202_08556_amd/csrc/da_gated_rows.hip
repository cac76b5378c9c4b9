// The gated feed-forward block forward for few rows (single tokens): every weight is read for a handful of products, so
// memory bounds it and the vector units do the arithmetic.
//
// A thread owns 16 bytes of a weight's line (V columns) and goes down the lines; LN threads lie side by side along the
// columns (up to 256, 4 KB of a line), the others of a block take other lines, U lines on their way at once.  Lines are
// also dealt to `splits` blocks until the chip is full; their sums meet in gated_rows_join_kernel in a fixed order.
// What is multiplied by the weights lies in LDS, R numbers (rows) to a line, so that one read serves them all.  a stays in
// 32 bits between the two products: in bfloat16 it would be the larger part of the error.
// One row of 4096 x 12288 bf16: 73 us for 302 MB (4.1 TB/s; a large copy 5.2); per element one instruction and one more for
// each row, so that memory stays the bound up to eight rows.
#pragma once
#include "da_gated_kernels.hip"

namespace daspmm {

constexpr int kRowsMost = 8, kRowsBlock = 256, kRowsLines = 256;      // rows; threads; lines whose factors are in LDS at once

template <class T> struct RowsArgs {
    const T *W0, *W1;            // kGate: gate and up
    int rows, N, K;
    int LN;                      // threads along the columns, a power of two
    int splits, per;             // blocks along the lines, lines of one
    float* part;                 // splits > 1: [split][row][N], of u and v side by side for kGate
    float* A32;                  // kGate: act(u) v
    T* C;                        // kStore: the result; kGate: act(u) v rounded, where not null
    float *U, *V;                // kGate: where not null
    int act;
};

// 16 bytes of a line, of which `left` elements are there, as they come from memory
template <class T> struct LinePiece {
    typename Mma<T>::Memory raw;
    __device__ __forceinline__ void load(const T* __restrict__ p, int left) {
        if (left >= Mma<T>::VEC) {
            raw = *reinterpret_cast<const typename Mma<T>::Memory*>(p);
        } else {
            const uint4 v = edge_chunk(p, left);
            __builtin_memcpy(&raw, &v, 16);
        }
    }
    __device__ __forceinline__ float get(int i) const {
        if constexpr (sizeof(T) == 2) return __uint_as_float((uint32_t)raw[i] << 16);
        else return raw[i];
    }
};

// What a finished sum becomes: columns n .. n + COUNT - 1 of row r, `left` of them there
template <class T, int EPI, int COUNT>
__device__ __forceinline__ void rows_finish(const RowsArgs<T>& g, int r, int n, int left, float (&x)[COUNT], float (&v)[COUNT]) {
    const long at = (long)r * g.N + n;
    if constexpr (EPI == kGate) {
        float a[COUNT];
#pragma unroll
        for (int i = 0; i < COUNT; ++i) a[i] = x[i];
        act_values(g.act, a);
#pragma unroll
        for (int i = 0; i < COUNT; ++i) {
            if (i >= left) break;
            const float one[1] = {a[i] * v[i]};
            g.A32[at + i] = one[0];
            if (g.C) store_floats<1>(g.C + at + i, one);
            if (g.U) { g.U[at + i] = x[i]; g.V[at + i] = v[i]; }
        }
    } else {
#pragma unroll
        for (int i = 0; i < COUNT; ++i) {
            const float one[1] = {x[i]};
            if (i < left) store_floats<1>(g.C + at + i, one);
        }
    }
}

// X: rows x K of TX (T, or float between the products), ldx
template <class T, class TX, int R, int EPI>
__global__ __launch_bounds__(kRowsBlock) void gated_rows_kernel(RowsArgs<T> g, const TX* __restrict__ X, long ldx)
{
    constexpr int V = Mma<T>::VEC, S = EPI == kGate ? 2 : 1, U = EPI == kGate ? 4 : 8;
    __shared__ __attribute__((aligned(16))) float factor[kRowsLines][R];
    __shared__ float sums[kRowsBlock][V];
    const int tid = threadIdx.x, ln = tid & (g.LN - 1), kg = tid / g.LN, KG = kRowsBlock / g.LN;
    const int n = (blockIdx.x * g.LN + ln) * V, left = g.N - n;
    const int k0 = blockIdx.y * g.per, k1 = min(k0 + g.per, g.K);
    float acc[S][R][V] = {};
    auto add = [&](int line, const LinePiece<T> (&w)[S]) {
        float f[R];
#pragma unroll
        for (int r = 0; r < R; ++r) f[r] = factor[line][r];
#pragma unroll
        for (int s = 0; s < S; ++s)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float x = w[s].get(i);
#pragma unroll
                for (int r = 0; r < R; ++r) acc[s][r][i] += f[r] * x;
            }
    };
    for (int base = k0; base < k1; base += kRowsLines) {
        const int lines = min(kRowsLines, k1 - base);
        const T* __restrict__ p0 = g.W0 + (long)base * g.N + n;
        const T* __restrict__ p1 = EPI == kGate ? g.W1 + (long)base * g.N + n : nullptr;
        LinePiece<T> next[U][S];
        auto load = [&](int from) {                          // lines past the last are the last one
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const long at = (long)min(from + u * KG, lines - 1) * g.N;
                next[u][0].load(p0 + at, left);
                if constexpr (EPI == kGate) next[u][1].load(p1 + at, left);
            }
        };
        load(kg);                                            // on their way while the factors are laid out
        __syncthreads();
        for (int q = tid; q < lines * R; q += kRowsBlock) {
            const int r = q / lines, line = q % lines;
            float one[1] = {0.f};
            if (r < g.rows) load_floats<1>(X + r * ldx + base + line, one);
            factor[line][r] = one[0];
        }
        __syncthreads();
        for (int line = kg; line < lines; line += U * KG) {
            LinePiece<T> now[U][S];
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int s = 0; s < S; ++s) now[u][s] = next[u][s];
            if (line + U * KG < lines) load(line + U * KG);
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (line + u * KG < lines) add(line + u * KG, now[u]);
        }
    }
    // over the lines' threads, one row and weight at a time
#pragma unroll
    for (int r = 0; r < R; ++r) {
        if (r >= g.rows) break;                              // the same for all
        float x[S][V];
#pragma unroll
        for (int s = 0; s < S; ++s) {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < V; ++i) sums[tid][i] = acc[s][r][i];
            __syncthreads();
            if (kg == 0)
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    float t = sums[ln][i];
                    for (int q = 1; q < KG; ++q) t += sums[ln + q * g.LN][i];
                    x[s][i] = t;
                }
        }
        if (kg != 0 || left <= 0) continue;
        if (g.splits > 1) {
            float* p = g.part + ((long)blockIdx.y * g.rows + r) * g.N * S + n;
#pragma unroll
            for (int s = 0; s < S; ++s)
#pragma unroll
                for (int i = 0; i < V; ++i)
                    if (i < left) p[(long)s * g.N + i] = x[s][i];
        } else {
            rows_finish<T, EPI, V>(g, r, n, left, x[0], x[S - 1]);
        }
    }
}

// Adds the splits' sums: 64 columns to a block, 4 shares of the splits
template <class T, int EPI>
__global__ __launch_bounds__(kRowsBlock) void gated_rows_join_kernel(RowsArgs<T> g)
{
    constexpr int S = EPI == kGate ? 2 : 1, U = 8;
    __shared__ float sums[S][4][64];
    const int col = threadIdx.x & 63, share = threadIdx.x >> 6, n = blockIdx.x * 64 + col, r = blockIdx.y;
    const long plane = (long)g.rows * g.N * S;
    float x[S] = {};
    if (n < g.N) {
        const float* __restrict__ p = g.part + (long)r * g.N * S + n;
#pragma unroll
        for (int s = 0; s < S; ++s) {
            float a[U] = {};
            int k = share;
            for (; k + (U - 1) * 4 < g.splits; k += U * 4)
#pragma unroll
                for (int u = 0; u < U; ++u) a[u] += p[(k + u * 4) * plane + (long)s * g.N];
            for (; k < g.splits; k += 4) a[0] += p[k * plane + (long)s * g.N];
#pragma unroll
            for (int u = 0; u < U; ++u) x[s] += a[u];
        }
    }
#pragma unroll
    for (int s = 0; s < S; ++s) sums[s][share][col] = x[s];
    __syncthreads();
    if (share == 0 && n < g.N) {
        float a[1] = {(sums[0][0][col] + sums[0][1][col]) + (sums[0][2][col] + sums[0][3][col])};
        float v[1] = {(sums[S - 1][0][col] + sums[S - 1][1][col]) + (sums[S - 1][2][col] + sums[S - 1][3][col])};
        rows_finish<T, EPI, 1>(g, r, n, 1, a, v);
    }
}

}  // namespace daspmm
