// Group norm with an activation, channels last, on samples of any length.
//
//   mean, var over the n = rows x cg numbers of a sample and group;  r = 1 / sqrt(var + eps)
//   xh = (x - mean) r,  z = xh w + b,  y = act(z)
//   dz = dy act'(z),  db = sum dz,  dw = sum dz xh,  e = dz w,  dx = r (e - mean(e) - xh mean(e xh))
//
// Memory bounds it: x in and y out, and x, dy in and dx out.  Three ways through the data, by the size of a sample
// (the host chooses):
//   each   a sample is one row: the numbers of one group are a few lanes' registers
//   team   a sample (some of its groups) is one wave's or block's: read once where the registers hold it
//   split  a sample is cut into chunks of rows, one block each: partial statistics, their sum, and a second pass
// Statistics are held in 32 bits: as sums of squares about the mean where the data stays in registers, about the
// first number of a chunk's column otherwise, joined by the formula for the variance of a union; never as the mean of
// squares less the square of the mean, which loses everything where the mean is large.
// All sums are taken in an order that follows from the sizes alone: results are the same from run to run.
#pragma once
#include "da_layer_common.h"

namespace daspmm {

constexpr int kNormBlock = 256;

struct NormShape {
    long rows, samples;
    const int* offsets;          // rows of sample s: offsets[s] .. offsets[s + 1]; null: every sample has `length`
    long length;
    int C, G, cg;
    float eps;
    int act, param_dtype;
    const void *w, *b;           // null: 1 and 0

    __device__ void range(long s, long* r0, long* r1) const {
        if (offsets) {           // offsets that are no valid ones read and write no other memory
            const long a = offsets[s], e = offsets[s + 1];
            *r0 = a < 0 ? 0 : a > rows ? rows : a;
            *r1 = e < *r0 ? *r0 : e > rows ? rows : e;
        } else {
            *r0 = s * length;
            *r1 = *r0 + length;
        }
    }
    template <int V> __device__ void params(int col, float (&wv)[V], float (&bv)[V]) const {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            wv[i] = w ? load_param(w, param_dtype, col + i) : 1.f;
            bv[i] = b ? load_param(b, param_dtype, col + i) : 0.f;
        }
    }
};

// ------------------------------------------------------------------------------------------
// each: P lanes hold the cg numbers of one row and group, E accesses of V numbers a lane.  The lane groups of a
// launch are a multiple of G, so that a lane keeps its columns (parameters and their gradients in registers) from
// row to row.  BWD: statistics are taken again from the registers; part receives this block's sums of dw and db.
// ------------------------------------------------------------------------------------------
template <class T, int V, int E, bool BWD>
__global__ __launch_bounds__(kNormBlock) void norm_each_kernel(NormShape sh, int P, const T* __restrict__ x, long ldx,
                                                               const T* __restrict__ dy, long ldy, T* __restrict__ out,
                                                               float* __restrict__ part)
{
    __shared__ float sums[BWD ? 2 * kNormBlock * V * E : 1];
    const int lane = threadIdx.x & (P - 1), per_block = kNormBlock / P;
    const long first = (long)blockIdx.x * per_block + threadIdx.x / P;
    const long groups = (long)gridDim.x * per_block;
    const int g = (int)(first % sh.G);
    const long step = groups / sh.G;
    const float inv = 1.f / (float)sh.cg;
    float wv[E][V], bv[E][V], aw[E][V] = {}, ab[E][V] = {};
    bool on[E];
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const int at = (lane + P * e) * V;
        on[e] = at < sh.cg;
        sh.params<V>(g * sh.cg + (on[e] ? at : 0), wv[e], bv[e]);
    }
    for (long row = first / sh.G; row < sh.rows; row += step) {
        float v[E][V], d[E][V];
        float s = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int col = g * sh.cg + (lane + P * e) * V;
            if (on[e]) {
                load_floats<V>(x + row * ldx + col, v[e]);
                if constexpr (BWD) load_floats<V>(dy + row * ldy + col, d[e]);
            }
        }
#pragma unroll
        for (int e = 0; e < E; ++e)
#pragma unroll
            for (int i = 0; i < V; ++i) s += on[e] ? v[e][i] : 0.f;
        const float mean = wave_sum(s, P) * inv;
        s = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                v[e][i] -= mean;
                s += on[e] ? v[e][i] * v[e][i] : 0.f;
            }
        const float r = 1.f / sqrtf(wave_sum(s, P) * inv + sh.eps);
        if constexpr (!BWD) {
#pragma unroll
            for (int e = 0; e < E; ++e) {
                if (!on[e]) continue;
#pragma unroll
                for (int i = 0; i < V; ++i) v[e][i] = act_value(sh.act, v[e][i] * r * wv[e][i] + bv[e][i]);
                store_floats<V>(out + row * sh.C + g * sh.cg + (lane + P * e) * V, v[e]);
            }
        } else {
            float s1 = 0.f, s2 = 0.f;
#pragma unroll
            for (int e = 0; e < E; ++e) {
                if (!on[e]) continue;
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    float value;
                    const float xh = v[e][i] * r;
                    const float dz = d[e][i] * act_slope(sh.act, xh * wv[e][i] + bv[e][i], &value);
                    aw[e][i] += dz * xh;
                    ab[e][i] += dz;
                    d[e][i] = dz * wv[e][i];
                    v[e][i] = xh;
                    s1 += d[e][i];
                    s2 += d[e][i] * xh;
                }
            }
            s1 = wave_sum(s1, P) * inv;
            s2 = wave_sum(s2, P) * inv;
#pragma unroll
            for (int e = 0; e < E; ++e) {
                if (!on[e]) continue;
#pragma unroll
                for (int i = 0; i < V; ++i) v[e][i] = r * (d[e][i] - s1 - v[e][i] * s2);
                store_floats<V>(out + row * sh.C + g * sh.cg + (lane + P * e) * V, v[e]);
            }
        }
    }
    if constexpr (BWD) {
        // [lane group][position in the group], once for dw and once for db
        const int width = P * E * V;
#pragma unroll
        for (int e = 0; e < E; ++e)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int at = (threadIdx.x / P) * width + (lane + P * e) * V + i;
                sums[at] = aw[e][i];
                sums[kNormBlock * V * E + at] = ab[e][i];
            }
        __syncthreads();
        const long base = (long)blockIdx.x * per_block;
        for (int c = threadIdx.x; c < 2 * sh.C; c += kNormBlock) {
            const int col = c < sh.C ? c : c - sh.C, cg = col / sh.cg, pos = col % sh.cg;
            float s = 0.f;
            for (int j = (int)(((long)cg - base % sh.G + sh.G) % sh.G); j < per_block; j += sh.G)
                s += sums[(c < sh.C ? 0 : kNormBlock * V * E) + j * width + pos];
            part[(long)blockIdx.x * 2 * sh.C + c] = s;
        }
    }
}

// ------------------------------------------------------------------------------------------
// team: TEAM threads own a sample's GT groups (blockIdx.y says which), TX = GT cg / V of them side by side along the
// columns, the others along the rows, kTeamRows rows a thread in registers; rows beyond that are read again.
// stats: mean and r of every sample and group, written forward and read backward.
// Samples of more than `longest` rows are left to the split kernels.
// ------------------------------------------------------------------------------------------
template <int V> constexpr int team_rows() { return V >= 8 ? 4 : 8; }

template <int TEAM> __device__ __forceinline__ void team_sync() {
    if constexpr (TEAM == 64) {
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    } else {
        __syncthreads();
    }
}

template <class T, int V, int TEAM, bool BWD>
__global__ __launch_bounds__(TEAM < 256 ? 256 : TEAM) void norm_team_kernel(
    NormShape sh, int GT, long longest, const T* __restrict__ x, long ldx, const T* __restrict__ dy, long ldy,
    T* __restrict__ out, float* __restrict__ stats, float* __restrict__ part)
{
    constexpr int BLOCK = TEAM < 256 ? 256 : TEAM, TEAMS = BLOCK / TEAM, E = team_rows<V>();
    __shared__ float red_mem[TEAMS][2][TEAM], tot_mem[TEAMS][2][TEAM];
    const int team = threadIdx.x / TEAM, t = threadIdx.x % TEAM;
    float (&red)[2][TEAM] = red_mem[team];
    float (&tot)[2][TEAM] = tot_mem[team];
    const int cgv = sh.cg / V, TX = GT * cgv, TY = TEAM / TX;
    const int tx = t % TX, ty = t / TX;
    const int g0 = blockIdx.y * GT, gn = min(GT, sh.G - g0);
    const bool on = ty < TY && tx < gn * cgv;
    const int col = g0 * sh.cg + tx * V, g = g0 + tx / cgv;

    // sums over a group's threads, for every thread of the group
    auto join = [&](float& a, float& b) {
        red[0][t] = on ? a : 0.f;
        red[1][t] = on ? b : 0.f;
        team_sync<TEAM>();
        if (t < TX) {
            float p = 0.f, q = 0.f;
            for (int k = 0; k < TY; ++k) { p += red[0][t + k * TX]; q += red[1][t + k * TX]; }
            red[0][t] = p;
            red[1][t] = q;
        }
        team_sync<TEAM>();
        if (t < GT) {
            float p = 0.f, q = 0.f;
            for (int k = 0; k < cgv; ++k) { p += red[0][t * cgv + k]; q += red[1][t * cgv + k]; }
            tot[0][t] = p;
            tot[1][t] = q;
        }
        team_sync<TEAM>();
        a = tot[0][tx / cgv];
        b = tot[1][tx / cgv];
    };

    float wv[V], bv[V], aw[V] = {}, ab[V] = {};
    sh.params<V>(on ? col : 0, wv, bv);
    for (long s = (long)blockIdx.x * TEAMS + team; s < sh.samples; s += (long)gridDim.x * TEAMS) {
        long r0, r1;
        sh.range(s, &r0, &r1);
        const int n = r1 - r0 > longest ? 0 : (int)(r1 - r0);
        if (n == 0) continue;                                // the whole team's
        const float inv = 1.f / ((float)n * (float)sh.cg);
        const T* __restrict__ xp = x + r0 * ldx + col;
        const T* __restrict__ dp = BWD ? dy + r0 * ldy + col : nullptr;
        T* __restrict__ op = out + r0 * sh.C + col;
        float v[E][V], d[BWD ? E : 1][V];
        if (on) {
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const int row = ty + TY * e;
                if (row < n) {
                    load_floats<V>(xp + (long)row * ldx, v[e]);
                    if constexpr (BWD) load_floats<V>(dp + (long)row * ldy, d[e]);
                }
            }
        }
        const int rest = ty + TY * E;                        // first row that is not in registers
        if constexpr (!BWD) {
            float a = 0.f, b = 0.f;
            if (on) {
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (ty + TY * e < n)
#pragma unroll
                        for (int i = 0; i < V; ++i) a += v[e][i];
                for (int row = rest; row < n; row += TY) {
                    float u[V];
                    load_floats<V>(xp + (long)row * ldx, u);
#pragma unroll
                    for (int i = 0; i < V; ++i) a += u[i];
                }
            }
            join(a, b);
            const float mean = a * inv;
            a = 0.f;
            if (on) {
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (ty + TY * e < n)
#pragma unroll
                        for (int i = 0; i < V; ++i) { v[e][i] -= mean; a += v[e][i] * v[e][i]; }
                for (int row = rest; row < n; row += TY) {
                    float u[V];
                    load_floats<V>(xp + (long)row * ldx, u);
#pragma unroll
                    for (int i = 0; i < V; ++i) { u[i] -= mean; a += u[i] * u[i]; }
                }
            }
            join(a, b);
            const float r = 1.f / sqrtf(a * inv + sh.eps);
            if (stats && t < gn) {
                float q = 0.f;
                q = tot[0][t];
                stats[(s * sh.G + g0 + t) * 2 + 1] = 1.f / sqrtf(q * inv + sh.eps);
            }
            if (stats && on && ty == 0 && tx % cgv == 0) stats[(s * sh.G + g) * 2] = mean;
            if (on) {
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const int row = ty + TY * e;
                    if (row < n) {
#pragma unroll
                        for (int i = 0; i < V; ++i) v[e][i] = act_value(sh.act, v[e][i] * r * wv[i] + bv[i]);
                        store_floats<V>(op + (long)row * sh.C, v[e]);
                    }
                }
                for (int row = rest; row < n; row += TY) {
                    float u[V];
                    load_floats<V>(xp + (long)row * ldx, u);
#pragma unroll
                    for (int i = 0; i < V; ++i) u[i] = act_value(sh.act, (u[i] - mean) * r * wv[i] + bv[i]);
                    store_floats<V>(op + (long)row * sh.C, u);
                }
            }
        } else {
            float s1 = 0.f, s2 = 0.f, mean = 0.f, r = 0.f;
            auto step = [&](float (&u)[V], float (&dd)[V]) {     // x and dy become xh and e
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    float value;
                    const float xh = (u[i] - mean) * r;
                    const float dz = dd[i] * act_slope(sh.act, xh * wv[i] + bv[i], &value);
                    u[i] = xh;
                    dd[i] = dz * wv[i];
                    aw[i] += dz * xh;
                    ab[i] += dz;
                    s1 += dd[i];
                    s2 += dd[i] * xh;
                }
            };
            if (on) {
                mean = stats[(s * sh.G + g) * 2];
                r = stats[(s * sh.G + g) * 2 + 1];
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (ty + TY * e < n) step(v[e], d[e]);
                for (int row = rest; row < n; row += TY) {
                    float u[V], dd[V];
                    load_floats<V>(xp + (long)row * ldx, u);
                    load_floats<V>(dp + (long)row * ldy, dd);
                    step(u, dd);
                }
            }
            join(s1, s2);
            const float m1 = s1 * inv, m2 = s2 * inv;
            if (on) {
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const int row = ty + TY * e;
                    if (row < n) {
#pragma unroll
                        for (int i = 0; i < V; ++i) v[e][i] = r * (d[e][i] - m1 - v[e][i] * m2);
                        store_floats<V>(op + (long)row * sh.C, v[e]);
                    }
                }
                for (int row = rest; row < n; row += TY) {
                    float u[V], dd[V];
                    load_floats<V>(xp + (long)row * ldx, u);
                    load_floats<V>(dp + (long)row * ldy, dd);
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        float value;
                        const float xh = (u[i] - mean) * r;
                        const float e = dd[i] * act_slope(sh.act, xh * wv[i] + bv[i], &value) * wv[i];
                        u[i] = r * (e - m1 - xh * m2);
                    }
                    store_floats<V>(op + (long)row * sh.C, u);
                }
            }
        }
    }
    if constexpr (BWD) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            __syncthreads();
            red[0][t] = on ? aw[i] : 0.f;
            red[1][t] = on ? ab[i] : 0.f;
            __syncthreads();
            if (threadIdx.x < gn * cgv) {
                float p = 0.f, q = 0.f;
                for (int m = 0; m < TEAMS; ++m)
                    for (int k = 0; k < TY; ++k) { p += red_mem[m][0][t + k * TX]; q += red_mem[m][1][t + k * TX]; }
                part[(long)blockIdx.x * 2 * sh.C + col + i] = p;
                part[(long)blockIdx.x * 2 * sh.C + sh.C + col + i] = q;
            }
        }
    }
}

// ------------------------------------------------------------------------------------------
// split: chunks of `per` rows of one sample.  Ragged samples' chunks come from a table that norm_long_kernel fills
// with the samples of more than `longest` rows (in any order: nothing is summed in the order of the table).
// ------------------------------------------------------------------------------------------
struct NormChunks {
    long per, each, count;       // rows of a chunk; chunks of a sample of equal samples; chunks (the most, where ragged)
    const int2* table;           // ragged: sample and number within the sample of a chunk; null: equal samples
    const int* counts;           // ragged: chunks, long samples
    const int4* list;            // ragged: sample, its first chunk, its chunks

    __device__ bool find(const NormShape& sh, long c, long* s, long* r0, long* r1) const {
        long i;
        if (table) {
            if (c >= counts[0]) return false;
            const int2 e = table[c];
            *s = e.x;
            i = e.y;
        } else {
            *s = c / each;
            i = c % each;
        }
        long a, e;
        sh.range(*s, &a, &e);
        *r0 = a + i * per;
        *r1 = min(*r0 + per, e);
        return true;
    }
    // the k-th sample's number, first chunk and chunks
    __device__ bool sample(long k, long* s, long* first, long* n) const {
        if (table) {
            if (k >= counts[1]) return false;
            const int4 e = list[k];
            *s = e.x;
            *first = e.y;
            *n = e.z;
        } else {
            *s = k;
            *first = k * each;
            *n = each;
        }
        return true;
    }
};

__global__ __launch_bounds__(64) void norm_clear_kernel(int* counts) {
    if (threadIdx.x < 2) counts[threadIdx.x] = 0;
}

__global__ __launch_bounds__(256) void norm_long_kernel(NormShape sh, long longest, long per, int* counts, int2* table,
                                                        int4* list)
{
    const long s = (long)blockIdx.x * 256 + threadIdx.x;
    long r0 = 0, r1 = 0;
    if (s < sh.samples) sh.range(s, &r0, &r1);
    const bool is_long = r1 - r0 > longest;
    int n = 0, first = 0;
    if (is_long) {
        n = (int)((r1 - r0 + per - 1) / per);
        first = atomicAdd(&counts[0], n);
        list[atomicAdd(&counts[1], 1)] = make_int4((int)s, first, n, 0);
    }
    for (unsigned long long left = __ballot(is_long); left; left &= left - 1) {
        const int who = __ffsll(left) - 1;
        const int m = __shfl(n, who), f = __shfl(first, who), sample = __shfl((int)s, who);
        for (int i = threadIdx.x & 63; i < m; i += 64) table[f + i] = make_int2(sample, i);
    }
}

// mean and sum of squares about it of a chunk's columns, V columns together
template <class T, int V>
__global__ __launch_bounds__(kNormBlock) void norm_stats_kernel(NormShape sh, NormChunks ch, int TX, const T* __restrict__ x,
                                                                long ldx, float2* __restrict__ part)
{
    __shared__ float red[2][kNormBlock];
    long s, r0, r1;
    if (!ch.find(sh, blockIdx.x, &s, &r0, &r1)) return;
    const int TY = kNormBlock / TX, t = threadIdx.x, tx = t % TX, ty = t / TX, cv = sh.C / V;
    const int vec = blockIdx.y * TX + tx;
    const bool on = ty < TY && vec < cv;
    const T* __restrict__ xp = x + (long)vec * V;
    float a = 0.f, b = 0.f, shift = 0.f;
    if (on) {
        float u[V];
        load_floats<V>(xp + r0 * ldx, u);
        shift = u[0];
        constexpr int U = 4;
        long row = r0 + ty;
        for (; row + (U - 1) * TY < r1; row += U * TY) {
            float m[U][V];
#pragma unroll
            for (int k = 0; k < U; ++k) load_floats<V>(xp + (row + k * TY) * ldx, m[k]);
#pragma unroll
            for (int k = 0; k < U; ++k)
#pragma unroll
                for (int i = 0; i < V; ++i) { const float c = m[k][i] - shift; a += c; b += c * c; }
        }
        for (; row < r1; row += TY) {
            load_floats<V>(xp + row * ldx, u);
#pragma unroll
            for (int i = 0; i < V; ++i) { const float c = u[i] - shift; a += c; b += c * c; }
        }
    }
    red[0][t] = a;
    red[1][t] = b;
    __syncthreads();
    if (t < TX && vec < cv) {
        for (int k = 1; k < TY; ++k) { a += red[0][t + k * TX]; b += red[1][t + k * TX]; }
        const float n = (float)(r1 - r0) * V, m = a / n;
        part[(long)blockIdx.x * cv + vec] = make_float2(shift + m, fmaxf(b - a * m, 0.f) + (b - b));   // NaN stays NaN
    }
}

// Joins a sample's parts: one wave for a sample and group
template <int V>
__global__ __launch_bounds__(64) void norm_join_kernel(NormShape sh, NormChunks ch, const float2* __restrict__ part,
                                                       float* __restrict__ stats)
{
    long s, first, chunks, r0, r1;
    if (!ch.sample(blockIdx.x, &s, &first, &chunks)) return;
    sh.range(s, &r0, &r1);
    const int g = blockIdx.y, cgv = sh.cg / V, cv = sh.C / V;
    const long parts = chunks * cgv;
    const float total = (float)(r1 - r0) * (float)sh.cg;
    auto at = [&](long k, float* n) {
        const long c = k / cgv;
        const long rows = min(ch.per, (r1 - r0) - c * ch.per);
        *n = (float)rows * V;
        return part[(first + c) * cv + g * cgv + k % cgv];
    };
    float a = 0.f, n;
    const float origin = at(0, &n).x;
    for (long k = threadIdx.x; k < parts; k += 64) { const float2 p = at(k, &n); a += (p.x - origin) * n; }
    const float mean = origin + wave_sum(a, 64) / total;
    float m2 = 0.f;
    for (long k = threadIdx.x; k < parts; k += 64) {
        const float2 p = at(k, &n);
        m2 += p.y + n * (p.x - mean) * (p.x - mean);
    }
    m2 = wave_sum(m2, 64);
    if (threadIdx.x == 0) {
        stats[(s * sh.G + g) * 2] = mean;
        stats[(s * sh.G + g) * 2 + 1] = 1.f / sqrtf(m2 / total + sh.eps);
    }
}

// y of a chunk; BWD: dx, with the means of e and e xh of every sample and group in `means`
template <class T, int V, bool BWD>
__global__ __launch_bounds__(kNormBlock) void norm_apply_kernel(NormShape sh, NormChunks ch, int TX, const T* __restrict__ x,
                                                                long ldx, const T* __restrict__ dy, long ldy,
                                                                const float* __restrict__ stats,
                                                                const float* __restrict__ means, T* __restrict__ out)
{
    long s, r0, r1;
    if (!ch.find(sh, blockIdx.x, &s, &r0, &r1)) return;
    const int TY = kNormBlock / TX, tx = threadIdx.x % TX, ty = threadIdx.x / TX;
    const int vec = blockIdx.y * TX + tx;
    if (ty >= TY || vec >= sh.C / V) return;
    const int col = vec * V, g = col / sh.cg;
    float wv[V], bv[V];
    sh.params<V>(col, wv, bv);
    const float mean = stats[(s * sh.G + g) * 2], r = stats[(s * sh.G + g) * 2 + 1];
    float m1 = 0.f, m2 = 0.f;
    if constexpr (BWD) {
        m1 = means[(s * sh.G + g) * 2];
        m2 = means[(s * sh.G + g) * 2 + 1];
    }
    constexpr int U = 2;
    auto put = [&](long row, float (&u)[V], float (&d)[V]) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float xh = (u[i] - mean) * r, z = xh * wv[i] + bv[i];
            if constexpr (!BWD) {
                u[i] = act_value(sh.act, z);
            } else {
                float value;
                u[i] = r * (d[i] * act_slope(sh.act, z, &value) * wv[i] - m1 - xh * m2);
            }
        }
        store_floats<V>(out + row * sh.C + col, u);
    };
    long row = r0 + ty;
    for (; row + (U - 1) * TY < r1; row += U * TY) {
        float u[U][V], d[U][V];
#pragma unroll
        for (int k = 0; k < U; ++k) {
            load_floats<V>(x + (row + k * TY) * ldx + col, u[k]);
            if constexpr (BWD) load_floats<V>(dy + (row + k * TY) * ldy + col, d[k]);
        }
#pragma unroll
        for (int k = 0; k < U; ++k) put(row + k * TY, u[k], d[k]);
    }
    for (; row < r1; row += TY) {
        float u[V], d[V];
        load_floats<V>(x + row * ldx + col, u);
        if constexpr (BWD) load_floats<V>(dy + row * ldy + col, d);
        put(row, u, d);
    }
}

// Sums of dz xh and of dz over a chunk's columns
template <class T, int V>
__global__ __launch_bounds__(kNormBlock) void norm_grad_stats_kernel(NormShape sh, NormChunks ch, int TX, const T* __restrict__ x,
                                                                     long ldx, const T* __restrict__ dy, long ldy,
                                                                     const float* __restrict__ stats, float* __restrict__ part)
{
    __shared__ float red[2][kNormBlock];
    long s, r0, r1;
    if (!ch.find(sh, blockIdx.x, &s, &r0, &r1)) return;
    const int TY = kNormBlock / TX, t = threadIdx.x, tx = t % TX, ty = t / TX;
    const int vec = blockIdx.y * TX + tx, col = vec * V;
    const bool on = ty < TY && col < sh.C;
    float aw[V] = {}, ab[V] = {};
    if (on) {
        const int g = col / sh.cg;
        const float mean = stats[(s * sh.G + g) * 2], r = stats[(s * sh.G + g) * 2 + 1];
        float wv[V], bv[V];
        sh.params<V>(col, wv, bv);
        constexpr int U = 2;
        auto add = [&](float (&u)[V], float (&d)[V]) {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                float value;
                const float xh = (u[i] - mean) * r;
                const float dz = d[i] * act_slope(sh.act, xh * wv[i] + bv[i], &value);
                aw[i] += dz * xh;
                ab[i] += dz;
            }
        };
        long row = r0 + ty;
        for (; row + (U - 1) * TY < r1; row += U * TY) {
            float u[U][V], d[U][V];
#pragma unroll
            for (int k = 0; k < U; ++k) {
                load_floats<V>(x + (row + k * TY) * ldx + col, u[k]);
                load_floats<V>(dy + (row + k * TY) * ldy + col, d[k]);
            }
#pragma unroll
            for (int k = 0; k < U; ++k) add(u[k], d[k]);
        }
        for (; row < r1; row += TY) {
            float u[V], d[V];
            load_floats<V>(x + row * ldx + col, u);
            load_floats<V>(dy + row * ldy + col, d);
            add(u, d);
        }
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
        __syncthreads();
        red[0][t] = aw[i];
        red[1][t] = ab[i];
        __syncthreads();
        if (t < TX && col < sh.C) {
            float p = 0.f, q = 0.f;
            for (int k = 0; k < TY; ++k) { p += red[0][t + k * TX]; q += red[1][t + k * TX]; }
            part[(long)blockIdx.x * 2 * sh.C + col + i] = p;
            part[(long)blockIdx.x * 2 * sh.C + sh.C + col + i] = q;
        }
    }
}

// Means of e and e xh of a sample and group from the sums of its chunks' columns (e = dz w)
__global__ __launch_bounds__(256) void norm_grad_join_kernel(NormShape sh, NormChunks ch, const float* __restrict__ part,
                                                             float* __restrict__ means)
{
    __shared__ float red[2][4];
    long s, first, chunks, r0, r1;
    if (!ch.sample(blockIdx.x, &s, &first, &chunks)) return;
    sh.range(s, &r0, &r1);
    const int g = blockIdx.y;
    const long n = chunks * sh.cg;
    float a = 0.f, b = 0.f;
    for (long k = threadIdx.x; k < n; k += 256) {
        const int col = g * sh.cg + (int)(k % sh.cg);
        const float w = sh.w ? load_param(sh.w, sh.param_dtype, col) : 1.f;
        const float* __restrict__ p = part + (first + k / sh.cg) * 2 * sh.C + col;
        a += w * p[sh.C];
        b += w * p[0];
    }
    a = wave_sum(a, 64);
    b = wave_sum(b, 64);
    if ((threadIdx.x & 63) == 0) { red[0][threadIdx.x >> 6] = a; red[1][threadIdx.x >> 6] = b; }
    __syncthreads();
    if (threadIdx.x == 0) {
        const float total = (float)(r1 - r0) * (float)sh.cg;
        means[(s * sh.G + g) * 2] = (red[0][0] + red[0][1] + red[0][2] + red[0][3]) / total;
        means[(s * sh.G + g) * 2 + 1] = (red[1][0] + red[1][1] + red[1][2] + red[1][3]) / total;
    }
}

// dw and db from the parts of all blocks: `fixed` rows of 2 C sums, then counts[0] (or `more`) rows at part2
__global__ __launch_bounds__(1024) void norm_param_grads_kernel(int C, const float* __restrict__ part, long fixed,
                                                                const float* __restrict__ part2, long more,
                                                                const int* __restrict__ counts, void* dw, void* db, int dtype)
{
    __shared__ float sh[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int c = blockIdx.x * 64 + lane;
    if (counts) more = counts[0];
    float s = 0.f;
    if (c < 2 * C) {
        constexpr int U = 8;
        float a[U] = {};
        auto sum = [&](const float* __restrict__ p, long n) {
            long k = wave;
            for (; k + (U - 1) * 16 < n; k += U * 16)
#pragma unroll
                for (int u = 0; u < U; ++u) a[u] += p[(k + u * 16) * 2 * C + c];
            for (; k < n; k += 16) a[0] += p[k * 2 * C + c];
        };
        sum(part, fixed);
        sum(part2, more);
#pragma unroll
        for (int u = 0; u < U; ++u) s += a[u];
    }
    sh[wave][lane] = s;
    __syncthreads();
    if (wave == 0 && c < 2 * C) {
        for (int k = 1; k < 16; ++k) s += sh[k][lane];
        if (c < C) { if (dw) store_param(dw, dtype, c, s); }
        else if (db) store_param(db, dtype, c - C, s);
    }
}

}  // namespace daspmm
