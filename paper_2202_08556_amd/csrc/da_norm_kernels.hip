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
// Variance: where every row is a sample, sums of squares about the mean, both from registers.  Elsewhere one pass takes the
// sums of c = x - s and of c^2, s the first number of the sample's or chunk's group, in 64 bits: s is one of the n numbers,
// so sum c^2 exceeds the sum of squares about the mean by a factor of at most about n, however far s is from the others (a
// first row of padding, a mean that is large), and the difference keeps all 24 bits.  In 32 bits it would lose them.  Chunks
// are joined by the formula for the variance of a union, in 64 bits for the same reason.  The additions in 64 bits took a
// first pass from 31 to 33 us (8000 samples of 23 rows x 96 float32), from 16 to 19 (30011 x 602 bf16, accesses of 4 bytes) and
// nothing where memory is the bound (262144 x 256 float32).  All else is held in 32 bits.
// All sums are taken in an order that follows from the sizes alone: results are the same from run to run.
#pragma once
#include "da_layer_common.h"

#include <type_traits>

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
// launch are a multiple of G (or have a row each), so that a lane keeps its columns (parameters and their gradients in
// registers) from row to row.  BWD: statistics are taken again from the registers; part receives sums of dw and db: a row of
// 2 C for every block, or, where a block has no group twice, for every lane group of a group.  (A row for every block would be
// 64 MB for one row of 8008 numbers in 1001 groups.)
// 262144 rows of 128 bf16 in groups of 32 with gelu: 37 us forward, 59 backward (3.6 and 3.4 TB/s; a copy 5.2).  The vector
// instructions, some 27 and 45 a number, take as long as the bytes.
// ------------------------------------------------------------------------------------------
template <class T, int V, int E, bool BWD>
__global__ __launch_bounds__(kNormBlock) void norm_each_kernel(NormShape sh, int P, const T* __restrict__ x, long ldx,
                                                               const T* __restrict__ dy, long ldy, T* __restrict__ out,
                                                               float* __restrict__ part)
{
    constexpr int U = E * V <= 8 ? (BWD ? 2 : 4) : E * V <= 16 ? 2 : 1;  // rows whose loads are in flight together
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
    const int col = g * sh.cg + lane * V;
    for (long row0 = first / sh.G; row0 < sh.rows; row0 += U * step) {
        float v[U][E][V], d[BWD ? U : 1][E][V], mean[U], r[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const long row = row0 + u * step;
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const bool in = on[e] && row < sh.rows;
                if (in) {
                    load_floats<V>(x + row * ldx + col + P * e * V, v[u][e]);
                    if constexpr (BWD) load_floats<V>(dy + row * ldy + col + P * e * V, d[u][e]);
                } else {
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        v[u][e][i] = 0.f;
                        if constexpr (BWD) d[u][e][i] = 0.f;
                    }
                }
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float s = 0.f;
#pragma unroll
            for (int e = 0; e < E; ++e)
#pragma unroll
                for (int i = 0; i < V; ++i) s += v[u][e][i];
            mean[u] = s;
        }
        for (int k = 1; k < P; k <<= 1)
#pragma unroll
            for (int u = 0; u < U; ++u) mean[u] += __shfl_xor(mean[u], k, 64);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            mean[u] *= inv;
            float s = 0.f;
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float m = on[e] ? mean[u] : 0.f;
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    v[u][e][i] -= m;
                    s += v[u][e][i] * v[u][e][i];
                }
            }
            r[u] = s;
        }
        for (int k = 1; k < P; k <<= 1)
#pragma unroll
            for (int u = 0; u < U; ++u) r[u] += __shfl_xor(r[u], k, 64);
#pragma unroll
        for (int u = 0; u < U; ++u) r[u] = __builtin_amdgcn_rsqf(r[u] * inv + sh.eps);
        if constexpr (!BWD) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const long row = row0 + u * step;
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    if (!on[e] || row >= sh.rows) continue;
#pragma unroll
                    for (int i = 0; i < V; ++i) v[u][e][i] = v[u][e][i] * r[u] * wv[e][i] + bv[e][i];
                    act_values(sh.act, v[u][e]);
                    store_floats<V>(out + row * sh.C + col + P * e * V, v[u][e]);
                }
            }
        } else {
            float s1[U], s2[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                s1[u] = s2[u] = 0.f;
                if (row0 + u * step >= sh.rows) continue;
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    if (!on[e]) continue;
                    float z[V];
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        v[u][e][i] *= r[u];
                        z[i] = v[u][e][i] * wv[e][i] + bv[e][i];
                    }
                    act_slopes(sh.act, z);
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        const float xh = v[u][e][i], dz = d[u][e][i] * z[i];
                        aw[e][i] += dz * xh;
                        ab[e][i] += dz;
                        d[u][e][i] = dz * wv[e][i];
                        s1[u] += d[u][e][i];
                        s2[u] += d[u][e][i] * xh;
                    }
                }
            }
            for (int k = 1; k < P; k <<= 1)
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    s1[u] += __shfl_xor(s1[u], k, 64);
                    s2[u] += __shfl_xor(s2[u], k, 64);
                }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const long row = row0 + u * step;
                s1[u] *= inv;
                s2[u] *= inv;
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    if (!on[e] || row >= sh.rows) continue;
#pragma unroll
                    for (int i = 0; i < V; ++i) v[u][e][i] = r[u] * (d[u][e][i] - s1[u] - v[u][e][i] * s2[u]);
                    store_floats<V>(out + row * sh.C + col + P * e * V, v[u][e]);
                }
            }
        }
    }
    if constexpr (BWD) {
        if (per_block <= sh.G) {                             // the same for all
            const long slot = first / sh.G;                  // lane group of its group; those without a row are past the last slot
            if (slot < min(sh.rows, step)) {
                float* __restrict__ to = part + slot * 2 * sh.C + col;
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    if (!on[e]) continue;
                    store_floats<V>(to + P * e * V, aw[e]);
                    store_floats<V>(to + sh.C + P * e * V, ab[e]);
                }
            }
            return;
        }
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
// team: TEAM threads own a sample's GT groups (`tile` says which), TX = GT cg / V of them side by side along the
// columns, the others along the rows, E rows a thread in registers; rows beyond that are read again.
// stats: mean and r of every sample and group, written forward and read backward.
// Samples of more than `longest` rows are left to the split kernels.
// 8000 samples of 23 rows x 96 float32: 33 us forward, 53 backward (4.1 and 3.8 TB/s): a sample's loads, its three barriers and
// its stores follow one another, other blocks fill the gaps.
// ------------------------------------------------------------------------------------------
// Sum of squares about the mean from b = sum c^2, a = sum c and a / n; NaN and infinities stay visible.
__device__ __forceinline__ double variance(double b, double a, double m) { return fmax(b - a * m, 0.0) + (b - b); }

template <int TEAM> __device__ __forceinline__ void team_sync() {
    if constexpr (TEAM == 64) {
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    } else {
        __syncthreads();
    }
}

struct TeamPlan {
    int GT, tiles;               // groups of a tile, tiles of a sample
    long blocks;                 // blocks of a tile
    long longest;
};

template <class T, int V, int TEAM, int E, bool BWD>
__device__ __forceinline__ void norm_team(const NormShape& sh, const TeamPlan& tp, long block, int tile, const T* __restrict__ x,
                                          long ldx, const T* __restrict__ dy, long ldy, T* __restrict__ out,
                                          float* __restrict__ stats, float* __restrict__ part)
{
    constexpr int BLOCK = TEAM < 256 ? 256 : TEAM, TEAMS = BLOCK / TEAM;
    typedef typename std::conditional<BWD, float, double>::type Sum;
    __shared__ Sum red_mem[TEAMS][2][TEAM], tot_mem[TEAMS][2][TEAM];
    const int team = threadIdx.x / TEAM, t = threadIdx.x % TEAM, GT = tp.GT;
    Sum (&red)[2][TEAM] = red_mem[team];
    Sum (&tot)[2][TEAM] = tot_mem[team];
    const int cgv = sh.cg / V, TX = GT * cgv, TY = TEAM / TX;
    const int tx = t % TX, ty = t / TX;
    const int g0 = tile * GT, gn = min(GT, sh.G - g0);
    const bool on = ty < TY && tx < gn * cgv;
    const int col = g0 * sh.cg + tx * V, g = g0 + tx / cgv;

    // sums over a group's threads, for every thread of the group
    auto join = [&](Sum& a, Sum& b) {
        red[0][t] = on ? a : 0;
        red[1][t] = on ? b : 0;
        team_sync<TEAM>();
        if (t < TX) {
            Sum p = 0, q = 0;
            for (int k = 0; k < TY; ++k) { p += red[0][t + k * TX]; q += red[1][t + k * TX]; }
            red[0][t] = p;
            red[1][t] = q;
        }
        team_sync<TEAM>();
        if (t < GT) {
            Sum p = 0, q = 0;
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
    long s = block * TEAMS + team, next0 = 0, next1 = 0;
    if (s < sh.samples) sh.range(s, &next0, &next1);
    for (; s < sh.samples; s += tp.blocks * TEAMS) {
        const long r0 = next0, r1 = next1;
        if (s + tp.blocks * TEAMS < sh.samples) sh.range(s + tp.blocks * TEAMS, &next0, &next1);     // in flight beside the rows
        const int n = r1 - r0 > tp.longest ? 0 : (int)(r1 - r0);
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
            double a = 0.0, b = 0.0;
            float shift = 0.f;
            if (on) {
                float first[1];
                load_floats<1>(x + r0 * ldx + (long)g * sh.cg, first);
                shift = first[0];
                auto add = [&](const float (&u)[V]) {
#pragma unroll
                    for (int i = 0; i < V; ++i) { const double c = u[i] - shift; a += c; b = fma(c, c, b); }
                };
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (ty + TY * e < n) add(v[e]);
                for (int row = rest; row < n; row += TY) {
                    float u[V];
                    load_floats<V>(xp + (long)row * ldx, u);
                    add(u);
                }
            }
            join(a, b);
            double share = inv;                              // 1 / count in 32 bits, and a step of Newton's method
            share *= 2.0 - share * ((double)n * (double)sh.cg);
            const double m = a * share;
            const float mean = shift + (float)m;
            const float r = __builtin_amdgcn_rsqf((float)(variance(b, a, m) * share) + sh.eps);
            if (stats && on && ty == 0 && tx % cgv == 0) {
                stats[(s * sh.G + g) * 2] = mean;
                stats[(s * sh.G + g) * 2 + 1] = r;
            }
            if (on) {
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const int row = ty + TY * e;
                    if (row < n) {
#pragma unroll
                        for (int i = 0; i < V; ++i) v[e][i] = (v[e][i] - mean) * r * wv[i] + bv[i];
                        act_values(sh.act, v[e]);
                        store_floats<V>(op + (long)row * sh.C, v[e]);
                    }
                }
                for (int row = rest; row < n; row += TY) {
                    float u[V];
                    load_floats<V>(xp + (long)row * ldx, u);
#pragma unroll
                    for (int i = 0; i < V; ++i) u[i] = (u[i] - mean) * r * wv[i] + bv[i];
                    act_values(sh.act, u);
                    store_floats<V>(op + (long)row * sh.C, u);
                }
            }
        } else {
            float s1 = 0.f, s2 = 0.f, mean = 0.f, r = 0.f;
            auto step = [&](float (&u)[V], float (&dd)[V]) {     // x and dy become xh and e
                float z[V];
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    u[i] = (u[i] - mean) * r;
                    z[i] = u[i] * wv[i] + bv[i];
                }
                act_slopes(sh.act, z);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float xh = u[i], dz = dd[i] * z[i];
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
                    float z[V];
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        u[i] = (u[i] - mean) * r;
                        z[i] = u[i] * wv[i] + bv[i];
                    }
                    act_slopes(sh.act, z);
#pragma unroll
                    for (int i = 0; i < V; ++i) u[i] = r * (dd[i] * z[i] * wv[i] - m1 - u[i] * m2);
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
                part[block * 2 * sh.C + col + i] = p;
                part[block * 2 * sh.C + sh.C + col + i] = q;
            }
        }
    }
}

// ------------------------------------------------------------------------------------------
// split: chunks of `per` rows, one block each (and column tile).  Equal samples are cut one by one.  Ragged ones are cut
// together, every `per` rows: a chunk has parts of at most two samples of more than `longest` >= per rows, the one that its
// first row belongs to (slot 2 c) and the one that its last row belongs to (slot 2 c + 1); the others are the teams'.
// With per == 1 (groups too wide for a team) every sample is split, and a chunk has one slot.
// A column tile is whole groups, or a piece of one.
// 262144 x 256 float32 as one sample: statistics 64 us and y 88, sums backward 120 and dx 136 (4.2, 6.1, 4.5 and 5.9 TB/s; the
// second passes find the last chunks of the first in the caches), joining 11 and 8.
// ------------------------------------------------------------------------------------------
struct SplitPlan {
    int each, chunks;            // chunks of a sample of equal samples; chunks
    long slots;                  // parts of a group (piece): part[group or piece][slot], which a joining wave reads side by side
    long per, longest;           // rows of a chunk
    int gpt, pieces, tiles;      // groups of a tile, tiles of a group (one of the two is 1), tiles
    int TX;                      // accesses side by side in a tile
};

// the k-th V numbers of an array
template <int V, int N> __device__ __forceinline__ float (&part_of(float (&x)[N], int k))[V] {
    return *reinterpret_cast<float (*)[V]>(x + k * V);
}

struct Segment { long s, r0, r1, slot; };

// A chunk of ragged samples: its parts (s < 0: none).  The first pass finds them and the later ones read them.
struct ChunkEntry { Segment seg[2]; };

struct ColumnTile { int g0, gn, vec0, width; };              // groups; accesses

template <int V> __device__ __forceinline__ ColumnTile column_tile(const NormShape& sh, const SplitPlan& sp, int tile) {
    const int cgv = sh.cg / V;
    if (sp.pieces == 1) {
        const int g0 = tile * sp.gpt, gn = min(sp.gpt, sh.G - g0);
        return ColumnTile{g0, gn, g0 * cgv, gn * cgv};
    }
    const int g = tile / sp.pieces, from = tile % sp.pieces * sp.TX;
    return ColumnTile{g, 1, g * cgv + from, min(sp.TX, cgv - from)};
}

// Last sample that begins at `row` or before: a wave looks at 64 offsets at a time (8000 samples take 3 dependent loads,
// one offset at a time 13).  All lanes of the wave take part.
__device__ __forceinline__ long sample_of(const NormShape& sh, long row) {
    long lo = 0, hi = sh.samples - 1;
    const int lane = threadIdx.x & 63;
    while (lo < hi) {
        const long step = (hi - lo + 63) / 64, at = lo + (lane + 1) * step;
        const bool before = at <= hi && sh.offsets[at] <= row;
        lo += __popcll(__ballot(before)) * step;
        hi = min(lo + step - 1, hi);
    }
    return lo;
}

// The parts of a chunk that are to be computed
__device__ __forceinline__ void segments_of(const NormShape& sh, const SplitPlan& sp, int c, Segment (&out)[2], ChunkEntry* table,
                                            bool first_pass) {
    out[0].s = out[1].s = -1;
    if (!sh.offsets) {
        const int s = c / sp.each;
        const long r0 = s * sh.length + (long)(c % sp.each) * sp.per;
        out[0] = Segment{s, r0, min(r0 + sp.per, (s + 1) * sh.length), c};
        return;
    }
    if (!first_pass) {
        out[0] = table[c].seg[0];
        out[1] = table[c].seg[1];
        return;
    }
    const long a = c * sp.per, e = min(a + sp.per, sh.rows);
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        if (q && sp.per == 1) break;
        const long s = sample_of(sh, q ? e - 1 : a);
        long r0, r1;
        sh.range(s, &r0, &r1);
        if (r1 - r0 > sp.longest && r0 < e && r1 > a && (q ? s != out[0].s : r0 <= a))
            out[q] = Segment{s, max(r0, a), min(r1, e), sp.per == 1 ? (long)c : 2L * c + q};
    }
    if (threadIdx.x == 0) {                                  // by all column tiles alike
        table[c].seg[0] = out[0];
        table[c].seg[1] = out[1];
    }
}

// A sample's parts, in order: slot and rows of the k-th
struct Parts {
    int first, n;                // first chunk, chunks
    long r0, r1, per;
    bool ragged, late;           // late: begins inside its first chunk

    __device__ long slot(int k) const { return !ragged || per == 1 ? first + k : 2L * (first + k) + (k == 0 && late ? 1 : 0); }
    __device__ long rows(int k) const {
        if (!ragged) return min(per, r1 - r0 - k * per);
        const long a = (first + k) * per;
        return min(r1, a + per) - max(r0, a);
    }
};

// The sample that block k of the joining kernels is to join, if any: equal samples by number, a ragged one by the chunk
// in which it begins (two may begin in one chunk only where the first is no long one).
__device__ __forceinline__ bool sample_to_join(const NormShape& sh, const SplitPlan& sp, int k, const ChunkEntry* table, long* s,
                                               Parts* p) {
    if (!sh.offsets) {
        *s = k;
        *p = Parts{k * sp.each, sp.each, k * sh.length, (k + 1) * sh.length, sp.per, false, false};
        return true;
    }
    const long a = k * sp.per;
    for (int q = 0; q < 2; ++q) {
        *s = table[k].seg[q].s;
        if (*s < 0) continue;
        long r0, r1;
        sh.range(*s, &r0, &r1);
        if (r0 < a) continue;
        *p = Parts{k, (int)((r1 - 1) / sp.per) - k + 1, r0, r1, sp.per, true, r0 > a};
        return true;
    }
    return false;
}

// Sums of two numbers over the threads of a block that share a group (gn == 1: over all), left in red[.][group]
template <class Sum>
__device__ __forceinline__ void join_groups(Sum (&red)[2][kNormBlock], Sum a, Sum b, int TX, int TY, int cgv, int gn) {
    const int t = threadIdx.x;
    __syncthreads();
    red[0][t] = a;
    red[1][t] = b;
    __syncthreads();
    if (t < TX) {
        for (int k = 1; k < TY; ++k) { a += red[0][t + k * TX]; b += red[1][t + k * TX]; }
        red[0][t] = a;
        red[1][t] = b;
    }
    __syncthreads();
    const int width = gn == 1 ? TX : cgv;
    if (gn == 1 && t < 64) {                                 // up to 256 numbers: a wave
        a = b = 0;
        for (int k = t; k < width; k += 64) { a += red[0][k]; b += red[1][k]; }
        a = wave_sum(a, 64);
        b = wave_sum(b, 64);
    } else if (gn > 1 && t < gn) {
        a = b = 0;
        for (int k = 0; k < width; ++k) { a += red[0][t * width + k]; b += red[1][t * width + k]; }
    }
    __syncthreads();
    if (t < gn) {
        red[0][t] = a;
        red[1][t] = b;
    }
}

// Mean and sum of squares about it of a chunk's groups: part[tile's group or piece][slot]
template <class T, int V>
__device__ __forceinline__ void norm_stats(const NormShape& sh, const SplitPlan& sp, int chunk, int tile, const T* __restrict__ x,
                                           long ldx, ChunkEntry* __restrict__ table, float2* __restrict__ part)
{
    __shared__ double red[2][kNormBlock];
    Segment seg[2];
    segments_of(sh, sp, chunk, seg, table, true);
    const ColumnTile ct = column_tile<V>(sh, sp, tile);
    const int TX = sp.TX, TY = kNormBlock / TX, t = threadIdx.x, tx = t % TX, ty = t / TX, cgv = sh.cg / V;
    const bool on = ty < TY && tx < ct.width;
    const int vec = ct.vec0 + tx;
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        if (seg[q].s < 0) continue;
        const long r0 = seg[q].r0, r1 = seg[q].r1;
        double a = 0.0, b = 0.0;
        float shift = 0.f;
        if (on) {
            const T* __restrict__ xp = x + (long)vec * V;
            const int from = ct.gn == 1 ? ct.vec0 : vec / cgv * cgv;
            float one[1];
            load_floats<1>(x + r0 * ldx + (long)from * V, one);
            shift = one[0];
            auto add = [&](const float (&u)[V]) {
#pragma unroll
                for (int i = 0; i < V; ++i) { const double c = u[i] - shift; a += c; b = fma(c, c, b); }
            };
            constexpr int U = 8;
            long row = r0 + ty;
            for (; row + (U - 1) * TY < r1; row += U * TY) {
                float m[U][V];
#pragma unroll
                for (int k = 0; k < U; ++k) load_floats<V>(xp + (row + k * TY) * ldx, m[k]);
#pragma unroll
                for (int k = 0; k < U; ++k) add(m[k]);
            }
            for (; row < r1; row += TY) {
                float u[V];
                load_floats<V>(xp + row * ldx, u);
                add(u);
            }
        }
        // every group's first number, for its thread
        const int width = ct.gn == 1 ? ct.width : cgv;
        join_groups(red, a, b, TX, TY, cgv, ct.gn);
        if (t < ct.gn) {
            float one[1];
            load_floats<1>(x + r0 * ldx + ((long)ct.vec0 + (long)t * cgv) * V, one);
            const double m = red[0][t] / ((double)(r1 - r0) * (double)(width * V));
            const long at = sp.pieces == 1 ? ct.g0 + t : tile;
            part[at * sp.slots + seg[q].slot] = make_float2(one[0] + (float)m, (float)variance(red[1][t], red[0][t], m));
        }
    }
}

constexpr int kJoinBlock = 1024, kJoinGroups = kJoinBlock / 64;

// f(part, piece, chunk) for a wave's share of the parts of a sample and group, U of them on their way at once
template <class F>
__device__ __forceinline__ void for_parts(const NormShape& sh, const SplitPlan& sp, const Parts& p, int g,
                                          const float2* __restrict__ part, F&& f) {
    constexpr int U = 8;
    for (int piece = 0; piece < sp.pieces; ++piece) {
        const float2* __restrict__ from = part + ((long)g * sp.pieces + piece) * sp.slots;
        for (int c = threadIdx.x & 63; c < p.n; c += U * 64) {
            float2 v[U];
#pragma unroll
            for (int u = 0; u < U; ++u) v[u] = from[p.slot(min(c + u * 64, p.n - 1))];
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (c + u * 64 < p.n) f(v[u], piece, c + u * 64);
        }
    }
}

// Joins the parts of a sample and group by the formula for the variance of a union; a wave owns a group
template <int V>
__global__ __launch_bounds__(kJoinBlock) void norm_join_kernel(NormShape sh, SplitPlan sp, int from, const ChunkEntry* __restrict__ table,
                                                               const float2* __restrict__ part, float* __restrict__ stats)
{
    long s;
    Parts p;
    if (!sample_to_join(sh, sp, from + blockIdx.x, table, &s, &p)) return;
    const int g = blockIdx.y * kJoinGroups + (threadIdx.x >> 6), lane = threadIdx.x & 63, pieces = sp.pieces, cgv = sh.cg / V;
    if (g >= sh.G) return;
    const double total = (double)(p.r1 - p.r0) * (double)sh.cg;
    double a = 0.0, b = 0.0;
    // relative to the first part's mean, which may be that of a single row
    const float origin = part[(long)g * pieces * sp.slots + p.slot(0)].x;
    for_parts(sh, sp, p, g, part, [&](float2 v, int piece, int c) {
        const int width = pieces == 1 ? cgv : min(sp.TX, cgv - piece * sp.TX);
        const double d = (double)v.x - origin, n = (double)p.rows(c) * (double)(width * V);
        a += d * n;
        b += v.y + d * d * n;
    });
    a = wave_sum(a, 64);
    b = wave_sum(b, 64);
    if (lane == 0) {
        const double m = a / total;
        stats[(s * sh.G + g) * 2] = origin + (float)m;
        stats[(s * sh.G + g) * 2 + 1] = 1.f / sqrtf((float)(variance(b, a, m) / total) + sh.eps);
    }
}

// y of a chunk; BWD: dx, with the means of e and e xh of every sample and group in `means`.  The last chunks first: they
// are the ones that the pass before has left in the caches.
template <class T, int V, bool BWD>
__global__ __launch_bounds__(kNormBlock) void norm_apply_kernel(NormShape sh, SplitPlan sp, int last, const T* __restrict__ x, long ldx,
                                                                const T* __restrict__ dy, long ldy,
                                                                const float* __restrict__ stats,
                                                                const float* __restrict__ means, ChunkEntry* __restrict__ table,
                                                                T* __restrict__ out)
{
    Segment seg[2];
    segments_of(sh, sp, last - blockIdx.x, seg, table, false);
    const ColumnTile ct = column_tile<V>(sh, sp, blockIdx.y);
    const int TX = sp.TX, TY = kNormBlock / TX, tx = threadIdx.x % TX, ty = threadIdx.x / TX;
    if ((seg[0].s < 0 && seg[1].s < 0) || ty >= TY || tx >= ct.width) return;
    const int col = (ct.vec0 + tx) * V, g = col / sh.cg;
    float wv[V], bv[V];
    sh.params<V>(col, wv, bv);
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        if (seg[q].s < 0) continue;
        const long s = seg[q].s, r0 = seg[q].r0, r1 = seg[q].r1;
        const float mean = stats[(s * sh.G + g) * 2], r = stats[(s * sh.G + g) * 2 + 1];
        float m1 = 0.f, m2 = 0.f;
        if constexpr (BWD) {
            m1 = means[(s * sh.G + g) * 2];
            m2 = means[(s * sh.G + g) * 2 + 1];
        }
        auto put = [&](auto& u, auto& d) {                   // several rows' numbers, V to a row
            constexpr int N = sizeof(u) / sizeof(float);
            float z[N];
#pragma unroll
            for (int i = 0; i < N; ++i) {
                u[i] = (u[i] - mean) * r;
                z[i] = u[i] * wv[i % V] + bv[i % V];
            }
            if constexpr (!BWD) {
                act_values(sh.act, z);
#pragma unroll
                for (int i = 0; i < N; ++i) u[i] = z[i];
            } else {
                act_slopes(sh.act, z);
#pragma unroll
                for (int i = 0; i < N; ++i) u[i] = r * (d[i] * z[i] * wv[i % V] - m1 - u[i] * m2);
            }
        };
        constexpr int U = 4;
        long row = r0 + ty;
        for (; row + (U - 1) * TY < r1; row += U * TY) {
            float u[U * V], d[U * V];
#pragma unroll
            for (int k = 0; k < U; ++k) {
                load_floats<V>(x + (row + k * TY) * ldx + col, part_of<V>(u, k));
                if constexpr (BWD) load_floats<V>(dy + (row + k * TY) * ldy + col, part_of<V>(d, k));
            }
            put(u, d);
#pragma unroll
            for (int k = 0; k < U; ++k) store_floats<V>(out + (row + k * TY) * sh.C + col, part_of<V>(u, k));
        }
        for (; row < r1; row += TY) {
            float u[V], d[V];
            load_floats<V>(x + row * ldx + col, u);
            if constexpr (BWD) load_floats<V>(dy + row * ldy + col, d);
            put(u, d);
            store_floats<V>(out + row * sh.C + col, u);
        }
    }
}

// Of a chunk: sums of dz xh and of dz over its columns (cols), which dw and db are made of, and of e and e xh over its
// groups (part).  Slots that no sample has are cleared.
template <class T, int V>
__device__ __forceinline__ void norm_grad_stats(const NormShape& sh, const SplitPlan& sp, int chunk, int tile,
                                                const T* __restrict__ x, long ldx, const T* __restrict__ dy, long ldy,
                                                const float* __restrict__ stats, ChunkEntry* __restrict__ table,
                                                float2* __restrict__ part, float* __restrict__ cols)
{
    __shared__ float red[2][kNormBlock];
    Segment seg[2];
    segments_of(sh, sp, chunk, seg, table, true);
    const ColumnTile ct = column_tile<V>(sh, sp, tile);
    const int TX = sp.TX, TY = kNormBlock / TX, t = threadIdx.x, tx = t % TX, ty = t / TX, cgv = sh.cg / V;
    const bool on = ty < TY && tx < ct.width;
    const int col = (ct.vec0 + tx) * V;
    float aw[V] = {}, ab[V] = {}, wv[V], bv[V];
    const bool some = seg[0].s >= 0 || seg[1].s >= 0;
    if (on && some) sh.params<V>(col, wv, bv);
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        if (seg[q].s < 0) continue;
        float s1 = 0.f, s2 = 0.f;
        if (on) {
            const long r0 = seg[q].r0, r1 = seg[q].r1;
            const int g = col / sh.cg;
            const float mean = stats[(seg[q].s * sh.G + g) * 2], r = stats[(seg[q].s * sh.G + g) * 2 + 1];
            auto add = [&](auto& u, auto& d) {
                constexpr int N = sizeof(u) / sizeof(float);
                float z[N];
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    u[i] = (u[i] - mean) * r;
                    z[i] = u[i] * wv[i % V] + bv[i % V];
                }
                act_slopes(sh.act, z);
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const float dz = d[i] * z[i], e = dz * wv[i % V];
                    aw[i % V] += dz * u[i];
                    ab[i % V] += dz;
                    s1 += e;
                    s2 += e * u[i];
                }
            };
            constexpr int U = 4;
            long row = r0 + ty;
            for (; row + (U - 1) * TY < r1; row += U * TY) {
                float u[U * V], d[U * V];
#pragma unroll
                for (int k = 0; k < U; ++k) {
                    load_floats<V>(x + (row + k * TY) * ldx + col, part_of<V>(u, k));
                    load_floats<V>(dy + (row + k * TY) * ldy + col, part_of<V>(d, k));
                }
                add(u, d);
            }
            for (; row < r1; row += TY) {
                float u[V], d[V];
                load_floats<V>(x + row * ldx + col, u);
                load_floats<V>(dy + row * ldy + col, d);
                add(u, d);
            }
        }
        join_groups(red, s1, s2, TX, TY, cgv, ct.gn);
        if (t < ct.gn) {
            const long at = sp.pieces == 1 ? ct.g0 + t : tile;
            part[at * sp.slots + seg[q].slot] = make_float2(red[0][t], red[1][t]);
        }
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
        float p = aw[i], q = ab[i];
        if (some) {                                          // the same for all threads
            __syncthreads();
            red[0][t] = on ? p : 0.f;
            red[1][t] = on ? q : 0.f;
            __syncthreads();
            if (t < ct.width)
                for (int k = 1; k < TY; ++k) { p += red[0][t + k * TX]; q += red[1][t + k * TX]; }
        }
        if (t < ct.width) {
            cols[(long)chunk * 2 * sh.C + col + i] = p;
            cols[(long)chunk * 2 * sh.C + sh.C + col + i] = q;
        }
    }
}

// First pass: teams in the first blocks of a launch, chunks in the others.  Ragged samples may be of both kinds and only
// the device knows, so both are one launch then (TEAM threads and chunks): an empty one would take as long as a small
// sample.  Equal samples are all of one kind; their launches hold registers for that kind only.
template <class T, int V, int TEAM, int E, bool CHUNKS, bool BWD>
__global__ __launch_bounds__(TEAM < 256 ? 256 : TEAM) void norm_first_kernel(
    NormShape sh, TeamPlan tp, SplitPlan sp, int from, const T* __restrict__ x, long ldx, const T* __restrict__ dy, long ldy,
    T* __restrict__ out, float* __restrict__ stats, float* __restrict__ team_cols, ChunkEntry* __restrict__ table,
    float2* __restrict__ part, float* __restrict__ cols)
{
    const unsigned teams = (unsigned)tp.blocks * tp.tiles;
    if (E > 0 && (!CHUNKS || blockIdx.x < teams)) {
        if constexpr (E > 0)
            norm_team<T, V, TEAM, E, BWD>(sh, tp, blockIdx.x / tp.tiles, blockIdx.x % tp.tiles, x, ldx, dy, ldy, out, stats, team_cols);
    } else if constexpr (CHUNKS) {
        const unsigned k = blockIdx.x - teams, chunk = from + k / sp.tiles, tile = k % sp.tiles;
        if constexpr (BWD) norm_grad_stats<T, V>(sh, sp, chunk, tile, x, ldx, dy, ldy, stats, table, part, cols);
        else norm_stats<T, V>(sh, sp, chunk, tile, x, ldx, table, part);
    }
}

// Second pass backward: the means of e and e xh of every split sample and group (first `joins` blocks, kJoinGroups groups
// to a block, from the from-th on), and dw, db from `rows` rows of 2 C sums, 16 columns to a block.
__global__ __launch_bounds__(kJoinBlock) void norm_grad_join_kernel(NormShape sh, SplitPlan sp, int from, int joins,
                                                                    const ChunkEntry* __restrict__ table, const float2* __restrict__ part, float* __restrict__ means,
                                                                    const float* __restrict__ cols, long rows, void* dw, void* db)
{
    __shared__ float red[kJoinBlock];
    const int t = threadIdx.x;
    if (blockIdx.x < joins) {
        const int blocks = (sh.G + kJoinGroups - 1) / kJoinGroups;
        long s;
        Parts p;
        if (!sample_to_join(sh, sp, from + blockIdx.x / blocks, table, &s, &p)) return;
        const int g = (int)(blockIdx.x % blocks) * kJoinGroups + (t >> 6);
        if (g >= sh.G) return;
        float a = 0.f, b = 0.f;
        for_parts(sh, sp, p, g, part, [&](float2 v, int, int) {
            a += v.x;
            b += v.y;
        });
        a = wave_sum(a, 64);
        b = wave_sum(b, 64);
        if ((t & 63) == 0) {
            const float total = (float)(p.r1 - p.r0) * (float)sh.cg;
            means[(s * sh.G + g) * 2] = a / total;
            means[(s * sh.G + g) * 2 + 1] = b / total;
        }
        return;
    }
    const int c = (int)(blockIdx.x - joins) * 16 + (t & 15);
    float s = 0.f;
    if (c < 2 * sh.C) {
        constexpr int U = 8;
        float a[U] = {};
        long k = t >> 4;
        for (; k + (U - 1) * 64 < rows; k += U * 64)
#pragma unroll
            for (int u = 0; u < U; ++u) a[u] += cols[(k + u * 64) * 2 * sh.C + c];
        for (; k < rows; k += 64) a[0] += cols[k * 2 * sh.C + c];
#pragma unroll
        for (int u = 0; u < U; ++u) s += a[u];
    }
    red[t] = s;
    for (int d = kJoinBlock / 2; d >= 16; d >>= 1) {
        __syncthreads();
        if (t < d) red[t] += red[t + d];
    }
    if (t < 16 && c < 2 * sh.C) {
        if (c < sh.C) { if (dw) store_param(dw, sh.param_dtype, c, red[t]); }
        else if (db) store_param(db, sh.param_dtype, c - sh.C, red[t]);
    }
}

}  // namespace daspmm
