// Root-mean-square norm of rows with the residual's addition, forward (also with a result in e4m3) and backward.
//   s = x + residual,  r = 1 / sqrt(mean(s^2) + eps),  y = w s r
//   e = dy w,  dx = r (e - s r mean(e s r)) + dsum,  dw = sum over rows of dy s r
//
// Memory bounds it: a row is read once and waits in the registers of a team (lanes of a wave, or a block) while its sums
// are joined.  r is not kept for the backward pass, which has the row in registers anyway.  A team's lanes hold their columns
// of dw over all of its rows; the teams' parts are added in one order.  262144 x 128 float32 with a residual: 104 us forward and 111
// backward, 5.1 and 4.8 TB/s (a large copy 5.2); 8192 x 4096 bf16: 56 and 59, 4.8 and 4.5.
#include "da_training.h"

#include "da_gated_plan.h"
#include "da_internal.h"
#include "da_layer_common.h"
#include "da_spmm.h"

#include <algorithm>

namespace daspmm {
namespace {

constexpr int kRmsBlock = 256, kRmsMost = 1024, kRmsHeld = 16;       // threads; numbers of a row in a lane

template <class T> struct RmsArgs {
    const T *x, *res, *dy, *dsum;            // x: s backward
    long ldx, ldr, ldy, ldd;
    const void* w;
    int w_type;
    long rows;
    int C;
    float eps;
    T *sum, *y;                              // y: dx backward
    uint32_t* q;
    float *scale, *part;
};

// V numbers of a row from column c on, `left` of them there; the others 0
template <int V, class T> __device__ __forceinline__ void load_some(const T* __restrict__ p, int left, float (&v)[V]) {
    if (left >= V) {
        load_floats<V>(p, v);
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = 0.f;
#pragma unroll
        for (int i = 0; i + 1 < V; ++i)
            if (i < left) {
                float one[1];
                load_floats<1>(p + i, one);
                v[i] = one[0];
            }
    }
}
template <int V, class T> __device__ __forceinline__ void store_some(T* __restrict__ p, int left, const float (&v)[V]) {
    if (left >= V) {
        store_floats<V>(p, v);
    } else {
#pragma unroll
        for (int i = 0; i + 1 < V; ++i)
            if (i < left) {
                const float one[1] = {v[i]};
                store_floats<1>(p + i, one);
            }
    }
}
template <int V> __device__ __forceinline__ void load_weights(const void* w, int type, int c, int left, float (&v)[V]) {
    if (!w) {
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = 1.f;
    } else if (type == DA_F32) {
        load_some<V>(static_cast<const float*>(w) + c, left, v);
    } else {
        load_some<V>(static_cast<const bf16*>(w) + c, left, v);
    }
}

// The larger of two magnitudes; NaN wins
__device__ __forceinline__ float larger(float a, float b) { return b > a || b != b ? b : a; }

// COUNT numbers of all lanes of a team joined by f: P lanes of a wave, or a block of `waves` waves
template <int COUNT, class F>
__device__ __forceinline__ void team_join(float (&x)[COUNT], int P, int waves, float (*lds)[kRmsMost / 64], F&& f) {
    for (int d = 1; d < P && d < 64; d <<= 1)
#pragma unroll
        for (int i = 0; i < COUNT; ++i) x[i] = f(x[i], __shfl_xor(x[i], d, 64));
    if (waves > 1) {
        __syncthreads();                     // the numbers of the row before have been read
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int i = 0; i < COUNT; ++i) lds[i][threadIdx.x >> 6] = x[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < COUNT; ++i) {
            x[i] = lds[i][0];
            for (int k = 1; k < waves; ++k) x[i] = f(x[i], lds[i][k]);
        }
    }
}
__device__ __forceinline__ float add(float a, float b) { return a + b; }

// Squares of numbers this large or small are no floats any more: the row is taken times 2^-76 or 2^60 then (1 otherwise).  2^20 squares of
// numbers below 2^(128 - 76) are below 2^124, and the largest of a row whose squares come to 1e38 is 2^53 at least.
__device__ __forceinline__ float other_scale(float sum, float inv, float eps) {
    if (!(sum < 1e38f)) return 0x1p-76f;
    return sum * inv + eps < 1e-24f && sum > 0.f || (sum == 0.f && eps < 1e-24f) ? 0x1p60f : 1.f;
}

// Rounded to the nearest number of e4m3, ties to even; |x| <= 448 but for a scale that lost digits below 2^-126
__device__ __forceinline__ float in_e4m3(float x) { return x > 448.f ? 448.f : x < -448.f ? -448.f : x; }
template <int V> __device__ __forceinline__ void store_e4m3(uint8_t* p, int left, const float (&x)[V]) {
    uint32_t word[V / 4];
#pragma unroll
    for (int i = 0; i < V / 4; ++i) {
        int k = __builtin_amdgcn_cvt_pk_fp8_f32(in_e4m3(x[4 * i]), in_e4m3(x[4 * i + 1]), 0, false);
        word[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(in_e4m3(x[4 * i + 2]), in_e4m3(x[4 * i + 3]), k, true);
    }
    if (left >= V) {
        typedef typename Pack<uint8_t, V>::type Bytes;
        Bytes b;
        __builtin_memcpy(&b, word, V);
        *reinterpret_cast<Bytes*>(p) = b;
    } else {
#pragma unroll
        for (int i = 0; i + 1 < V; ++i)
            if (i < left) p[i] = (uint8_t)(word[i / 4] >> (i % 4 * 8));
    }
}

// A team of P lanes goes from row to row; a lane has E pieces of V columns, P pieces apart.  E == 0: a row of any length
// is read again instead of held.
template <class T, int V, int E, bool EIGHT>
__global__ __launch_bounds__(kRmsMost) void rms_kernel(RmsArgs<T> a, int P)
{
    __shared__ float lds[1][kRmsMost / 64];
    const int waves = P > 64 ? P / 64 : 1, lane = threadIdx.x & (P - 1), teams = blockDim.x / P;
    constexpr int N = E ? E : 1;
    const float inv = a.C ? 1.f / (float)a.C : 0.f;
    float w[N][V];
    if constexpr (E > 0)
#pragma unroll
        for (int e = 0; e < E; ++e) load_weights<V>(a.w, a.w_type, (lane + e * P) * V, a.C - (lane + e * P) * V, w[e]);
    for (long row = (long)blockIdx.x * teams + threadIdx.x / P; row < a.rows; row += (long)gridDim.x * teams) {
        const T* __restrict__ x = a.x + row * a.ldx;
        const T* __restrict__ res = a.res ? a.res + row * a.ldr : nullptr;
        T* __restrict__ sum = a.res ? a.sum + row * a.C : nullptr;
        auto get = [&](int c, float (&v)[V]) {               // s of columns c and on
            const int left = a.C - c;
            load_some<V>(x + c, left, v);
            if (res) {
                float u[V];
                load_some<V>(res + c, left, u);
#pragma unroll
                for (int i = 0; i < V; ++i) v[i] += u[i];
                if constexpr (sizeof(T) == 2)
#pragma unroll
                    for (int i = 0; i < V; ++i) v[i] = (float)(bf16)v[i];
            }
        };
        float v[N][V], ss[1] = {0.f}, k = 1.f;
        auto count = [&](float (&p)[V]) {
#pragma unroll
            for (int i = 0; i < V; ++i) ss[0] += p[i] * p[i];
        };
        // E == 0: the row again, as this thread wrote it where there is a residual
        auto again = [&](int c, float (&p)[V]) {
            load_some<V>((res ? (const T*)sum : x) + c, a.C - c, p);
#pragma unroll
            for (int i = 0; i < V; ++i) p[i] *= k;
        };
        if constexpr (E > 0) {
#pragma unroll
            for (int e = 0; e < E; ++e) get((lane + e * P) * V, v[e]);
#pragma unroll
            for (int e = 0; e < E; ++e) count(v[e]);
            if (res)
#pragma unroll
                for (int e = 0; e < E; ++e) store_some<V>(sum + (lane + e * P) * V, a.C - (lane + e * P) * V, v[e]);
        } else {
            for (int c = lane * V; c < a.C; c += P * V) {
                get(c, v[0]);
                count(v[0]);
                if (res) store_some<V>(sum + c, a.C - c, v[0]);
            }
        }
        team_join<1>(ss, P, waves, lds, add);
        k = other_scale(ss[0], inv, a.eps);
        if (k != 1.f) {
            ss[0] = 0.f;
            if constexpr (E > 0) {
#pragma unroll
                for (int e = 0; e < E; ++e) {
#pragma unroll
                    for (int i = 0; i < V; ++i) v[e][i] *= k;
                    count(v[e]);
                }
            } else {
                for (int c = lane * V; c < a.C; c += P * V) {
                    again(c, v[0]);
                    count(v[0]);
                }
            }
            team_join<1>(ss, P, waves, lds, add);
        }
        const float r = 1.f / sqrtf(ss[0] * inv + a.eps * k * k);
        auto scaled = [&](float (&p)[V], float (&u)[V]) {                    // y
#pragma unroll
            for (int i = 0; i < V; ++i) p[i] = p[i] * r * u[i];
        };
        auto result = [&](int c) {                           // E == 0
            again(c, v[0]);
            load_weights<V>(a.w, a.w_type, c, a.C - c, w[0]);
            scaled(v[0], w[0]);
        };
        if constexpr (!EIGHT) {
            T* __restrict__ y = a.y + row * a.C;
            if constexpr (E > 0) {
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    scaled(v[e], w[e]);
                    store_some<V>(y + (lane + e * P) * V, a.C - (lane + e * P) * V, v[e]);
                }
            } else {
                for (int c = lane * V; c < a.C; c += P * V) {
                    result(c);
                    store_some<V>(y + c, a.C - c, v[0]);
                }
            }
        } else {
            uint8_t* __restrict__ q = reinterpret_cast<uint8_t*>(a.q) + row * a.C;
            float most[1] = {0.f};
            if constexpr (E > 0) {
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    scaled(v[e], w[e]);
#pragma unroll
                    for (int i = 0; i < V; ++i) most[0] = larger(most[0], fabsf(v[e][i]));
                }
            } else {
                for (int c = lane * V; c < a.C; c += P * V) {
                    result(c);
#pragma unroll
                    for (int i = 0; i < V; ++i) most[0] = larger(most[0], fabsf(v[0][i]));
                }
            }
            team_join<1>(most, P, waves, lds, larger);
            const float scale = most[0] / 448.f, by = scale > 0.f ? scale : 1.f;
            if (lane == 0) a.scale[row] = scale;
            if constexpr (E > 0) {
#pragma unroll
                for (int e = 0; e < E; ++e) {
#pragma unroll
                    for (int i = 0; i < V; ++i) v[e][i] /= by;
                    store_e4m3<V>(q + (lane + e * P) * V, a.C - (lane + e * P) * V, v[e]);
                }
            } else {
                for (int c = lane * V; c < a.C; c += P * V) {
                    result(c);
#pragma unroll
                    for (int i = 0; i < V; ++i) v[0][i] /= by;
                    store_e4m3<V>(q + c, a.C - c, v[0]);
                }
            }
        }
    }
}

// a.part: a row of C numbers for every block, its part of dw
template <class T, int V, int E>
__global__ __launch_bounds__(kRmsMost) void rms_grad_kernel(RmsArgs<T> a, int P)
{
    __shared__ float lds[2][kRmsMost / 64];
    extern __shared__ float columns[];       // teams of less than a wave to a block: [threads][E V], their parts of dw
    const int waves = P > 64 ? P / 64 : 1, lane = threadIdx.x & (P - 1), teams = blockDim.x / P;
    constexpr int N = E ? E : 1;
    const float inv = a.C ? 1.f / (float)a.C : 0.f;
    float w[N][V], dw[N][V];
    float* __restrict__ mine = a.part ? a.part + (long)blockIdx.x * a.C : nullptr;
    if constexpr (E > 0)
#pragma unroll
        for (int e = 0; e < E; ++e) {
            load_weights<V>(a.w, a.w_type, (lane + e * P) * V, a.C - (lane + e * P) * V, w[e]);
#pragma unroll
            for (int i = 0; i < V; ++i) dw[e][i] = 0.f;
        }
    bool first = true;
    for (long row = (long)blockIdx.x * teams + threadIdx.x / P; row < a.rows; row += (long)gridDim.x * teams) {
        const T* __restrict__ s = a.x + row * a.ldx;
        const T* __restrict__ dy = a.dy ? a.dy + row * a.ldy : nullptr;
        const T* __restrict__ more = a.dsum ? a.dsum + row * a.ldd : nullptr;
        T* __restrict__ dx = a.y ? a.y + row * a.C : nullptr;
        auto get = [&](const T* p, int c, float (&v)[V]) {
            if (p) load_some<V>(p + c, a.C - c, v);
            else
#pragma unroll
                for (int i = 0; i < V; ++i) v[i] = 0.f;
        };
        float v[N][V], g[N][V], d[N][V], sums[2] = {0.f, 0.f}, k = 1.f;
        auto count = [&](float (&p)[V], const float (&u)[V], const float (&f)[V]) {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                sums[0] += p[i] * p[i];
                sums[1] += p[i] * (u[i] * f[i]);
            }
        };
        auto scaled = [&](float (&p)[V]) {
#pragma unroll
            for (int i = 0; i < V; ++i) p[i] *= k;
        };
        auto walk = [&] {                                    // E == 0
            for (int c = lane * V; c < a.C; c += P * V) {
                get(s, c, v[0]);
                get(dy, c, g[0]);
                load_weights<V>(a.w, a.w_type, c, a.C - c, w[0]);
                scaled(v[0]);
                count(v[0], g[0], w[0]);
            }
        };
        if constexpr (E > 0) {
#pragma unroll
            for (int e = 0; e < E; ++e) {
                get(s, (lane + e * P) * V, v[e]);
                get(dy, (lane + e * P) * V, g[e]);
                get(more, (lane + e * P) * V, d[e]);
            }
#pragma unroll
            for (int e = 0; e < E; ++e) count(v[e], g[e], w[e]);
        } else {
            walk();
        }
        team_join<2>(sums, P, waves, lds, add);
        k = other_scale(sums[0], inv, a.eps);
        if (k != 1.f) {
            sums[0] = sums[1] = 0.f;
            if constexpr (E > 0) {
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    scaled(v[e]);
                    count(v[e], g[e], w[e]);
                }
            } else {
                walk();
            }
            team_join<2>(sums, P, waves, lds, add);
        }
        const float r = 1.f / sqrtf(sums[0] * inv + a.eps * k * k), m = sums[1] * r * inv, rk = r * k;
        auto finish = [&](int c, float (&p)[V], float (&u)[V], float (&f)[V], float (&plus)[V], float (&t)[V]) {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float xh = p[i] * r;
                p[i] = rk * (u[i] * f[i] - xh * m) + plus[i];
                t[i] += u[i] * xh;
            }
            if (dx) store_some<V>(dx + c, a.C - c, p);
        };
        if constexpr (E > 0) {
#pragma unroll
            for (int e = 0; e < E; ++e) finish((lane + e * P) * V, v[e], g[e], w[e], d[e], dw[e]);
        } else {
            for (int c = lane * V; c < a.C; c += P * V) {
                get(s, c, v[0]);
                get(dy, c, g[0]);
                get(more, c, d[0]);
                load_weights<V>(a.w, a.w_type, c, a.C - c, w[0]);
                scaled(v[0]);
                if (first || !mine)
#pragma unroll
                    for (int i = 0; i < V; ++i) dw[0][i] = 0.f;
                else load_some<V>(mine + c, a.C - c, dw[0]);
                finish(c, v[0], g[0], w[0], d[0], dw[0]);
                if (mine) store_some<V>(mine + c, a.C - c, dw[0]);
            }
            first = false;
        }
    }
    if constexpr (E > 0) {
        if (!mine) return;
        if (teams == 1) {
#pragma unroll
            for (int e = 0; e < E; ++e) store_some<V>(mine + (lane + e * P) * V, a.C - (lane + e * P) * V, dw[e]);
            return;
        }
#pragma unroll
        for (int e = 0; e < E; ++e)
#pragma unroll
            for (int i = 0; i < V; ++i) columns[(threadIdx.x / P * E + e) * P * V + lane * V + i] = dw[e][i];
        __syncthreads();
        for (int c = threadIdx.x; c < a.C; c += blockDim.x) {
            float t = 0.f;
            for (int k = 0; k < teams; ++k) t += columns[k * E * P * V + c];
            mine[c] = t;
        }
    }
}

// dw from `count` parts: 16 columns and 16 parts at once to a block
__global__ __launch_bounds__(256) void rms_join_kernel(const float* __restrict__ part, long count, int C, void* dw, int type)
{
    __shared__ float red[16][17];
    const int c = blockIdx.x * 16 + (threadIdx.x & 15), k0 = threadIdx.x >> 4;
    constexpr int U = 4;
    float s[U] = {};
    if (c < C) {
        long k = k0;
        for (; k + (U - 1) * 16 < count; k += U * 16)
#pragma unroll
            for (int u = 0; u < U; ++u) s[u] += part[(k + u * 16) * C + c];
        for (; k < count; k += 16) s[0] += part[k * C + c];
    }
    red[k0][threadIdx.x & 15] = (s[0] + s[1]) + (s[2] + s[3]);
    __syncthreads();
    if (threadIdx.x < 16 && c < C) {
        float t = 0.f;
        for (int i = 0; i < 16; ++i) t += red[i][threadIdx.x];
        store_param(dw, type, c, t);
    }
}

// ------------------------------------------------------------------------------------------
struct RmsPlan {
    int E, P, threads;           // pieces to a lane (0: any number, one after the other), lanes and threads of a block
    int64_t grid;
};

// A lane holds 16 numbers of a row; fewer where that leaves the chip with less than a block of 256 threads to a unit (one
// row of 4096: 1024 lanes of 4).
RmsPlan rms_plan(int64_t rows, int64_t C, int V) {
    RmsPlan p{};
    const int64_t pieces = ceil_div(std::max<int64_t>(C, 1), V), cus = compute_units();
    auto lanes = [&](int E) {
        int P = 1;
        while ((int64_t)P * E < pieces && P < kRmsMost) P *= 2;
        return P;
    };
    p.E = kRmsHeld / V;
    while (p.E > 1 && rows * lanes(p.E) < cus * kRmsBlock && lanes(p.E / 2) * (p.E / 2) >= pieces) p.E /= 2;
    p.P = lanes(p.E);
    if ((int64_t)p.P * p.E < pieces) p.E = 0;
    p.threads = p.P > 64 ? p.P : kRmsBlock;                  // waves that are joined through LDS are one team
    const int64_t teams = p.threads / p.P;
    p.grid = std::max<int64_t>(1, std::min(ceil_div(rows, teams), cus * (2048 / p.threads)));
    return p;
}
// Backward a block leaves a part of dw: no more blocks than are resident
int64_t rms_grad_grid(const RmsPlan& p) { return std::min<int64_t>(p.grid, compute_units() * std::max(1, 1024 / p.threads)); }

int fail(int code, const char* text) { return set_error(code, text); }
int launched(const char* where) {
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? DA_OK : set_hip_error(e, where);
}
bool known(int d) { return d == DA_F32 || d == DA_BF16; }

int rms_check(int dtype, int64_t rows, int64_t C, int param_dtype, float eps) {
    if (!known(dtype) || !known(param_dtype)) return fail(DA_ERR_UNSUPPORTED, "dtype is neither DA_F32 nor DA_BF16");
    if (rows < 0 || C < 0) return fail(DA_ERR_INVALID_ARG, "negative size");
    if (rows > INT32_MAX || C > 1 << 20) return fail(DA_ERR_UNSUPPORTED, "size too large");
    if (!(eps >= 0.f)) return fail(DA_ERR_INVALID_ARG, "eps is negative or no number");
    return DA_OK;
}

template <class T, int V, bool EIGHT> void launch(const RmsArgs<T>& a, hipStream_t s) {
    const RmsPlan p = rms_plan(a.rows, a.C, V);
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((unsigned)p.grid), dim3(p.threads), 0, s, a, p.P); };
    if (p.E == 0) return go(rms_kernel<T, V, 0, EIGHT>);
    if (p.E == 1) return go(rms_kernel<T, V, 1, EIGHT>);
    if (p.E == 2) return go(rms_kernel<T, V, 2, EIGHT>);
    if constexpr (V == 4) return go(rms_kernel<T, V, 4, EIGHT>);
}

template <class T, int V> void launch_grad(const RmsArgs<T>& a, void* dw, int type, hipStream_t s) {
    const RmsPlan p = rms_plan(a.rows, a.C, V);
    const int64_t grid = rms_grad_grid(p);
    const size_t lds = p.E && p.P <= 64 && p.threads > p.P && a.part ? (size_t)p.threads * p.E * V * sizeof(float) : 0;
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(p.threads), lds, s, a, p.P); };
    if (p.E == 0) go(rms_grad_kernel<T, V, 0>);
    else if (p.E == 1) go(rms_grad_kernel<T, V, 1>);
    else if (p.E == 2) go(rms_grad_kernel<T, V, 2>);
    if constexpr (V == 4) {
        if (p.E == 4) go(rms_grad_kernel<T, V, 4>);
    }
    if (dw)
        hipLaunchKernelGGL(rms_join_kernel, dim3((unsigned)ceil_div(a.C, 16)), dim3(256), 0, s, a.part, (long)(a.rows ? grid : 0), a.C, dw,
                           type);
}

template <class T> constexpr int rms_access() { return sizeof(T) == 4 ? 4 : 8; }

template <class T, bool EIGHT>
void forward(int64_t rows, int64_t C, const void* x, int64_t ldx, const void* res, int64_t ldr, const void* w, int w_type, float eps,
             void* sum, void* y, void* q, float* scale, hipStream_t s) {
    RmsArgs<T> a{};
    a.x = static_cast<const T*>(x);
    a.res = static_cast<const T*>(res);
    a.ldx = ldx;
    a.ldr = ldr;
    a.w = w;
    a.w_type = w_type;
    a.rows = rows;
    a.C = (int)C;
    a.eps = eps;
    a.sum = static_cast<T*>(sum);
    a.y = static_cast<T*>(y);
    a.q = static_cast<uint32_t*>(q);
    a.scale = scale;
    launch<T, rms_access<T>(), EIGHT>(a, s);
}

size_t rms_part_bytes(int dtype, int64_t rows, int64_t C) {
    return (size_t)rms_grad_grid(rms_plan(rows, C, dtype == DA_F32 ? 4 : 8)) * C * sizeof(float);
}

}  // namespace
}  // namespace daspmm

using namespace daspmm;

extern "C" int da_rms_norm_workspace(int dtype, int64_t rows, int64_t channels, size_t* backward_bytes)
{
    if (!backward_bytes) return fail(DA_ERR_INVALID_ARG, "null output");
    const int st = rms_check(dtype, rows, channels, DA_F32, 0.f);
    if (st != DA_OK) return st;
    *backward_bytes = rms_part_bytes(dtype, rows, channels);
    return DA_OK;
}

static int rms_forward_check(int dtype, int64_t rows, int64_t C, const void* x, int64_t ldx, const void* res, int64_t ldr, int param_dtype,
                             float eps, const void* sum, const void* y) {
    const int st = rms_check(dtype, rows, C, param_dtype, eps);
    if (st != DA_OK) return st;
    if (ldx < C || (res && ldr < C)) return fail(DA_ERR_INVALID_ARG, "leading dimension smaller than the extent it strides over");
    if (rows > 0 && C > 0 && (!x || !y || (res && !sum))) return fail(DA_ERR_INVALID_ARG, "null x, sum or result");
    return DA_OK;
}

extern "C" int da_rms_norm(int dtype, int64_t rows, int64_t channels, const void* x, int64_t ldx, const void* residual, int64_t ldr,
                           const void* w, int param_dtype, float eps, void* sum, void* y, void* stream)
{
    const int st = rms_forward_check(dtype, rows, channels, x, ldx, residual, ldr, param_dtype, eps, sum, y);
    if (st != DA_OK || rows == 0 || channels == 0) return st;
    if (dtype == DA_F32)
        forward<float, false>(rows, channels, x, ldx, residual, ldr, w, param_dtype, eps, sum, y, nullptr, nullptr, (hipStream_t)stream);
    else
        forward<bf16, false>(rows, channels, x, ldx, residual, ldr, w, param_dtype, eps, sum, y, nullptr, nullptr, (hipStream_t)stream);
    return launched("da_rms_norm launch");
}

extern "C" int da_rms_norm_e4m3(int dtype, int64_t rows, int64_t channels, const void* x, int64_t ldx, const void* residual, int64_t ldr,
                                const void* w, int param_dtype, float eps, void* sum, void* q, float* scale, void* stream)
{
    const int st = rms_forward_check(dtype, rows, channels, x, ldx, residual, ldr, param_dtype, eps, sum, q);
    if (st != DA_OK || rows == 0) return st;
    if (!scale) return fail(DA_ERR_INVALID_ARG, "null scale");
    if (dtype == DA_F32)
        forward<float, true>(rows, channels, x, ldx, residual, ldr, w, param_dtype, eps, sum, nullptr, q, scale, (hipStream_t)stream);
    else
        forward<bf16, true>(rows, channels, x, ldx, residual, ldr, w, param_dtype, eps, sum, nullptr, q, scale, (hipStream_t)stream);
    return launched("da_rms_norm_e4m3 launch");
}

extern "C" int da_rms_norm_backward(int dtype, int64_t rows, int64_t channels, const void* s, int64_t lds, const void* dy, int64_t ldy,
                                    const void* dsum, int64_t ldd, const void* w, int param_dtype, float eps, void* dx, void* dw,
                                    void* workspace, size_t workspace_bytes, void* stream)
{
    const int st = rms_check(dtype, rows, channels, param_dtype, eps);
    if (st != DA_OK) return st;
    if (lds < channels || (dy && ldy < channels) || (dsum && ldd < channels))
        return fail(DA_ERR_INVALID_ARG, "leading dimension smaller than the extent it strides over");
    if (channels == 0 || (!dx && !dw)) return DA_OK;
    if (rows > 0 && !s) return fail(DA_ERR_INVALID_ARG, "null s");
    if (dw && (!workspace || workspace_bytes < rms_part_bytes(dtype, rows, channels) || reinterpret_cast<uintptr_t>(workspace) % 16 != 0))
        return fail(DA_ERR_INVALID_ARG, "workspace missing, misaligned or smaller than reported");
    auto go = [&](auto tag) {
        typedef decltype(tag) T;
        RmsArgs<T> a{};
        a.x = static_cast<const T*>(s);
        a.dy = static_cast<const T*>(dy);
        a.dsum = static_cast<const T*>(dsum);
        a.ldx = lds;
        a.ldy = ldy;
        a.ldd = ldd;
        a.w = w;
        a.w_type = param_dtype;
        a.rows = rows;
        a.C = (int)channels;
        a.eps = eps;
        a.y = static_cast<T*>(dx);
        a.part = dw ? static_cast<float*>(workspace) : nullptr;
        launch_grad<T, rms_access<T>()>(a, dw, param_dtype, (hipStream_t)stream);
    };
    if (dtype == DA_F32) go(float());
    else go(bf16());
    return launched("da_rms_norm_backward launch");
}
