// Orthogonalised updates of small matrices: up to 64 x 512 (or turned around), one block to a matrix, which stays in LDS for all
// steps.  The products are da_planes.h's, of pairs of fp16 halves; with a launch to each product the steps of a 64 x 256 matrix
// took 68 us, nearly all of it launches.
//
// A wave of the 16 owns a fragment of A and of b A + c A^2, which takes A's place, and every sixteenth 16 columns of X,
// which it replaces after reading them: only the two small matrices have to be waited for.
// 64 x 64, 64 x 256 and 64 x 512 float32, five steps: 18, 35 and 58 us; a step of 64 x 256 is 5.4, 1.4 of it at the matrix cores' rate of
// one unit.  (Blocks of 32 x 32 of A to a wave, with a quarter of the inner axis each, read half as much from LDS and took as long.)
#pragma once
#include "da_planes.h"

namespace daspmm {

constexpr int kSmallSide = 64, kSmallLong = 512, kSmallThreads = 1024, kSmallSteps = 64;

struct SmallStep {
    float gram, poly_b, poly_c, a, by;       // A = gram X X^T;  B = poly_b A + poly_c A A;  X <- a X + by B X, in their scales
};
struct SmallArgs {
    long ldg, stride;
    int rows, cols, steps;
    float eps, first, last;                  // scale of X at first, what its last scale is divided by
    SmallStep step[kSmallSteps];
};

constexpr int small_pitch(int n) { return n * 4 + 16; }                      // bytes of n pairs
inline size_t small_lds(int n) { return (size_t)kSmallSide * (small_pitch(n) + small_pitch(kSmallSide)); }

// Fragments of pairs in LDS, lines along or across the inner axis
__device__ __forceinline__ f16x8 small_along(const char* at, int pitch, int o, int k, int s) {
    const int i = threadIdx.x & 15, h = (threadIdx.x & 63) >> 4;
    return *reinterpret_cast<const f16x8*>(at + (o + i) * pitch + k * 128 + s * 64 + h * 16);
}
__device__ __forceinline__ f16x8 small_across(const char* at, int pitch, int o, int k, int s) {
    typedef __attribute__((address_space(3))) s16x4* Lds;
    const int i = threadIdx.x & 15, h = (threadIdx.x & 63) >> 4;
    union { s16x4 half[2]; f16x8 all; } f;
#pragma unroll
    for (int n = 0; n < 2; ++n)
        f.half[n] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (Lds)(at + (k * 32 + h * 8 + n * 4 + i / 4) * pitch + o / 32 * 128 + s * 64 + o % 32 * 2 + (i & 3) * 8));
    return f.all;
}

template <class T>
__global__ __launch_bounds__(kSmallThreads) void orth_small_kernel(const T* __restrict__ g, T* __restrict__ out, SmallArgs a, int n)
{
    extern __shared__ __attribute__((aligned(16))) char lds[];
    __shared__ double red[kSmallThreads / 64];
    constexpr int PA = small_pitch(kSmallSide);
    const int PX = small_pitch(n), tid = threadIdx.x, lane = tid & 63, i16 = lane & 15, h = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    char* const X = lds;
    char* const A = lds + kSmallSide * PX;
    const bool tall = a.rows > a.cols;
    const T* __restrict__ p = g + blockIdx.x * a.stride;
    // A thread's fours of neighbours in a row, all of them on their way at once
    constexpr int FOURS = kSmallSide * kSmallLong / 4 / kSmallThreads;
    const int across = (a.cols + 3) / 4, all = a.rows * across;
    f32x4 x[FOURS];
    auto each = [&](auto&& f) {
#pragma unroll
        for (int i = 0; i < FOURS; ++i) {
            const int k = tid + i * kSmallThreads;
            if (k < all) f(x[i], k / across, k % across * 4);
        }
    };
    each([&](f32x4& v, int r, int c) {
        const T* __restrict__ q = p + r * a.ldg + c;
        float y[4] = {0.f, 0.f, 0.f, 0.f};
        if (c + 4 <= a.cols) {
            load_floats<4>(q, y);
        } else {
#pragma unroll
            for (int i = 0; i < 3; ++i)
                if (c + i < a.cols) {
                    float one[1];
                    load_floats<1>(q + i, one);
                    y[i] = one[0];
                }
        }
        v = f32x4{y[0], y[1], y[2], y[3]};
    });
    for (int k = tid * 16; k < kSmallSide * PX; k += kSmallThreads * 16) *reinterpret_cast<uint4*>(X + k) = make_uint4(0, 0, 0, 0);
    double s = 0.0;
    each([&](f32x4& v, int, int) {
#pragma unroll
        for (int i = 0; i < 4; ++i) s += (double)v[i] * (double)v[i];
    });
    s = wave_sum(s, 64);
    if (lane == 0) red[wave] = s;
    __syncthreads();
    s = 0.0;
    for (int k = 0; k < kSmallThreads / 64; ++k) s += red[k];
    const double f = (double)a.first / (sqrt(s) + (double)a.eps);
    each([&](f32x4& v, int r, int c) {
        float y[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = (float)((double)v[i] * f);
        if (tall) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float one[1] = {y[i]};
                if (c + i < a.cols) put_values<Halves, 1>(in_line<Halves>(reinterpret_cast<uint16_t*>(X + (c + i) * PX), r), one);
            }
        } else {
            put_values<Halves, 4>(in_line<Halves>(reinterpret_cast<uint16_t*>(X + r * PX), c), y);
        }
    });
    __syncthreads();

    // the wave's fragment: rows m and on, columns j and on
    const int m = wave / 4 * 16, j = wave % 4 * 16;
    // n inner positions, two steps at a time; three sums, whose products need not wait for each other
    auto square = [&](const char* from, int pitch, int positions) {
        f32x4 acc[3] = {};
        for (int k = 0; k < positions / 32; k += 2) {
            f16x8 x[2][2], y[2][2];
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    x[u][s] = small_along(from, pitch, m, k + u, s);
                    y[u][s] = small_along(from, pitch, j, k + u, s);
                }
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                acc[0] = Halves::mul(y[u][0], x[u][0], acc[0]);
                acc[1] = Halves::mul(y[u][1], x[u][0], acc[1]);
                acc[2] = Halves::mul(y[u][0], x[u][1], acc[2]);
            }
        }
        return acc[0] + (acc[1] + acc[2]);
    };
    uint16_t* const mine = in_line<Halves>(reinterpret_cast<uint16_t*>(A + (m + i16) * PA), j + 4 * h);
    for (int k = 0; k < a.steps; ++k) {
        const SmallStep& t = a.step[k];
        f32x4 acc = square(X, PX, n);
        float v[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) v[q] = t.gram * acc[q];
        put_values<Halves, 4>(mine, v);
        __syncthreads();
        acc = square(A, PA, kSmallSide);
        get_values<Halves, 4>(mine, v);
#pragma unroll
        for (int q = 0; q < 4; ++q) v[q] = t.poly_b * v[q] + t.poly_c * acc[q];
        __syncthreads();                                     // A has been read
        put_values<Halves, 4>(mine, v);
        __syncthreads();
        f16x8 b[4][2][2];                                    // rows, inner positions, halves
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int q = 0; q < 4; ++q) b[r][q / 2][q % 2] = small_along(A, PA, r * 16, q / 2, q % 2);
        for (int c = wave * 16; c < n; c += kSmallThreads / 64 * 16) {
            f32x4 sum[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) sum[r] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const f16x8 x = small_across(X, PX, c, q, 0), x2 = small_across(X, PX, c, q, 1);
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    sum[r] = Halves::mul(x, b[r][q][0], sum[r]);
                    sum[r] = Halves::mul(x2, b[r][q][0], sum[r]);
                    sum[r] = Halves::mul(x, b[r][q][1], sum[r]);
                }
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                uint16_t* const to = in_line<Halves>(reinterpret_cast<uint16_t*>(X + (r * 16 + i16) * PX), c + 4 * h);
                float x[4];
                get_values<Halves, 4>(to, x);
#pragma unroll
                for (int q = 0; q < 4; ++q) x[q] = t.a * x[q] + t.by * sum[r][q];
                put_values<Halves, 4>(to, x);
            }
        }
        __syncthreads();
    }
    T* __restrict__ o = out + (long)blockIdx.x * a.rows * a.cols;
    each([&](f32x4&, int r, int c) {
        float y[4];
        if (tall) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float one[1];
                get_values<Halves, 1>(in_line<Halves>(reinterpret_cast<const uint16_t*>(X + (c + i) * PX), r), one);      // lines up to 63 are there
                y[i] = one[0];
            }
        } else {
            get_values<Halves, 4>(in_line<Halves>(reinterpret_cast<const uint16_t*>(X + r * PX), c), y);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] *= a.last;
        T* __restrict__ q = o + r * a.cols + c;
        if (c + 4 <= a.cols) {
            store_floats<4>(q, y);
        } else {
#pragma unroll
            for (int i = 0; i < 3; ++i) {
                const float one[1] = {y[i]};
                if (c + i < a.cols) store_floats<1>(q + i, one);
            }
        }
    });
}

}  // namespace daspmm
