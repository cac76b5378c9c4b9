// Device helpers of the layers around an aggregation: vectors of float or bf16 as floats, activations.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "da_layers.h"

namespace daspmm {

typedef __bf16 bf16;

// V neighbouring elements as one access, at any address that an element may have: the memory system takes wide
// accesses at the alignment of an element, so V follows from the sizes alone.
template <class T, int V> struct Pack { typedef T type __attribute__((ext_vector_type(V), aligned(sizeof(T)))); };
template <class T> struct Pack<T, 1> { typedef T type; };

template <int V> __device__ __forceinline__ void load_floats(const float* __restrict__ p, float (&x)[V]) {
    const typename Pack<float, V>::type v = *reinterpret_cast<const typename Pack<float, V>::type*>(p);
    if constexpr (V == 1) x[0] = v;
    else
#pragma unroll
        for (int i = 0; i < V; ++i) x[i] = v[i];
}

// bf16 is the upper half of a float
template <int V> __device__ __forceinline__ void load_floats(const bf16* __restrict__ p, float (&x)[V]) {
    const typename Pack<uint16_t, V>::type v = *reinterpret_cast<const typename Pack<uint16_t, V>::type*>(p);
    if constexpr (V == 1) x[0] = __uint_as_float((uint32_t)v << 16);
    else
#pragma unroll
        for (int i = 0; i < V; ++i) x[i] = __uint_as_float((uint32_t)v[i] << 16);
}

template <int V> __device__ __forceinline__ void store_floats(float* __restrict__ p, const float (&x)[V]) {
    typename Pack<float, V>::type v;
    if constexpr (V == 1) v = x[0];
    else
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = x[i];
    *reinterpret_cast<typename Pack<float, V>::type*>(p) = v;
}

// Rounds once, to nearest even
template <int V> __device__ __forceinline__ void store_floats(bf16* __restrict__ p, const float (&x)[V]) {
    typename Pack<bf16, V>::type v;
    if constexpr (V == 1) v = (bf16)x[0];
    else
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = (bf16)x[i];
    *reinterpret_cast<typename Pack<bf16, V>::type*>(p) = v;
}

// A number of an array whose type is known at run time only (parameters; a few loads a thread)
__device__ __forceinline__ float load_param(const void* p, int dtype, long at) {
    return dtype == DA_F32 ? static_cast<const float*>(p)[at]
                           : __uint_as_float((uint32_t) static_cast<const uint16_t*>(p)[at] << 16);
}
__device__ __forceinline__ void store_param(void* p, int dtype, long at, float x) {
    if (dtype == DA_F32) static_cast<float*>(p)[at] = x;
    else static_cast<bf16*>(p)[at] = (bf16)x;
}

// ------------------------------------------------------------------------------------------
// Activations, several numbers at once: the choice is one branch for all of them, and their instructions interleave.
// 2^x and 1 / x are the hardware's (1 unit in the last place; the argument of 2^x is rounded: |z| 2^-24 of the result).
// ------------------------------------------------------------------------------------------
__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float rcp_hw(float x) { return __builtin_amdgcn_rcpf(x); }

__device__ __forceinline__ float logistic(float z) { return rcp_hw(1.f + exp2_hw(-1.44269504088896f * z)); }

// Normal distribution function: the logistic function of an odd polynomial of z, fitted by weighted least squares to
// log(cdf(z) / cdf(-z)) for |z| up to 6.5 and growing beyond; off by 7e-8 at most, 1.2e-7 with roundings.  Relative to the
// value that is 1.5e-5 at -3, 3e-4 at -4, 4e-2 at -5 and all of it below -6, as in (1 + erf(z / sqrt 2)) / 2 taken in float32
// (1.1e-5, 5e-4, 5e-2); z times it is off by 2e-7 at most, and by less than 8e-8 below -1.  One exponential and one reciprocal: the
// library's erfc, which keeps the tail's digits, made the bf16 passes over 262 144 x 128 compute-bound.
__device__ __forceinline__ float gauss_cdf(float z) {
    constexpr float L = -1.44269504088896f;
    const float q = z * z;
    float p = L * 3.6186230580754275e-09f;
    p = p * q + L * -2.672895868257473e-07f;
    p = p * q + L * 7.946166252355732e-06f;
    p = p * q + L * -0.00011055548966006326f;
    p = p * q + L * -6.59107019500109e-05f;
    p = p * q + L * 0.07266782413685334f;
    p = p * q + L * 1.5957689848135383f;
    return rcp_hw(1.f + exp2_hw(p * z));
}
__device__ __forceinline__ float gauss_density(float z) {
    return 0.39894228040143268f * exp2_hw(-0.72134752044448f * z * z);
}

// z becomes act(z)
template <int N> __device__ __forceinline__ void act_values(int act, float (&z)[N]) {
    switch (act) {
        case DA_ACT_RELU:
#pragma unroll
            for (int i = 0; i < N; ++i) z[i] = z[i] > 0.f || z[i] != z[i] ? z[i] : 0.f;    // NaN stays NaN
            break;
        case DA_ACT_SILU:
#pragma unroll
            for (int i = 0; i < N; ++i) z[i] *= logistic(z[i]);
            break;
        case DA_ACT_GELU:
#pragma unroll
            for (int i = 0; i < N; ++i) z[i] *= gauss_cdf(z[i]);
            break;
        case DA_ACT_SIGMOID:
#pragma unroll
            for (int i = 0; i < N; ++i) z[i] = logistic(z[i]);
            break;
        default: break;
    }
}

// z becomes act(z), slope its derivative
template <int N> __device__ __forceinline__ void act_both(int act, float (&z)[N], float (&slope)[N]) {
    switch (act) {
        case DA_ACT_RELU:
#pragma unroll
            for (int i = 0; i < N; ++i) {
                slope[i] = z[i] > 0.f ? 1.f : z[i] != z[i] ? z[i] : 0.f;
                z[i] = z[i] > 0.f || z[i] != z[i] ? z[i] : 0.f;
            }
            break;
        case DA_ACT_SILU:
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float s = logistic(z[i]);
                slope[i] = s * (1.f + z[i] * (1.f - s));
                z[i] *= s;
            }
            break;
        case DA_ACT_GELU:
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float c = gauss_cdf(z[i]);
                slope[i] = c + z[i] * gauss_density(z[i]);
                z[i] *= c;
            }
            break;
        case DA_ACT_SIGMOID:
#pragma unroll
            for (int i = 0; i < N; ++i) {
                z[i] = logistic(z[i]);
                slope[i] = z[i] * (1.f - z[i]);
            }
            break;
        default:
#pragma unroll
            for (int i = 0; i < N; ++i) slope[i] = 1.f;
            break;
    }
}

// z becomes the derivative
template <int N> __device__ __forceinline__ void act_slopes(int act, float (&z)[N]) {
    float slope[N];
    act_both(act, z, slope);
#pragma unroll
    for (int i = 0; i < N; ++i) z[i] = slope[i];
}

template <class S> __device__ __forceinline__ S wave_sum(S x, int lanes) {
    for (int d = 1; d < lanes; d <<= 1) x += __shfl_xor(x, d, 64);
    return x;
}

}  // namespace daspmm
