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
// Activations.  exp goes to the hardware's 2^x (relative error about |z| 2^-24), the reciprocal of a
// logistic sum to v_rcp (1 unit in the last place).
// ------------------------------------------------------------------------------------------
__device__ __forceinline__ float logistic(float z) { return __builtin_amdgcn_rcpf(1.f + __expf(-z)); }

__device__ __forceinline__ float gauss_cdf(float z) { return 0.5f * erfcf(-0.70710678118654752f * z); }

__device__ __forceinline__ float act_value(int act, float z) {
    switch (act) {
        case DA_ACT_RELU: return z > 0.f || z != z ? z : 0.f;              // NaN stays NaN
        case DA_ACT_SILU: return z * logistic(z);
        case DA_ACT_GELU: return z * gauss_cdf(z);
        case DA_ACT_SIGMOID: return logistic(z);
        default: return z;
    }
}

// Value and derivative
__device__ __forceinline__ float act_slope(int act, float z, float* value) {
    switch (act) {
        case DA_ACT_RELU: *value = z > 0.f || z != z ? z : 0.f; return z > 0.f ? 1.f : z != z ? z : 0.f;
        case DA_ACT_SILU: {
            const float s = logistic(z);
            *value = z * s;
            return s * (1.f + z * (1.f - s));
        }
        case DA_ACT_GELU: {
            const float c = gauss_cdf(z);
            *value = z * c;
            return c + z * 0.39894228040143268f * __expf(-0.5f * z * z);
        }
        case DA_ACT_SIGMOID: {
            const float s = logistic(z);
            *value = s;
            return s * (1.f - s);
        }
        default: *value = z; return 1.f;
    }
}

__device__ __forceinline__ float wave_sum(float x, int lanes) {
    for (int d = 1; d < lanes; d <<= 1) x += __shfl_xor(x, d, 64);
    return x;
}

}  // namespace daspmm
