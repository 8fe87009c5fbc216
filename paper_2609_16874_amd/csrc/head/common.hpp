// common.hpp -- element types, vector access and activations shared by
// the head operators (group norm, linear).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "cpe_head.h"

namespace cpe {

typedef __bf16 bf16_t;

// V elements that need no more than their own alignment: global memory
// serves vector accesses at any element boundary with the same instruction.
template <typename T, int V>
struct __attribute__((packed, aligned(sizeof(T)))) Vec {
    T v[V];
};

template <typename T, int V>
__device__ __forceinline__ Vec<T, V> load_vec(const T *p)
{
    return *reinterpret_cast<const Vec<T, V> *>(p);
}
template <typename T, int V>
__device__ __forceinline__ void store_vec(T *p, const Vec<T, V> &v)
{
    *reinterpret_cast<Vec<T, V> *>(p) = v;
}

constexpr float kLog2e = 1.44269504088896340736f;

__device__ __forceinline__ float sigmoid(float u)
{
    return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-kLog2e * u));
}

// Phi(-|u|) / e^(-u^2 / 2), Phi the standard normal distribution: a polynomial
// in t = 1 / (1 + 0.305 |u|), fitted for the least relative error (9.4e-8; 4e-7
// as binary32 evaluates it).  The exponential is left to the caller, which
// needs it for the density as well; erff costs about twice the instructions.
__device__ __forceinline__ float normal_tail(float u)
{
    const float t = __builtin_amdgcn_rcpf(fmaf(0.305f, fabsf(u), 1.0f));
    float q = fmaf(0.0366991939f, t, -0.152988325f);
    q = fmaf(q, t, 0.185716921f);
    q = fmaf(q, t, -0.0379768429f);
    q = fmaf(q, t, 0.121021685f);
    q = fmaf(q, t, 0.103420864f);
    q = fmaf(q, t, 0.122466817f);
    q = fmaf(q, t, 0.121639733f);
    return q * t;
}
__device__ __forceinline__ float gauss(float u) { return __builtin_amdgcn_exp2f(-0.5f * kLog2e * u * u); }

// act(u), in binary32.  A NaN stays a NaN; SiLU and GELU of -infinity are
// the product -inf * 0, a NaN.
template <int ACT>
__device__ __forceinline__ float activate(float u)
{
    if constexpr (ACT == CPE_ACT_RELU) return u < 0.0f ? 0.0f : u;
    if constexpr (ACT == CPE_ACT_SILU) return u * sigmoid(u);
    if constexpr (ACT == CPE_ACT_GELU) {
        const float q = normal_tail(u) * gauss(u);
        return u * (u > 0.0f ? 1.0f - q : q);
    }
    return u;
}

// act'(u); ReLU's derivative at 0 is 0.  A NaN stays a NaN; SiLU's and GELU's
// at an infinity are products inf * 0, NaNs.
template <int ACT>
__device__ __forceinline__ float activate_grad(float u)
{
    if constexpr (ACT == CPE_ACT_RELU) return u > 0.0f ? 1.0f : u <= 0.0f ? 0.0f : u;
    if constexpr (ACT == CPE_ACT_SILU) {
        const float s = sigmoid(u);
        return s * (1.0f + u * (1.0f - s));
    }
    if constexpr (ACT == CPE_ACT_GELU) {
        const float e = gauss(u), q = normal_tail(u) * e;
        return fmaf(0.39894228040143267794f * u, e, u > 0.0f ? 1.0f - q : q);
    }
    return 1.0f;
}

// The work that workgroup w of n takes: workgroups are dealt to the eight XCDs
// in turn, so this gives each XCD a run of neighbours, which share lines of
// its L2.
__device__ __forceinline__ int xcd_order(int w, int n)
{
    const int each = n / 8, more = n % 8, x = w % 8;
    return x * each + (x < more ? x : more) + w / 8;
}

__host__ __device__ inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

inline bool aligned_to(const void *p, size_t a) { return ((uintptr_t)p % a) == 0; }
inline size_t element_size(cpe_head_dtype t) { return t == CPE_HEAD_F32 ? 4 : 2; }
inline size_t align256(size_t v) { return (v + 255) / 256 * 256; }

}  // namespace cpe
