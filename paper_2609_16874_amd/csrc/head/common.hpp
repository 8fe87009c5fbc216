// common.hpp -- element types, vector access and activations shared by
// the head operators (group norm, linear).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <initializer_list>
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

// (Stored as one vector of words: from the structure the compiler makes pieces of
// three words, one and a half where the same code stores single elements too, and
// the stores of 16-bit rows reach two thirds of their rate.  The group norm's gradient
// of 307,039 x 100 in f16 with ReLU takes 40 registers more so, which leaves three
// waves of a SIMD instead of four, and 70 us instead of 74.)  PAST: past the caches.
template <typename T, int V>
__device__ __forceinline__ Vec<T, V> load_vec(const T *p)
{
    return *reinterpret_cast<const Vec<T, V> *>(p);
}
template <bool PAST = false, typename T, int V>
__device__ __forceinline__ void store_words(T *p, const Vec<T, V> &v)
{
    typedef uint32_t words __attribute__((ext_vector_type(sizeof(v) / 4), aligned(sizeof(T))));
    words w;
    __builtin_memcpy(&w, &v, sizeof v);
    if constexpr (PAST)
        __builtin_nontemporal_store(w, reinterpret_cast<words *>(p));
    else
        *reinterpret_cast<words *>(p) = w;
}
template <typename T, int V>
__device__ __forceinline__ void store_vec(T *p, const Vec<T, V> &v)
{
    if constexpr (sizeof(v) % 8 == 0)
        store_words(p, v);
    else
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

// A binary32 result that is rounded to T as it stands.  (In f16 the compiler
// makes one instruction of a product or sum and its conversion, which rounds
// once, but not everywhere: equal operands would give different values.)
template <typename T>
__device__ __forceinline__ T rounded(float x)
{
    if constexpr (std::is_same<T, _Float16>::value) asm("" : "+v"(x));
    return (T)x;
}
// A byte times its row's scale.
template <typename T>
__device__ __forceinline__ T scaled_byte(int8_t q, float scale) { return rounded<T>((float)q * scale); }

// A row's scale as f p: where FOLD, f is its mantissa (1 <= f < 2) and p a
// power of two, by which bytes are exact in 16 bits; otherwise f is 1.  (So it
// is for scales without a mantissa: 0, infinities, NaNs, subnormal ones.)
struct ScaleParts {
    float f, p;
};
template <bool FOLD>
__device__ __forceinline__ ScaleParts scale_parts(float s)
{
    const uint32_t b = __builtin_bit_cast(uint32_t, s);
    const bool normal = FOLD && ((b >> 23) & 255) - 1 < 254;
    return {normal ? __builtin_bit_cast(float, (b & 0x007fffffu) | 0x3f800000u) : 1.0f,
            normal ? __builtin_bit_cast(float, b & 0xff800000u) : s};
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
// Whether an output (null: not wanted) is none of these arguments of its call.
inline bool apart(const void *out, std::initializer_list<const void *> others)
{
    for (const void *p : others)
        if (out && out == p) return false;
    return true;
}
inline size_t element_size(cpe_head_dtype t) { return t == CPE_HEAD_F32 ? 4 : 2; }
inline size_t align256(size_t v) { return (v + 255) / 256 * 256; }

}  // namespace cpe
