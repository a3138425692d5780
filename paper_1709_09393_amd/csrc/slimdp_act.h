// Activations of the product's epilogue and their slopes, binary32.  Included only by slimdp_train.hip.
#pragma once
#include "slimdp_train.h"

namespace slimdp {

enum : int { ACT_NONE = 0, ACT_RELU = 1, ACT_GELU = 2, ACT_GELU_TANH = 3, ACT_SILU = 4, ACTS = 5 };

constexpr float LOG2E = 1.4426950408889634f;

// exp(-a^2 / 2) and the normal distribution function at -a, for a >= 0.  The latter is exp(-a^2 / 2) times a function that varies
// slowly: a polynomial of degree 8 in 1 / (1 + 0.3 a), fitted here over a <= 14 by weighted least squares.  With the constants as they stand,
// rounded to binary32, it is off by 9.6e-8 of the value at most, and by 4.1e-7 where it is evaluated in binary32; behind 14 the exponential is
// zero in binary32.  The exponential adds a^2 / 2 times three roundings of its argument (1e-5 of the value at a = 12).  Twenty instructions, where
// the library's complementary error function takes more time than the memory this work waits for.
__device__ __forceinline__ float normal_tail(float a, float& density)
{
    a = a > 14.2f ? 14.2f : a;
    const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.3f, a, 1.0f));
    density = __builtin_amdgcn_exp2f(a * a * (-0.5f * LOG2E));
    float p = 0.038378290832042694f;
    p = __builtin_fmaf(p, t, -0.16916611790657043f);
    p = __builtin_fmaf(p, t, 0.22866007685661316f);
    p = __builtin_fmaf(p, t, -0.07650648057460785f);
    p = __builtin_fmaf(p, t, 0.1425355225801468f);
    p = __builtin_fmaf(p, t, 0.09468352049589157f);
    p = __builtin_fmaf(p, t, 0.12192033976316452f);
    p = __builtin_fmaf(p, t, 0.1194876879453659f);
    p = __builtin_fmaf(p, t, 7.168875981733436e-06f);
    return density * p;
}

// 1 / (1 + exp(-u)) and its slope, from one exponential of -|u| (no difference of nearly equal numbers on either side).
__device__ __forceinline__ float sigmoid(float u, float& slope)
{
    const float e = __builtin_amdgcn_exp2f(__builtin_fabsf(u) * -LOG2E);
    const float big = __builtin_amdgcn_rcpf(1.0f + e), small = e * big;
    slope = small * big;
    return u < 0.0f ? small : big;
}

// Where a zero would meet an infinite z, the factor z is held finite (a comparison lets a NaN through).
__device__ __forceinline__ float held(float z, float most) { return __builtin_fabsf(z) > most ? __builtin_copysignf(most, z) : z; }

constexpr float TANH_SCALE2 = 1.5957691216057308f;          // 2 sqrt(2 / pi): 0.5 (1 + tanh u) = 1 / (1 + exp(-2 u))

template <int ACT> __device__ __forceinline__ float act_slope(float z)
{
    if constexpr (ACT == ACT_RELU) return z > 0.0f ? 1.0f : 0.0f;
    if constexpr (ACT == ACT_GELU) {
        const float zz = held(z, 1000.0f);
        float density;
        const float tail = normal_tail(__builtin_fabsf(zz), density);
        return __builtin_fmaf(zz * 0.39894228040143268f, density, z < 0.0f ? tail : 1.0f - tail);
    }
    if constexpr (ACT == ACT_GELU_TANH) {
        const float zz = held(z, 1000.0f), z2 = zz * zz;
        float slope;
        const float s = sigmoid(TANH_SCALE2 * zz * __builtin_fmaf(0.044715f, z2, 1.0f), slope);
        return __builtin_fmaf(zz * slope * TANH_SCALE2, __builtin_fmaf(0.134145f, z2, 1.0f), s);
    }
    if constexpr (ACT == ACT_SILU) {
        const float zz = held(z, 1000.0f);
        float slope;
        const float s = sigmoid(zz, slope);
        return __builtin_fmaf(zz, slope, s);
    }
    return 1.0f;
}

template <int ACT> __device__ __forceinline__ float act_value(float z)
{
    if constexpr (ACT == ACT_RELU) return z < 0.0f ? 0.0f : z;
    if constexpr (ACT == ACT_GELU) {
        float density;
        const float tail = normal_tail(__builtin_fabsf(z), density);
        return z < 0.0f ? (z < -1000.0f ? 0.0f : z * tail) : __builtin_fmaf(-(z > 14.2f ? 0.0f : z), tail, z);
    }
    if constexpr (ACT == ACT_GELU_TANH || ACT == ACT_SILU) {
        const float zz = z < -1000.0f ? -1000.0f : z;
        float slope;
        if constexpr (ACT == ACT_SILU) return zz * sigmoid(zz, slope);
        const float c = held(zz, 1000.0f);
        return zz * sigmoid(TANH_SCALE2 * c * __builtin_fmaf(0.044715f, c * c, 1.0f), slope);
    }
    return z;
}

// One choice for several values.
template <class F> __device__ __forceinline__ void with_act(int act, F&& f)
{
    switch (act) {
    case ACT_RELU: f(std::integral_constant<int, ACT_RELU>{}); break;
    case ACT_GELU: f(std::integral_constant<int, ACT_GELU>{}); break;
    case ACT_GELU_TANH: f(std::integral_constant<int, ACT_GELU_TANH>{}); break;
    case ACT_SILU: f(std::integral_constant<int, ACT_SILU>{}); break;
    default: break;
    }
}
template <int N> __device__ __forceinline__ void act_values(float (&v)[N], int act)
{
    with_act(act, [&](auto a) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = act_value<decltype(a)::value>(v[i]);
    });
}

}  // namespace slimdp
