// Device-side building blocks of the worker side's training operators: element types, sums over groups of lanes.
// Included only by slimdp_train.hip.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <type_traits>

#include "slimdp.h"

namespace slimdp {

constexpr int MAXW_T = SLIMDP_MAX_WORKERS;
struct InTab { const void* p[MAXW_T]; };          // host pointer tables travel as kernel arguments
struct OutTab { void* p[MAXW_T]; };
struct RowTab { uint32_t n[MAXW_T]; };            // rows of every worker

// Sixteen bytes of elements at any address that an element may have: rows of odd width begin at odd places, and the hardware asks
// for no more (the types say so to the compiler, which would otherwise load element by element).
typedef uint32_t raw4 __attribute__((ext_vector_type(4)));
template <class T> struct Vec;
template <> struct Vec<float> {
    static constexpr int N = 4;
    typedef uint32_t any __attribute__((ext_vector_type(4), aligned(4)));
};
template <> struct Vec<_Float16> {
    static constexpr int N = 8;
    typedef uint32_t any __attribute__((ext_vector_type(4), aligned(2)));
};
template <> struct Vec<__bf16> {
    static constexpr int N = 8;
    typedef uint32_t any __attribute__((ext_vector_type(4), aligned(2)));
};

template <class T, int NT = 0> __device__ __forceinline__ raw4 load_raw(const T* p)
{
    typedef typename Vec<T>::any any;
    any v;
    if (NT) v = __builtin_nontemporal_load(reinterpret_cast<const any*>(p));
    else v = *reinterpret_cast<const any*>(p);
    return raw4{v.x, v.y, v.z, v.w};
}
template <class T, int NT = 0> __device__ __forceinline__ void store_raw(T* p, raw4 v)
{
    typedef typename Vec<T>::any any;
    any o = {v.x, v.y, v.z, v.w};
    if (NT) __builtin_nontemporal_store(o, reinterpret_cast<any*>(p));
    else *reinterpret_cast<any*>(p) = o;
}

template <class T> union Pack { raw4 r; T e[Vec<T>::N]; };

template <class T> __device__ __forceinline__ void unpack(raw4 r, float f[Vec<T>::N])
{
    Pack<T> p;
    p.r = r;
#pragma unroll
    for (int i = 0; i < Vec<T>::N; ++i) f[i] = (float)p.e[i];
}
// One rounding to nearest even for the sixteen-bit types.
template <class T> __device__ __forceinline__ raw4 pack(const float f[Vec<T>::N])
{
    Pack<T> p;
#pragma unroll
    for (int i = 0; i < Vec<T>::N; ++i) p.e[i] = (T)f[i];
    return p.r;
}

// Sixteen bytes moved down by k elements (0 < k < Vec<T>::N), zeros behind.
template <class T> __device__ __forceinline__ raw4 move_down(raw4 v, uint32_t k)
{
    const uint32_t words = sizeof(T) == 2 ? k >> 1 : k;
    if (words & 1u) v = raw4{v.y, v.z, v.w, 0};
    if (words & 2u) v = raw4{v.z, v.w, 0, 0};
    if (sizeof(T) == 2) {
        const uint32_t s = (k & 1u) * 16u;
        v = raw4{__builtin_amdgcn_alignbit(v.y, v.x, s), __builtin_amdgcn_alignbit(v.z, v.y, s), __builtin_amdgcn_alignbit(v.w, v.z, s), v.w >> s};
    }
    return v;
}

// Elements [c, c + N) of a row of `cols` (c < cols): what lies behind the row's end is not touched and reads as zero.  The last, broken vector
// of a row is taken from the sixteen bytes that end with the row, and moved down.  (Kernels that hold whole rows in registers take the
// elements behind the last whole vector one a lane instead: the code for broken vectors costs registers in every vector's place.)
template <class T, int NT = 0> __device__ __forceinline__ raw4 load_clip(const T* row, uint32_t c, uint32_t cols)
{
    constexpr uint32_t N = Vec<T>::N;
    if (c + N <= cols) return load_raw<T, NT>(row + c);
    if (cols >= N) return move_down<T>(load_raw<T, NT>(row + cols - N), c + N - cols);
    Pack<T> p;
    p.r = raw4{0, 0, 0, 0};
#pragma unroll
    for (uint32_t i = 0; i < N - 1; ++i)
        if (i < cols) p.e[i] = row[i];
    return p.r;
}
template <class T, int NT = 0> __device__ __forceinline__ void store_clip(T* row, uint32_t c, uint32_t cols, raw4 v)
{
    constexpr uint32_t N = Vec<T>::N;
    if (c + N <= cols) { store_raw<T, NT>(row + c, v); return; }
    Pack<T> p;
    p.r = v;
#pragma unroll
    for (uint32_t i = 0; i < N; ++i)
        if (c + i < cols) row[c + i] = p.e[i];
}

// N consecutive binary32 parameters from any address a float may have (c < cols).
template <int N> __device__ __forceinline__ void load_params(const float* row, uint32_t c, uint32_t cols, float (&f)[N])
{
#pragma unroll
    for (int i = 0; i < N; i += 4) {
        const raw4 v = c + i < cols ? load_clip<float>(row, c + i, cols) : raw4{0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < 4; ++j) f[i + j] = __uint_as_float(v[j]);
    }
}

template <int N> __device__ __forceinline__ void load_whole(const float* p, float (&f)[N])
{
#pragma unroll
    for (int i = 0; i < N; i += 4) {
        const raw4 v = load_raw<float>(p + i);
#pragma unroll
        for (int j = 0; j < 4; ++j) f[i + j] = __uint_as_float(v[j]);
    }
}

// Sum over a wave by data-parallel moves, the order of additions fixed; every lane gets it.
__device__ __forceinline__ float wave_sum_f(float v)
{
#define SLIMDP_ADD_DPP(ctrl, rows) v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), ctrl, rows, 0xF, false))
    SLIMDP_ADD_DPP(0x111, 0xF);
    SLIMDP_ADD_DPP(0x112, 0xF);
    SLIMDP_ADD_DPP(0x114, 0xF);
    SLIMDP_ADD_DPP(0x118, 0xF);
    SLIMDP_ADD_DPP(0x142, 0xA);
    SLIMDP_ADD_DPP(0x143, 0xC);
#undef SLIMDP_ADD_DPP
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}
__device__ __forceinline__ float wave_max_f(float v)
{
    const int low = __float_as_int(-__builtin_inff());
#define SLIMDP_MAX_DPP(ctrl, rows) v = fmaxf(v, __int_as_float(__builtin_amdgcn_update_dpp(low, __float_as_int(v), ctrl, rows, 0xF, false)))
    SLIMDP_MAX_DPP(0x111, 0xF);
    SLIMDP_MAX_DPP(0x112, 0xF);
    SLIMDP_MAX_DPP(0x114, 0xF);
    SLIMDP_MAX_DPP(0x118, 0xF);
    SLIMDP_MAX_DPP(0x142, 0xA);
    SLIMDP_MAX_DPP(0x143, 0xC);
#undef SLIMDP_MAX_DPP
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}

// Sum over groups of G lanes (up to a wave), or over a block of G threads (slots: G / 64 words of shared memory that no one reads
// any more; every thread of the block must call).
template <int G> __device__ __forceinline__ float group_sum(float v, float* slots)
{
    if constexpr (G < 64) {
#pragma unroll
        for (int m = G / 2; m; m >>= 1) v += __shfl_xor(v, m);
        return v;
    } else if constexpr (G == 64) {
        return wave_sum_f(v);
    } else {
        v = wave_sum_f(v);
        if ((threadIdx.x & 63u) == 0) slots[threadIdx.x >> 6] = v;
        __syncthreads();
        float s = slots[0];
#pragma unroll
        for (int w = 1; w < G / 64; ++w) s += slots[w];
        return s;
    }
}

}  // namespace slimdp
