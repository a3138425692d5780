// Layer norm of every worker's rows and its backward pass; gradient of the product's epilogue; the sums over rows that all
// parameter vectors' gradients are.  Included only by slimdp_train.hip.
#pragma once
#include "slimdp_train.h"

namespace slimdp {

struct NormArgs {
    InTab x, weight, bias;
    OutTab y, mean, rstd;
    RowTab rows;
    uint64_t ldx, ldy;
    uint32_t cols;
    float eps;
};

// y = (x - mean) * rstd * weight + bias, mean and rstd = 1 / sqrt(var + eps) over the row, var the mean of (x - mean)^2.
// TPR threads hold a row in registers, NC vectors of sixteen bytes each: the row is read once, and the variance is the sum of
// squared distances from the finished mean (no cancellation, whatever the mean).  All sums in binary32.
// grid (blocks, workers); groups of TPR threads take rows in turn.
template <class T, int TPR, int NC>
__global__ __launch_bounds__(TPR > 256 ? TPR : 256) void k_norm(NormArgs a)
{
    constexpr int BT = TPR > 256 ? TPR : 256, GROUPS = BT / TPR, V = Vec<T>::N;
    __shared__ float slots[2][BT / 64];
    const uint32_t q = blockIdx.y, rows = a.rows.n[q], cols = a.cols;
    const uint32_t lane = threadIdx.x % TPR, group = threadIdx.x / TPR;
    const T* x = static_cast<const T*>(a.x.p[q]);
    T* y = static_cast<T*>(a.y.p[q]);
    const float* weight = static_cast<const float*>(a.weight.p[q]);
    const float* bias = static_cast<const float*>(a.bias.p[q]);
    float* mean_out = static_cast<float*>(a.mean.p[q]);
    float* rstd_out = static_cast<float*>(a.rstd.p[q]);
    const float count = (float)cols;
    for (uint32_t r = blockIdx.x * GROUPS + group; r < rows; r += gridDim.x * GROUPS) {
        const T* xr = x + (size_t)r * a.ldx;
        float f[NC][V], s = 0.0f;
#pragma unroll
        for (int j = 0; j < NC; ++j) {
            const uint32_t c = ((uint32_t)j * TPR + lane) * V;
            if (c < cols) unpack<T>(load_clip(xr, c, cols), f[j]);
            else {
#pragma unroll
                for (int i = 0; i < V; ++i) f[j][i] = 0.0f;
            }
#pragma unroll
            for (int i = 0; i < V; ++i) s += f[j][i];
        }
        const float mean = group_sum<TPR>(s, slots[0]) / count;
        s = 0.0f;
#pragma unroll
        for (int j = 0; j < NC; ++j) {
            const uint32_t c = ((uint32_t)j * TPR + lane) * V;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                f[j][i] = c + i < cols ? f[j][i] - mean : 0.0f;
                s = __builtin_fmaf(f[j][i], f[j][i], s);
            }
        }
        const float var = group_sum<TPR>(s, slots[1]) / count;
        const float rstd = 1.0f / sqrtf(var + a.eps);
        if (lane == 0) {
            if (mean_out) mean_out[r] = mean;
            if (rstd_out) rstd_out[r] = rstd;
        }
        T* yr = y + (size_t)r * a.ldy;
#pragma unroll
        for (int j = 0; j < NC; ++j) {
            const uint32_t c = ((uint32_t)j * TPR + lane) * V;
            if (c < cols) {
                float g[V], b[V];
                if (weight) load_params<V>(weight, c, cols, g);
                if (bias) load_params<V>(bias, c, cols, b);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    f[j][i] *= rstd;
                    if (weight) f[j][i] *= g[i];
                    if (bias) f[j][i] += b[i];
                }
                store_clip(yr, c, cols, pack<T>(f[j]));
            }
        }
        if (TPR > 64) __syncthreads();           // the next row's sums go to the same slots
    }
}

struct NormBackArgs {
    InTab dy, x, weight, mean, rstd;
    OutTab dx;
    RowTab rows;
    uint64_t lddy, ldx, lddx;
    uint32_t cols;
};

// dx = rstd * (a - mean(a) - xh * mean(a * xh)),  a = weight * dy,  xh = (x - mean) * rstd.
// One block of 256 threads a row, which is read twice (the second time from the caches).
template <class T>
__global__ __launch_bounds__(256) void k_norm_back_rows(NormBackArgs a)
{
    constexpr int V = Vec<T>::N;
    __shared__ float slots[2][4];
    const uint32_t q = blockIdx.y, rows = a.rows.n[q], cols = a.cols;
    const T* dy = static_cast<const T*>(a.dy.p[q]);
    const T* x = static_cast<const T*>(a.x.p[q]);
    T* dx = static_cast<T*>(a.dx.p[q]);
    const float* weight = static_cast<const float*>(a.weight.p[q]);
    const float count = (float)cols;
    for (uint32_t r = blockIdx.x; r < rows; r += gridDim.x) {
        const float mean = static_cast<const float*>(a.mean.p[q])[r], rstd = static_cast<const float*>(a.rstd.p[q])[r];
        const T *dyr = dy + (size_t)r * a.lddy, *xr = x + (size_t)r * a.ldx;
        T* dxr = dx + (size_t)r * a.lddx;
        auto values = [&](uint32_t c, float av[V], float xh[V]) {
            float g[V];
            unpack<T>(load_clip(dyr, c, cols), av);
            unpack<T>(load_clip(xr, c, cols), xh);
            if (weight) load_params<V>(weight, c, cols, g);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                if (weight) av[i] *= g[i];
                xh[i] = (xh[i] - mean) * rstd;
            }
        };
        float s1 = 0.0f, s2 = 0.0f;
        for (uint32_t c = threadIdx.x * V; c < cols; c += 256 * V) {
            float av[V], xh[V];
            values(c, av, xh);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                s1 += av[i];
                s2 = __builtin_fmaf(av[i], xh[i], s2);
            }
        }
        s1 = group_sum<256>(s1, slots[0]) / count;
        s2 = group_sum<256>(s2, slots[1]) / count;
        for (uint32_t c = threadIdx.x * V; c < cols; c += 256 * V) {
            float av[V], xh[V];
            values(c, av, xh);
#pragma unroll
            for (int i = 0; i < V; ++i) av[i] = rstd * (av[i] - s1 - xh[i] * s2);
            store_clip(dxr, c, cols, pack<T>(av));
        }
        __syncthreads();
    }
}

// ---------------------------------------------------------------------------------------
// Sums over rows.  A block owns 64 vectors of consecutive columns and a slab of consecutive rows, its four waves every fourth row of it;
// the slabs' partial sums meet in k_column_sums.  Which rows a slab holds depends on the sizes alone and every sum has a
// fixed order: the same bits every time.
// ---------------------------------------------------------------------------------------
struct ColumnArgs {
    InTab a, b, mean, rstd;          // norm: dy, x;  epilogue: dy, z
    OutTab dz, out0, out1;           // norm: out0 = gradient of the weight, out1 of the bias;  epilogue: out1 = gradient of the bias
    RowTab rows;
    uint64_t lda, ldb, lddz;
    uint32_t cols, slab;             // rows of a slab
    float* partial;                  // [worker][slab][array][cols]; nullptr: one slab, results go out at once
    uint32_t slabs;                  // ... of the worker that has most
    int accumulate;
};

enum : int { ACT_NONE = 0, ACT_RELU = 1, ACT_GELU = 2, ACT_GELU_TANH = 3, ACT_SILU = 4, ACTS = 5 };

// Slope and value of the activation in binary32.  exp of a large argument is infinite and its reciprocal zero, so that no case is left out;
// where such a zero would meet an infinite z the factor z is held finite (comparisons let a NaN through).
__device__ __forceinline__ float act_slope(float z, int act)
{
    const float zz = z < -1000.0f ? -1000.0f : (z > 1000.0f ? 1000.0f : z);
    switch (act) {
    case ACT_RELU: return z > 0.0f ? 1.0f : 0.0f;
    case ACT_GELU: return 0.5f * erfcf(zz * -0.70710678118654752f) + zz * expf(-0.5f * zz * zz) * 0.39894228040143268f;
    case ACT_GELU_TANH: {
        // 0.5 (1 + tanh u) = 1 / (1 + exp(-2 u)) =: s, its slope in u 2 s (1 - s)
        const float u2 = 1.5957691216057308f * (zz + 0.044715f * zz * zz * zz);
        const float s = 1.0f / (1.0f + expf(-u2)), t = 1.0f / (1.0f + expf(u2));
        return s + zz * s * t * 1.5957691216057308f * (1.0f + 0.134145f * zz * zz);
    }
    case ACT_SILU: {
        const float s = 1.0f / (1.0f + expf(-zz)), t = 1.0f / (1.0f + expf(zz));
        return s + zz * s * t;
    }
    default: return 1.0f;
    }
}
__device__ __forceinline__ float act_value(float z, int act)
{
    const float zz = z < -1000.0f ? -1000.0f : z;
    switch (act) {
    case ACT_RELU: return z < 0.0f ? 0.0f : z;
    case ACT_GELU: return 0.5f * zz * erfcf(zz * -0.70710678118654752f);
    case ACT_GELU_TANH: return zz / (1.0f + expf(-1.5957691216057308f * (zz + 0.044715f * zz * zz * zz)));
    case ACT_SILU: return zz / (1.0f + expf(-zz));
    default: return z;
    }
}

// The same for several values: one choice for all of them.
template <int N> __device__ __forceinline__ void act_values(float (&v)[N], int act)
{
    auto all = [&](auto f) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = f(v[i]);
    };
    switch (act) {
    case ACT_RELU: all([](float z) { return act_value(z, ACT_RELU); }); break;
    case ACT_GELU: all([](float z) { return act_value(z, ACT_GELU); }); break;
    case ACT_GELU_TANH: all([](float z) { return act_value(z, ACT_GELU_TANH); }); break;
    case ACT_SILU: all([](float z) { return act_value(z, ACT_SILU); }); break;
    default: break;
    }
}

// NORM: out0 = sum dy * xh, out1 = sum dy.  Otherwise dz = dy * act'(z) and out1 = sum dz, from the values before they are rounded.
template <class T, bool NORM>
__global__ __launch_bounds__(256) void k_column_grads(ColumnArgs a, int act)
{
    constexpr int V = Vec<T>::N, ARR = NORM ? 2 : 1;
    __shared__ float part[3][ARR][V][64];
    const uint32_t q = blockIdx.z, rows = a.rows.n[q], cols = a.cols;
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
    const uint32_t c = (blockIdx.x * 64 + lane) * V, slab = blockIdx.y;
    const uint32_t r0 = slab * a.slab;
    if (r0 >= rows && slab) return;              // the whole block; the first slab of an empty worker writes zeros
    const uint32_t r1 = min(rows, r0 + a.slab);
    const T* pa = static_cast<const T*>(a.a.p[q]);
    const T* pb = static_cast<const T*>(a.b.p[q]);
    T* dz = static_cast<T*>(a.dz.p[q]);
    float s0[V], s1[V];
#pragma unroll
    for (int i = 0; i < V; ++i) s0[i] = s1[i] = 0.0f;
    if (c < cols)
        for (uint32_t r = r0 + wave; r < r1; r += 4) {
            float f[V], g[V];
            unpack<T>(load_clip(pa + (size_t)r * a.lda, c, cols), f);
            if (NORM) {
                const float mean = static_cast<const float*>(a.mean.p[q])[r], rstd = static_cast<const float*>(a.rstd.p[q])[r];
                unpack<T>(load_clip(pb + (size_t)r * a.ldb, c, cols), g);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    s0[i] = __builtin_fmaf(f[i], (g[i] - mean) * rstd, s0[i]);
                    s1[i] += f[i];
                }
            } else {
                if (act != ACT_NONE) {
                    unpack<T>(load_clip(pb + (size_t)r * a.ldb, c, cols), g);
#pragma unroll
                    for (int i = 0; i < V; ++i) f[i] *= act_slope(g[i], act);
                }
                if (dz) store_clip(dz + (size_t)r * a.lddz, c, cols, pack<T>(f));
#pragma unroll
                for (int i = 0; i < V; ++i) s1[i] += f[i];
            }
        }
    if (wave) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            if (NORM) part[wave - 1][ARR - 1][i][lane] = s0[i];
            part[wave - 1][0][i][lane] = s1[i];
        }
    }
    __syncthreads();
    if (wave == 0 && c < cols) {
        float* p0 = NORM ? static_cast<float*>(a.out0.p[q]) : nullptr;
        float* p1 = static_cast<float*>(a.out1.p[q]);
        if (a.partial) {
            p1 = a.partial + ((size_t)q * a.slabs + slab) * ARR * cols;
            if (NORM) { p0 = p1; p1 = p0 + cols; }
        }
        const bool add = !a.partial && a.accumulate;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            if (c + i >= cols) break;
#pragma unroll
            for (int w = 0; w < 3; ++w) {
                if (NORM) s0[i] += part[w][ARR - 1][i][lane];
                s1[i] += part[w][0][i][lane];
            }
            if (NORM && p0) p0[c + i] = add ? p0[c + i] + s0[i] : s0[i];
            if (p1) p1[c + i] = add ? p1[c + i] + s1[i] : s1[i];
        }
    }
}

// The slabs' sums of column c, added in the order of the slabs: sixteen threads a column take every sixteenth slab, then their sums in order.
struct ColumnSumArgs {
    const float* partial;
    OutTab out0, out1;
    RowTab rows;
    uint32_t cols, slab, slabs, arrays;
    int accumulate;
};
__global__ __launch_bounds__(256) void k_column_sums(ColumnSumArgs a)
{
    __shared__ float part[16][17];
    const uint32_t q = blockIdx.z, arr = blockIdx.y, tx = threadIdx.x & 15u, ty = threadIdx.x >> 4;
    const uint32_t c = blockIdx.x * 16 + tx;
    const uint32_t n = max(1u, (a.rows.n[q] + a.slab - 1) / a.slab);
    float s = 0.0f;
    if (c < a.cols)
        for (uint32_t p = ty; p < n; p += 16) s += a.partial[(((size_t)q * a.slabs + p) * a.arrays + arr) * a.cols + c];
    part[ty][tx] = s;
    __syncthreads();
    if (ty == 0 && c < a.cols) {
        float* out = static_cast<float*>(arr == 0 && a.arrays == 2 ? a.out0.p[q] : a.out1.p[q]);
        if (!out) return;
        for (int p = 1; p < 16; ++p) s += part[p][tx];
        out[c] = a.accumulate ? out[c] + s : s;
    }
}

}  // namespace slimdp
