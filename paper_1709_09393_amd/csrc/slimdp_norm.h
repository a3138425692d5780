// Layer norm of every worker's rows and its backward pass; gradient of the product's epilogue; the sums over rows that all
// parameter vectors' gradients are.  Included only by slimdp_train.hip.
#pragma once
#include "slimdp_act.h"
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
// squared distances from the finished mean (no cancellation, whatever the mean).  All sums in binary32.  Bound by memory: a block takes
// several rows and asks for the next one before it sums the present one; weight and bias stay in registers where they are few (KEEP).
// grid (blocks, workers); groups of TPR threads take rows in turn.
template <class T, int TPR, int NC, int NT>
__global__ __launch_bounds__(TPR > 256 ? TPR : 256) void k_norm(NormArgs a)
{
    constexpr int BT = TPR > 256 ? TPR : 256, GROUPS = BT / TPR, V = Vec<T>::N;
    constexpr bool KEEP = NC * V <= 16, AHEAD = NC < 8;
    __shared__ float slots[2][BT / 64];
    const uint32_t q = blockIdx.y, rows = a.rows.n[q], cols = a.cols;
    const uint32_t lane = threadIdx.x % TPR, group = threadIdx.x / TPR, step = gridDim.x * GROUPS;
    const T* x = static_cast<const T*>(a.x.p[q]);
    T* y = static_cast<T*>(a.y.p[q]);
    const float* weight = static_cast<const float*>(a.weight.p[q]);
    const float* bias = static_cast<const float*>(a.bias.p[q]);
    float* mean_out = static_cast<float*>(a.mean.p[q]);
    float* rstd_out = static_cast<float*>(a.rstd.p[q]);
    const float count = (float)cols;
    // whole vectors, and behind the last of them one element a lane
    const uint32_t main = cols / V * V, last = main + lane;
    const bool has_last = last < cols;
    auto column = [&](int j) { return ((uint32_t)j * TPR + lane) * V; };
    auto params = [&](int j, float (&g)[V], float (&b)[V]) {
#pragma unroll
        for (int i = 0; i < V; ++i) { g[i] = 1.0f; b[i] = 0.0f; }
        if (weight) load_whole<V>(weight + column(j), g);
        if (bias) load_whole<V>(bias + column(j), b);
    };
    float kg[KEEP ? NC : 1][V], kb[KEEP ? NC : 1][V];
    if constexpr (KEEP)
#pragma unroll
        for (int j = 0; j < NC; ++j)
            if (column(j) < main) params(j, kg[j], kb[j]);
    const float last_g = has_last && weight ? weight[last] : 1.0f, last_b = has_last && bias ? bias[last] : 0.0f;
    raw4 now[NC], next[AHEAD ? NC : 1];
    float now_last = 0.0f, next_last = 0.0f;
#pragma unroll
    for (int j = 0; j < NC; ++j) now[j] = raw4{0, 0, 0, 0};          // columns behind the row's end stay zero
    if constexpr (AHEAD)
#pragma unroll
        for (int j = 0; j < NC; ++j) next[j] = raw4{0, 0, 0, 0};
    auto load_row = [&](uint32_t r, auto& v, float& l) {
        if (r >= rows) return;
        const T* xr = x + (size_t)r * a.ldx;
#pragma unroll
        for (int j = 0; j < NC; ++j)
            if (column(j) < main) v[j] = load_raw<T, NT>(xr + column(j));
        if (has_last) l = (float)xr[last];
    };
    uint32_t r = blockIdx.x * GROUPS + group;
    if constexpr (AHEAD) load_row(r, next, next_last);
    for (; r < rows; r += step) {
        if constexpr (AHEAD) {
#pragma unroll
            for (int j = 0; j < NC; ++j) now[j] = next[j];
            now_last = next_last;
            load_row(r + step, next, next_last);
        } else load_row(r, now, now_last);
        float s = now_last;
#pragma unroll
        for (int j = 0; j < NC; ++j) {
            float f[V];
            unpack<T>(now[j], f);
#pragma unroll
            for (int i = 0; i < V; ++i) s += f[i];
        }
        const float mean = group_sum<TPR>(s, slots[0]) / count;
        s = has_last ? (now_last - mean) * (now_last - mean) : 0.0f;
#pragma unroll
        for (int j = 0; j < NC; ++j) {
            if (column(j) >= main) continue;
            float f[V];
            unpack<T>(now[j], f);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float d = f[i] - mean;
                s = __builtin_fmaf(d, d, s);
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
            if (column(j) >= main) continue;
            float f[V], g[V], b[V];
            unpack<T>(now[j], f);
            if constexpr (KEEP) {
#pragma unroll
                for (int i = 0; i < V; ++i) { g[i] = kg[j][i]; b[i] = kb[j][i]; }
            } else params(j, g, b);
#pragma unroll
            for (int i = 0; i < V; ++i) f[i] = __builtin_fmaf((f[i] - mean) * rstd, g[i], b[i]);
            store_raw<T, NT>(yr + column(j), pack<T>(f));
        }
        if (has_last) yr[last] = (T)__builtin_fmaf((now_last - mean) * rstd, last_g, last_b);
        // the next row's first sum goes to slots that all have read before this row's second one was whole, and so on
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

// The same with the gradients of weight and bias in the same pass: TPR threads hold a row (NC vectors each) and add dy * xh and dy of
// their columns up over all the rows they meet, so that either input is read once.  BT / TPR groups of a block take rows in turn; at the
// end their sums meet in the LDS in the order of the groups, and the blocks' sums in k_column_sums in the order of the blocks (one block
// alone: here).  Which rows a group takes depends on the sizes alone.
// Bound by memory: the next row's vectors are under way while a row is summed.
// grid (blocks, workers)
struct NormBackSums {
    OutTab dweight, dbias;
    float* partial;              // [worker][block][2][cols], of blocks that have rows; nullptr: one block a worker
    int accumulate;
};
template <class T, int TPR, int NC, int BT, int NT>
__global__ __launch_bounds__(BT) void k_norm_back(NormBackArgs a, NormBackSums o)
{
    constexpr int V = Vec<T>::N, GROUPS = BT / TPR, IN_WAVE = TPR < 64 ? 64 / TPR : 1, ROUNDS = GROUPS / IN_WAVE;
    constexpr int WIDTH = TPR * NC * V;
    __shared__ float slots[2][2][BT / 64];
    __shared__ float meet[ROUNDS > 1 ? 2 : 1][ROUNDS > 1 ? WIDTH + TPR : 1];      // the last TPR: the elements behind the vectors
    const uint32_t q = blockIdx.y, rows = a.rows.n[q], cols = a.cols;
    if (blockIdx.x * GROUPS >= rows && blockIdx.x) return;          // the whole block has no row; the first one of an empty worker writes zeros
    const uint32_t lane = threadIdx.x % TPR, group = threadIdx.x / TPR, step = gridDim.x * GROUPS;
    const T* dy = static_cast<const T*>(a.dy.p[q]);
    const T* x = static_cast<const T*>(a.x.p[q]);
    T* dx = static_cast<T*>(a.dx.p[q]);
    const float* weight = static_cast<const float*>(a.weight.p[q]);
    const float* means = static_cast<const float*>(a.mean.p[q]);
    const float* rstds = static_cast<const float*>(a.rstd.p[q]);
    const float count = (float)cols;
    // whole vectors, and behind the last of them one element a lane
    const uint32_t main = cols / V * V, last = main + lane;
    const bool has_last = last < cols;
    auto column = [&](int j) { return ((uint32_t)j * TPR + lane) * V; };
    float g[NC][V], sw[NC][V], sb[NC][V];
    const float last_g = has_last && weight ? weight[last] : 1.0f;
    float last_sw = 0.0f, last_sb = 0.0f;
#pragma unroll
    for (int j = 0; j < NC; ++j) {
#pragma unroll
        for (int i = 0; i < V; ++i) { g[j][i] = 1.0f; sw[j][i] = sb[j][i] = 0.0f; }
        if (weight && column(j) < main) load_whole<V>(weight + column(j), g[j]);
    }
    raw4 ny[NC], nx[NC];
#pragma unroll
    for (int j = 0; j < NC; ++j) ny[j] = nx[j] = raw4{0, 0, 0, 0};     // columns behind the row's end stay zero
    float nm = 0.0f, nr = 0.0f, last_ny = 0.0f, last_nx = 0.0f;
    auto load_row = [&](uint32_t r) {
        if (r >= rows) return;
        nm = means[r];
        nr = rstds[r];
        const T *yr = dy + (size_t)r * a.lddy, *xr = x + (size_t)r * a.ldx;
#pragma unroll
        for (int j = 0; j < NC; ++j)
            if (column(j) < main) {
                ny[j] = load_raw<T, NT>(yr + column(j));
                nx[j] = load_raw<T, NT>(xr + column(j));
            }
        if (has_last) {
            last_ny = (float)yr[last];
            last_nx = (float)xr[last];
        }
    };
    uint32_t r = blockIdx.x * GROUPS + group, turn = 0;
    load_row(r);
    // a block's groups go through the same number of turns: the sums of a row of more than one wave wait for the whole block
    for (uint32_t first = blockIdx.x * GROUPS; first < rows; first += step, r += step, turn ^= 1u) {
        raw4 py[NC], px[NC];
        const float mean = nm, rstd = nr, last_py = last_ny, last_px = last_nx;
#pragma unroll
        for (int j = 0; j < NC; ++j) { py[j] = ny[j]; px[j] = nx[j]; }
        load_row(r + step);
        float s1 = 0.0f, s2 = 0.0f;
        if (r < rows) {                          // a turn without a row adds nothing
#pragma unroll
            for (int j = 0; j < NC; ++j) {
                if (column(j) >= main) continue;
                float f[V], xh[V];
                unpack<T>(py[j], f);
                unpack<T>(px[j], xh);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    xh[i] = (xh[i] - mean) * rstd;
                    sw[j][i] = __builtin_fmaf(f[i], xh[i], sw[j][i]);
                    sb[j][i] += f[i];
                    const float av = f[i] * g[j][i];
                    s1 += av;
                    s2 = __builtin_fmaf(av, xh[i], s2);
                }
            }
            if (has_last) {
                const float xh = (last_px - mean) * rstd, av = last_py * last_g;
                last_sw = __builtin_fmaf(last_py, xh, last_sw);
                last_sb += last_py;
                s1 += av;
                s2 = __builtin_fmaf(av, xh, s2);
            }
        }
        if (!dx) continue;
        if constexpr (TPR <= 64) {
            s1 = group_sum<TPR>(s1, nullptr) / count;
            s2 = group_sum<TPR>(s2, nullptr) / count;
        } else {
            constexpr int W = TPR / 64;
            s1 = wave_sum_f(s1);
            s2 = wave_sum_f(s2);
            float* slot1 = slots[turn][0];
            float* slot2 = slots[turn][1];
            if ((threadIdx.x & 63u) == 0) {
                slot1[threadIdx.x >> 6] = s1;
                slot2[threadIdx.x >> 6] = s2;
            }
            __syncthreads();                     // two turns' slots: nobody is two turns ahead of a reader
            s1 = slot1[group * W];
            s2 = slot2[group * W];
#pragma unroll
            for (int w = 1; w < W; ++w) {
                s1 += slot1[group * W + w];
                s2 += slot2[group * W + w];
            }
            s1 /= count;
            s2 /= count;
        }
        if (r >= rows) continue;
        T* dxr = dx + (size_t)r * a.lddx;
#pragma unroll
        for (int j = 0; j < NC; ++j) {
            if (column(j) >= main) continue;
            float f[V], xh[V];
            unpack<T>(py[j], f);
            unpack<T>(px[j], xh);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                xh[i] = (xh[i] - mean) * rstd;
                f[i] = rstd * (__builtin_fmaf(f[i], g[j][i], -s1) - xh[i] * s2);
            }
            store_raw<T, NT>(dxr + column(j), pack<T>(f));
        }
        if (has_last) dxr[last] = (T)(rstd * (__builtin_fmaf(last_py, last_g, -s1) - (last_px - mean) * rstd * s2));
    }
    float* outw = static_cast<float*>(o.dweight.p[q]);
    float* outb = static_cast<float*>(o.dbias.p[q]);
    const bool want = o.partial || outw || outb;
    if (!want) return;
    // groups of one wave first, by exchanges between lanes
#pragma unroll
    for (int m = 32; m >= TPR && TPR < 64; m >>= 1)
#pragma unroll
        for (int j = 0; j < NC; ++j)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                sw[j][i] += __shfl_xor(sw[j][i], m);
                sb[j][i] += __shfl_xor(sb[j][i], m);
            }
#pragma unroll
    for (int m = 32; m >= TPR && TPR < 64; m >>= 1) {
        last_sw += __shfl_xor(last_sw, m);
        last_sb += __shfl_xor(last_sb, m);
    }
    const uint32_t round = group / IN_WAVE;
    const bool lead = group % IN_WAVE == 0;
    if constexpr (ROUNDS > 1) {
        for (uint32_t g0 = 1; g0 < ROUNDS; ++g0) {
            __syncthreads();
            if (round == g0 && lead) {
#pragma unroll
                for (int j = 0; j < NC; ++j)
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        meet[0][(j * V + i) * TPR + lane] = sw[j][i];
                        meet[1][(j * V + i) * TPR + lane] = sb[j][i];
                    }
                meet[0][WIDTH + lane] = last_sw;
                meet[1][WIDTH + lane] = last_sb;
            }
            __syncthreads();
            if (round == 0 && lead) {
#pragma unroll
                for (int j = 0; j < NC; ++j)
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        sw[j][i] += meet[0][(j * V + i) * TPR + lane];
                        sb[j][i] += meet[1][(j * V + i) * TPR + lane];
                    }
                last_sw += meet[0][WIDTH + lane];
                last_sb += meet[1][WIDTH + lane];
            }
        }
    }
    if (round != 0 || !lead) return;
    if (o.partial) {
        outw = o.partial + ((size_t)q * gridDim.x + blockIdx.x) * 2 * cols;
        outb = outw + cols;
    }
    const bool add = !o.partial && o.accumulate;
    auto put = [&](float* out, auto& v, float l) {
        if (!out) return;
#pragma unroll
        for (int j = 0; j < NC; ++j) {
            if (column(j) >= main) continue;
            if (add) {
                float old[V];
                load_whole<V>(out + column(j), old);
#pragma unroll
                for (int i = 0; i < V; ++i) v[j][i] += old[i];
            }
#pragma unroll
            for (int i = 0; i < V; i += 4)
                store_raw<float>(out + column(j) + i, raw4{__float_as_uint(v[j][i]), __float_as_uint(v[j][i + 1]), __float_as_uint(v[j][i + 2]),
                                                           __float_as_uint(v[j][i + 3])});
        }
        if (has_last) out[last] = add ? out[last] + l : l;
    };
    put(outw, sw, last_sw);
    put(outb, sb, last_sb);
}

// ---------------------------------------------------------------------------------------
// Sums over rows.  A block owns up to 64 vectors of consecutive columns (LX, as many as narrow matrices have) and a slab of consecutive
// rows, its 256 / LX groups of threads every so many rows of it;
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

// NT: streams pass the caches by.  NORM: out0 = sum dy * xh, out1 = sum dy.  Otherwise dz = dy * act'(z) and out1 = sum dz, from the values before they are rounded.
template <class T, bool NORM, int ACT, int LX, int NT>
__global__ __launch_bounds__(256) void k_column_grads(ColumnArgs a)
{
    constexpr int V = Vec<T>::N, ARR = NORM ? 2 : 1;
    constexpr uint32_t GROUPS = 256 / LX;
    __shared__ float part[ARR][V][256];
    const uint32_t q = blockIdx.z, rows = a.rows.n[q], cols = a.cols;
    const uint32_t lane = threadIdx.x % LX, group = threadIdx.x / LX;
    const uint32_t c = (blockIdx.x * LX + lane) * V, slab = blockIdx.y;
    const uint32_t r0 = slab * a.slab;
    if (r0 >= rows && slab) return;              // the whole block; the first slab of an empty worker writes zeros
    const uint32_t r1 = min(rows, r0 + a.slab);
    const T* pa = static_cast<const T*>(a.a.p[q]);
    const T* pb = static_cast<const T*>(a.b.p[q]);
    T* dz = static_cast<T*>(a.dz.p[q]);
    float s0[V], s1[V];
#pragma unroll
    for (int i = 0; i < V; ++i) s0[i] = s1[i] = 0.0f;
    auto one = [&](uint32_t r, raw4 va, raw4 vb) {
        float f[V], g[V];
        unpack<T>(va, f);
        if (NORM) {
            const float mean = static_cast<const float*>(a.mean.p[q])[r], rstd = static_cast<const float*>(a.rstd.p[q])[r];
            unpack<T>(vb, g);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                s0[i] = __builtin_fmaf(f[i], (g[i] - mean) * rstd, s0[i]);
                s1[i] += f[i];
            }
        } else {
            if constexpr (ACT != ACT_NONE) {
                unpack<T>(vb, g);
#pragma unroll
                for (int i = 0; i < V; ++i) f[i] *= act_slope<ACT>(g[i]);
            }
            if (dz) store_clip<T, NT>(dz + (size_t)r * a.lddz, c, cols, pack<T>(f));
#pragma unroll
            for (int i = 0; i < V; ++i) s1[i] += f[i];
        }
    };
    constexpr bool TWO = NORM || ACT != ACT_NONE;
    if (c < cols) {
        uint32_t r = r0 + group;
        for (; r + GROUPS < r1; r += 2 * GROUPS) {             // two rows' vectors under way at a time
            const raw4 a0 = load_clip<T, NT>(pa + (size_t)r * a.lda, c, cols), a1 = load_clip<T, NT>(pa + (size_t)(r + GROUPS) * a.lda, c, cols);
            const raw4 b0 = TWO ? load_clip<T, NT>(pb + (size_t)r * a.ldb, c, cols) : a0;
            const raw4 b1 = TWO ? load_clip<T, NT>(pb + (size_t)(r + GROUPS) * a.ldb, c, cols) : a1;
            one(r, a0, b0);
            one(r + GROUPS, a1, b1);
        }
        if (r < r1) {
            const raw4 a0 = load_clip<T, NT>(pa + (size_t)r * a.lda, c, cols);
            one(r, a0, TWO ? load_clip<T, NT>(pb + (size_t)r * a.ldb, c, cols) : a0);
        }
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
        if (NORM) part[ARR - 1][i][threadIdx.x] = s0[i];
        part[0][i][threadIdx.x] = s1[i];
    }
    __syncthreads();
    if (group == 0 && c < cols) {
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
            for (uint32_t g = 1; g < GROUPS; ++g) {
                if (NORM) s0[i] += part[ARR - 1][i][g * LX + lane];
                s1[i] += part[0][i][g * LX + lane];
            }
            if (NORM && p0) p0[c + i] = add ? p0[c + i] + s0[i] : s0[i];
            if (p1) p1[c + i] = add ? p1[c + i] + s1[i] : s1[i];
        }
    }
}

// The slabs' sums of column c: SL threads a column (16, or 64 of many slabs) take every SL-th slab, eight asked for at a time; their sums meet
// eight and eight.  The order goes by the number of slabs alone.  (With sixteen threads and one slab at a time the 1,024 slabs of 16,384 rows took as long as the rows.)
struct ColumnSumArgs {
    const float* partial;
    OutTab out0, out1;
    RowTab rows;
    uint32_t cols, slab, slabs, arrays;   // a worker has as many slabs as it has times `slab` rows, `slabs` at most
    int accumulate;
};
template <uint32_t SL>
__global__ __launch_bounds__(16 * SL) void k_column_sums(ColumnSumArgs a)
{
    __shared__ float part[SL][17];
    const uint32_t q = blockIdx.z, arr = blockIdx.y, tx = threadIdx.x & 15u, ty = threadIdx.x >> 4;
    const uint32_t c = blockIdx.x * 16 + tx;
    const uint32_t n = min(a.slabs, max(1u, (a.rows.n[q] + a.slab - 1) / a.slab));
    const float* from = a.partial + ((size_t)q * a.slabs * a.arrays + arr) * a.cols + c;
    const size_t step = (size_t)a.arrays * a.cols;
    float s = 0.0f;
    if (c < a.cols)
        for (uint32_t p = ty; p < n; p += 8 * SL) {
            float v[8];
#pragma unroll
            for (uint32_t i = 0; i < 8; ++i) v[i] = p + SL * i < n ? from[(p + SL * i) * step] : 0.0f;
#pragma unroll
            for (uint32_t i = 0; i < 8; ++i) s += v[i];
        }
    part[ty][tx] = s;
    __syncthreads();
    if (ty < 8) {
#pragma unroll
        for (uint32_t i = 1; i < SL / 8; ++i) s += part[ty + 8 * i][tx];
    }
    __syncthreads();
    if (ty < 8) part[ty][tx] = s;
    __syncthreads();
    if (ty == 0 && c < a.cols) {
        float* out = static_cast<float*>(arr == 0 && a.arrays == 2 ? a.out0.p[q] : a.out1.p[q]);
        if (!out) return;
#pragma unroll
        for (uint32_t i = 1; i < 8; ++i) s += part[i][tx];
        out[c] = a.accumulate ? out[c] + s : s;
    }
}

}  // namespace slimdp
