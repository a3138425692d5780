// Matrix products of the worker side: x W^T with bias, activation and residual in the epilogue, and the two products that are its
// gradients.  Included only by slimdp_train.hip.
#pragma once
#include <type_traits>

#include "slimdp_train.h"
#include "slimdp_norm.h"

namespace slimdp {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// C[m][n] = sum over k of A(m, k) B(n, k) for every worker.  An operand lies either with k running (rows of m or n) or with m or n
// running (rows of k: KROWS).
struct GemmArgs {
    InTab a, b, bias, residual;
    OutTab c, z;
    RowTab rows;                 // per worker: M, or with k_is_rows the length of the sum
    uint32_t M, N, K;            // the largest of the workers where it varies
    int k_is_rows;
    uint64_t lda, ldb, ldc, ldr, ldz;
    uint32_t splits, k_split;    // the sum in pieces of k_split (a multiple of the step), one block each
    float* partial;              // [worker][split][M][N] where splits > 1
    int act, accumulate;
    uint32_t blocks;             // of all workers (kernels that number only the blocks that have work)
    uint32_t each;               // of every worker, where all have the same number; otherwise 0, and ...
    uint32_t first[MAXW_T + 1];  // ... of the workers before each, and of all
    int spread;                  // workers differ in what a block of theirs takes
};

// The worker that a block belongs to, its first block and the number of its blocks.  (Halving takes five loads one after the other, half a
// microsecond of a launch: only where the workers differ.)
struct Share { uint32_t q, begin, count; };
__device__ __forceinline__ Share share_of(const GemmArgs& a, uint32_t unit)
{
    if (a.each) {
        const uint32_t q = unit / a.each;
        return {q, q * a.each, a.each};
    }
    static_assert(MAXW_T == 32, "five halvings");
    uint32_t q = 0;
#pragma unroll
    for (uint32_t half = 16; half; half >>= 1)
        if (unit >= a.first[q + half]) q += half;
    return {q, a.first[q], a.first[q + 1] - a.first[q]};
}

// 16 bytes of either operand a lane: eight products' steps of sixteen-bit elements in one instruction, four of binary32 in one each.
template <class T> struct Mma;
template <> struct Mma<_Float16> {
    static constexpr int PARTS = 1;
    static __device__ __forceinline__ f32x4 part(raw4 a, raw4 b, f32x4 c, int)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    }
};
template <> struct Mma<__bf16> {
    static constexpr int PARTS = 1;
    static __device__ __forceinline__ f32x4 part(raw4 a, raw4 b, f32x4 c, int)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    }
};
template <> struct Mma<float> {
    // the four parts take the elements k, k + 4, k + 8, k + 12 of sixteen, the same ones of both operands
    static constexpr int PARTS = 4;
    static __device__ __forceinline__ f32x4 part(raw4 a, raw4 b, f32x4 c, int e)
    {
        return __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a[e]), __uint_as_float(b[e]), c, 0, 0, 0);
    }
};

// N by N elements, a vector of sixteen bytes a row, turned over.
template <class T> __device__ __forceinline__ void transpose(raw4 (&v)[Vec<T>::N])
{
    constexpr int N = Vec<T>::N;
    raw4 o[N];
    if constexpr (N == 4) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) o[i][j] = v[j][i];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                o[i][j] = __builtin_amdgcn_perm(v[2 * j + 1][i >> 1], v[2 * j][i >> 1], (i & 1) ? 0x07060302u : 0x05040100u);
    }
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = o[i];
}

// What becomes of four consecutive columns of one row of the sum.
//   EPI 0: z = sum + bias, c = act(z) + residual, both in T      EPI 1: c = sum in T      EPI 2: c = sum in binary32, or c + sum
template <class T> struct Four;
template <> struct Four<float> { typedef uint32_t any __attribute__((ext_vector_type(4), aligned(4))); };
template <> struct Four<_Float16> { typedef uint32_t any __attribute__((ext_vector_type(2), aligned(2))); };
template <> struct Four<__bf16> { typedef uint32_t any __attribute__((ext_vector_type(2), aligned(2))); };
template <class T> union FourPack { typename Four<T>::any r; T e[4]; };

// Four consecutive elements, `left` of them inside the row.
template <class T> __device__ __forceinline__ void load4(const T* p, uint32_t left, float f[4])
{
    if (left >= 4) {
        FourPack<T> v;
        v.r = *reinterpret_cast<const typename Four<T>::any*>(p);
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = (float)v.e[i];
    } else {
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) f[i] = i < left ? (float)p[i] : 0.0f;
    }
}
template <class T> __device__ __forceinline__ void store4(T* p, uint32_t left, const float f[4])
{
    if (left >= 4) {
        FourPack<T> v;
#pragma unroll
        for (int i = 0; i < 4; ++i) v.e[i] = (T)f[i];
        *reinterpret_cast<typename Four<T>::any*>(p) = v.r;
    } else {
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i)
            if (i < left) p[i] = (T)f[i];
    }
}

template <class T, int EPI>
__device__ __forceinline__ void epilogue4(const GemmArgs& a, uint32_t q, uint32_t m, uint32_t n, uint32_t N, const float s[4])
{
    const uint32_t left = N - n;
    float v[4] = {s[0], s[1], s[2], s[3]}, x[4];
    if constexpr (EPI == 2) {
        float* c = static_cast<float*>(a.c.p[q]) + (size_t)m * a.ldc + n;
        if (a.accumulate) {
            load4(c, left, x);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] += x[i];
        }
        store4(c, left, v);
    } else {
        if constexpr (EPI == 0) {
            const float* bias = static_cast<const float*>(a.bias.p[q]);
            T* z = static_cast<T*>(a.z.p[q]);
            const T* res = static_cast<const T*>(a.residual.p[q]);
            if (bias) {
                load4(bias + n, left, x);
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] += x[i];
            }
            if (z) store4(z + (size_t)m * a.ldz + n, left, v);
            act_values(v, a.act);
            if (res) {
                load4(res + (size_t)m * a.ldr + n, left, x);
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] += x[i];
            }
        }
        store4(static_cast<T*>(a.c.p[q]) + (size_t)m * a.ldc + n, left, v);
    }
}

// Rows shorter than a vector, and sixteen-bit operands whose distances do not fit the tile kernel's offsets: 64 x 64 of C a block of four
// waves, 128 bytes of k a step, element by element where a row breaks off.  In the LDS either operand lies with k running, 128 bytes a row,
// its eight vectors exchanged by the row's number so that the sixteen rows that a read touches meet different banks; operands with
// rows of k are turned over in registers on the way.  What lies outside reads as zero.
// grid (tiles, 1, workers * splits)
template <class T, bool AK, bool BK_, int EPI>
__global__ __launch_bounds__(256) void k_gemm(GemmArgs a)
{
    constexpr uint32_t V = Vec<T>::N, BK = 8 * V, S = 64, F = S / 32, RUN = S / 32;
    __shared__ raw4 sa[S * 8], sb[S * 8];
    const uint32_t q = blockIdx.z / a.splits, split = blockIdx.z % a.splits;
    const uint32_t M = a.k_is_rows ? a.M : a.rows.n[q], N = a.N, Kall = a.k_is_rows ? a.rows.n[q] : a.K;
    const uint32_t across = (N + S - 1) / S, m0 = blockIdx.x / across * S, n0 = blockIdx.x % across * S;
    if (m0 >= M) return;
    const uint32_t k0 = min(Kall, split * a.k_split), K = min(Kall, k0 + a.k_split);
    const T* A = static_cast<const T*>(a.a.p[q]);
    const T* B = static_cast<const T*>(a.b.p[q]);
    const uint32_t t = threadIdx.x, lane = t & 63u, wave = t >> 6, wm = wave >> 1, wn = wave & 1u;

    // one operand's pieces of a step: RUN vectors a thread with k running, one square of V x V elements otherwise
    constexpr uint32_t SQ = S / V * 8;                             // squares of a tile
    constexpr int RA = AK ? (int)V : (int)RUN, RB = BK_ ? (int)V : (int)RUN;
    raw4 ra[RA], rb[RB];
    auto load = [&](auto krows, const T* P, uint64_t ld, uint32_t x0, uint32_t X, uint32_t kb, uint32_t tt, auto& reg) {
        if constexpr (!decltype(krows)::value) {
#pragma unroll
            for (uint32_t i = 0; i < RUN; ++i) {
                const uint32_t x = x0 + (t >> 3) + 32u * i, k = kb + (t & 7u) * V;
                reg[i] = x < X && k < K ? load_clip(P + (size_t)x * ld, k, K) : raw4{0, 0, 0, 0};
            }
        } else {
            if (tt >= SQ) return;
            const uint32_t x = x0 + (tt >> 3) * V, kr = kb + (tt & 7u) * V;        // eight lanes: a whole row of the LDS to write
#pragma unroll
            for (uint32_t i = 0; i < V; ++i) reg[i] = x < X && kr + i < K ? load_clip(P + (size_t)(kr + i) * ld, x, X) : raw4{0, 0, 0, 0};
        }
    };
    auto put = [&](auto krows, raw4* s, uint32_t tt, auto& reg) {
        if constexpr (!decltype(krows)::value) {
#pragma unroll
            for (uint32_t i = 0; i < RUN; ++i) {
                const uint32_t x = (t >> 3) + 32u * i;
                s[x * 8 + ((t & 7u) ^ ((x >> 1) & 7u))] = reg[i];
            }
        } else if (tt < SQ) {
            const uint32_t x = (tt >> 3) * V, ck = tt & 7u;
            transpose<T>(reg);
#pragma unroll
            for (uint32_t i = 0; i < V; ++i) s[(x + i) * 8 + (ck ^ (((x + i) >> 1) & 7u))] = reg[i];
        }
    };
    typedef std::integral_constant<bool, AK> ak_t;
    typedef std::integral_constant<bool, BK_> bk_t;
    // where squares occupy part of the block, the second operand's go to another part
    const uint32_t ta = t, tb = SQ < 256 && AK ? (t + 128u) & 255u : t;
    f32x4 acc[F][F];
#pragma unroll
    for (uint32_t i = 0; i < F; ++i)
#pragma unroll
        for (uint32_t j = 0; j < F; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    auto load_step = [&](uint32_t kb) {
        load(ak_t{}, A, a.lda, m0, M, kb, ta, ra);
        load(bk_t{}, B, a.ldb, n0, N, kb, tb, rb);
    };
    if (k0 < K) load_step(k0);
    for (uint32_t kb = k0; kb < K; kb += BK) {
        __syncthreads();
        put(ak_t{}, sa, ta, ra);
        put(bk_t{}, sb, tb, rb);
        __syncthreads();
        if (kb + BK < K) load_step(kb + BK);
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            raw4 fa[F], fb[F];
            const uint32_t ch = ks * 4 + (lane >> 4);
#pragma unroll
            for (uint32_t i = 0; i < F; ++i) {
                const uint32_t xa = wm * (S / 2) + i * 16 + (lane & 15u), xb = wn * (S / 2) + i * 16 + (lane & 15u);
                fa[i] = sa[xa * 8 + (ch ^ ((xa >> 1) & 7u))];
                fb[i] = sb[xb * 8 + (ch ^ ((xb >> 1) & 7u))];
            }
            // B first: a lane then holds four consecutive columns of one row of C
#pragma unroll
            for (int e = 0; e < Mma<T>::PARTS; ++e)
#pragma unroll
                for (uint32_t i = 0; i < F; ++i)
#pragma unroll
                    for (uint32_t j = 0; j < F; ++j) acc[i][j] = Mma<T>::part(fb[j], fa[i], acc[i][j], e);
        }
    }
#pragma unroll
    for (uint32_t i = 0; i < F; ++i) {
        const uint32_t m = m0 + wm * (S / 2) + i * 16 + (lane & 15u);
        if (m >= M) continue;
#pragma unroll
        for (uint32_t j = 0; j < F; ++j) {
            const uint32_t n = n0 + wn * (S / 2) + j * 16 + (lane >> 4) * 4;
            if (n >= N) continue;
            const float s[4] = {acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]};
            if (a.splits == 1) epilogue4<T, EPI>(a, q, m, n, N, s);
            else store4(a.partial + (((size_t)q * a.splits + split) * a.M + m) * N + n, N - n, s);
        }
    }
}

// Few rows (up to 16 * MF) of sixteen-bit types: the second operand's bytes are most of what there is to wait for (every block reads all of the
// first from the caches, M / 16 times the bytes of its own rows).  It goes from memory to registers as the instructions
// take it (16 rows, four vectors of each at a time), every element once; a block has 16 of its rows and its eight waves a share of k
// each, whose sums meet in the LDS in the order of the waves.  A wave has four to eight steps' vectors under way,
// the number that leaves the fewest places empty in its share (four of 64 rows: more do not fit the registers), and asks for all of them
// without a condition, from a place inside the row: loads behind a condition each took 57 us instead of 40 at 8 x 50 x 1024 x 4096 bf16,
// 25.8 instead of 18.6 at 4 x 33 x 1000 x 4000.  4 x 8 x 8192 x 8192 bf16 122 us (4.4 TB/s).
// grid (ceil(N / 16), 1, workers)
template <class T, int MF, int EPI>
__global__ __launch_bounds__(512) void k_gemm_few(GemmArgs a)
{
    constexpr uint32_t V = Vec<T>::N, STEP = 4 * V;
    __shared__ f32x4 meet[8][MF][64];
    const uint32_t q = blockIdx.z, M = a.rows.n[q], N = a.N, K = a.K, n0 = blockIdx.x * 16;
    if (M == 0) return;
    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), row = lane & 15u, part = (lane >> 4) * V;
    const T* A = static_cast<const T*>(a.a.p[q]);
    const T* B = static_cast<const T*>(a.b.p[q]) + (size_t)min(n0 + row, N - 1) * a.ldb;        // rows outside: another's, not kept
    const uint32_t steps = (K + STEP - 1) / STEP, share = (steps + 7) / 8;
    const uint32_t s0 = min(steps, wave * share), s1 = min(steps, s0 + share);
    f32x4 acc[MF];
#pragma unroll
    for (int f = 0; f < MF; ++f) acc[f] = f32x4{0.f, 0.f, 0.f, 0.f};
    auto row_of_a = [&](int f) { return A + (size_t)min((uint32_t)f * 16 + row, M - 1) * a.lda; };
    auto multiply = [&](raw4 vb, const raw4 (&va)[MF]) {
#pragma unroll
        for (int e = 0; e < Mma<T>::PARTS; ++e)
#pragma unroll
            for (int f = 0; f < MF; ++f) acc[f] = Mma<T>::part(vb, va[f], acc[f], e);
    };
    auto run = [&](auto ahead) {
        constexpr uint32_t D = decltype(ahead)::value;
        raw4 vb[D], va[D][MF];
        auto ask = [&](uint32_t s, uint32_t i) {
            const uint32_t k = min(min(s, s1 - 1) * STEP + part, K - V);
            vb[i] = load_raw<T, 1>(B + k);
#pragma unroll
            for (int f = 0; f < MF; ++f) va[i][f] = load_raw<T>(row_of_a(f) + k);
        };
        auto use = [&](uint32_t s, uint32_t i) {
            if ((s + 1) * STEP > K) {                                                            // the last step: what lies behind the rows' ends
                const uint32_t k = s * STEP + part;
                auto cut = [&](raw4& v) {
                    if (k < K && k + V > K) v = move_down<T>(v, k + V - K);
                    if (k >= K) v = raw4{0, 0, 0, 0};
                };
                cut(vb[i]);
#pragma unroll
                for (int f = 0; f < MF; ++f) cut(va[i][f]);
            }
            multiply(vb[i], va[i]);
        };
#pragma unroll
        for (uint32_t i = 0; i < D; ++i) ask(s0 + i, i);
        uint32_t s = s0;
        for (; s + D < s1; s += D)
#pragma unroll
            for (uint32_t i = 0; i < D; ++i) {
                multiply(vb[i], va[i]);                                                          // never the last step
                ask(s + D + i, i);
            }
#pragma unroll
        for (uint32_t i = 0; i < D; ++i)
            if (s + i < s1) use(s + i, i);
    };
    if (K < V) {
        if (wave == 0) {
            raw4 va[MF];
#pragma unroll
            for (int f = 0; f < MF; ++f) va[f] = part < K ? load_clip(row_of_a(f), part, K) : raw4{0, 0, 0, 0};
            multiply(part < K ? load_clip(B, part, K) : raw4{0, 0, 0, 0}, va);
        }
    } else if (s0 < s1) {
        if (MF == 4 || share <= 4) run(std::integral_constant<uint32_t, 4>{});
        else if constexpr (MF < 4) {
            if ((share + 4) / 5 * 5 < (share + 7) / 8 * 8) run(std::integral_constant<uint32_t, 5>{});
            else run(std::integral_constant<uint32_t, 8>{});
        }
    }
#pragma unroll
    for (int f = 0; f < MF; ++f) meet[wave][f][lane] = acc[f];
    __syncthreads();
    if (wave >= MF) return;
    f32x4 v = meet[0][wave][lane];
#pragma unroll
    for (int w = 1; w < 8; ++w) v += meet[w][wave][lane];
    const uint32_t m = wave * 16 + row, n = n0 + (lane >> 4) * 4;
    if (m >= M || n >= N) return;
    const float s[4] = {v[0], v[1], v[2], v[3]};
    epilogue4<T, EPI>(a, q, m, n, N, s);
}

// The pieces of split sums, added in order (eight asked for at a time, the last one again where there are fewer), and the epilogue.
// grid (blocks, rows in turn, workers)
template <class T, int EPI>
__global__ __launch_bounds__(256) void k_gemm_join(GemmArgs a)
{
    const uint32_t q = blockIdx.z, M = a.k_is_rows ? a.M : a.rows.n[q], N = a.N;
    const uint32_t n = (blockIdx.x * 256 + threadIdx.x) * 4;
    if (n >= N) return;
    // a worker whose sum is shorter than the longest has fewer pieces
    const uint32_t pieces = a.k_is_rows ? max(1u, (a.rows.n[q] + a.k_split - 1) / a.k_split) : a.splits;
    for (uint32_t m = blockIdx.y; m < M; m += gridDim.y) {
        float s[4] = {0.f, 0.f, 0.f, 0.f};
        const float* from = a.partial + (((size_t)q * a.splits) * a.M + m) * N + n;
        const size_t step = (size_t)a.M * N;
        for (uint32_t p = 0; p < pieces; p += 8) {
            float x[8][4];
#pragma unroll
            for (uint32_t i = 0; i < 8; ++i) load4(from + min(p + i, pieces - 1) * step, N - n, x[i]);
#pragma unroll
            for (uint32_t i = 0; i < 8; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (p + i < pieces) s[e] += x[i][e];
        }
        epilogue4<T, EPI>(a, q, m, n, N, s);
    }
}

}  // namespace slimdp
