// libslimdp, the worker side's training operators (layer norm, matrix product with epilogue, distillation loss, each with its
// gradients): argument checks and launches.  The kernels are in slimdp_norm.h, slimdp_linear.h and slimdp_distill.h.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <type_traits>

#include "slimdp.h"
#include "slimdp_host.h"
#include "slimdp_norm.h"
#include "slimdp_linear.h"
#include "slimdp_gemm.h"
#include "slimdp_gemm32.h"
#include "slimdp_distill.h"

using namespace slimdp;

namespace {

constexpr uint64_t LD_MAX = 1ull << 32;
// Streams of more than the last level's 256 MB pass the caches by.
constexpr uint64_t STREAM_BYTES = 256ull << 20;

// The context's device for the length of a call, whichever is current.
struct OnDevice {
    int before = -1;
    hipError_t e;
    explicit OnDevice(int device)
    {
        e = hipGetDevice(&before);
        if (e == hipSuccess && before != device) e = hipSetDevice(device); else before = -1;
    }
    ~OnDevice() { if (before >= 0) (void)hipSetDevice(before); }
};

struct Call {
    slimdp_ctx* ctx;
    const char* who;
    HostView v{};
    uint32_t W = 0;
    const uint64_t* rows = nullptr;
    uint64_t most = 0;               // rows of the worker that has most
    RowTab tab{};
    int rc = SLIMDP_OK;

    bool ok() const { return rc == SLIMDP_OK; }
    size_t esize = 4;

    int begin(slimdp_ctx* c, const char* name, uint32_t n_workers, const uint64_t* r, uint32_t dtype)
    {
        ctx = c;
        who = name;
        if (!c) return rc = SLIMDP_ERR_INVALID_ARG;
        v = host_view(c);
        W = n_workers;
        if (W == 0 || W > v.max_workers)
            return rc = host_fail(c, SLIMDP_ERR_INVALID_ARG, "%s: n_workers=%u outside [1, %u]", who, W, v.max_workers);
        if (!r) return rc = host_fail(c, SLIMDP_ERR_INVALID_ARG, "%s: rows is NULL", who);
        if (dtype > SLIMDP_BF16) return rc = host_fail(c, SLIMDP_ERR_INVALID_ARG, "%s: unknown dtype %u", who, dtype);
        esize = dtype == SLIMDP_F32 ? 4 : 2;
        rows = r;
        for (uint32_t q = 0; q < W; ++q) {
            if (r[q] > SLIMDP_MAX_ROWS)
                return rc = host_fail(c, SLIMDP_ERR_OUT_OF_RANGE, "%s: rows[%u] exceeds %llu", who, q, (unsigned long long)SLIMDP_MAX_ROWS);
            tab.n[q] = (uint32_t)r[q];
            most = std::max(most, r[q]);
        }
        return rc;
    }
    void size(const char* what, uint64_t n, uint64_t max)
    {
        if (!ok()) return;
        if (n == 0) rc = host_fail(ctx, SLIMDP_ERR_INVALID_ARG, "%s: %s is 0", who, what);
        else if (n > max) rc = host_fail(ctx, SLIMDP_ERR_OUT_OF_RANGE, "%s: %s exceeds %llu", who, what, (unsigned long long)max);
    }
    // A table of matrices with a row each of a worker's rows (their entries may be NULL where there are none).
    template <class P> void matrix(const char* what, P const* t, uint64_t ld, uint64_t cols, size_t es, bool optional = false)
    {
        if (!ok() || (!t && optional)) return;
        if (!t) { rc = host_fail(ctx, SLIMDP_ERR_INVALID_ARG, "%s: %s is NULL", who, what); return; }
        if (ld < cols || ld > LD_MAX) {
            rc = host_fail(ctx, SLIMDP_ERR_INVALID_ARG, "%s: rows of %s are %llu apart, with %llu elements each", who, what,
                           (unsigned long long)ld, (unsigned long long)cols);
            return;
        }
        for (uint32_t q = 0; q < W; ++q) entry(what, q, t[q], es, rows[q] != 0);
    }
    // A table of parameter vectors or matrices (needed whatever the rows); optional: the table, or single entries.
    template <class P> void params(const char* what, P const* t, size_t es, bool optional)
    {
        if (!ok() || (!t && optional)) return;
        if (!t) { rc = host_fail(ctx, SLIMDP_ERR_INVALID_ARG, "%s: %s is NULL", who, what); return; }
        for (uint32_t q = 0; q < W; ++q) entry(what, q, t[q], es, !optional);
    }
    void entry(const char* what, uint32_t q, const void* p, size_t es, bool needed)
    {
        if (!ok()) return;
        if (!p && needed) rc = host_fail(ctx, SLIMDP_ERR_INVALID_ARG, "%s: %s[%u] is NULL", who, what, q);
        else if (reinterpret_cast<uintptr_t>(p) % es) rc = host_fail(ctx, SLIMDP_ERR_INVALID_ARG, "%s: %s[%u] is not aligned to its elements", who, what, q);
    }
    // Outputs that may not be the given array; own: but for the same worker's.  per_row: matrices with a row for each of the worker's.
    template <class P, class R> void apart(const char* wa, P const* a, const char* wb, R const* b, bool own = false, bool per_row = true)
    {
        if (!ok() || !a || !b) return;
        for (uint32_t q = 0; q < W; ++q)
            for (uint32_t o = 0; o < W; ++o)
                if (a[q] && (!per_row || (rows[q] && rows[o])) && !(own && q == o) &&
                    static_cast<const void*>(a[q]) == static_cast<const void*>(b[o])) {
                    rc = host_fail(ctx, SLIMDP_ERR_INVALID_ARG, "%s: %s[%u] is %s[%u]", who, wa, q, wb, o);
                    return;
                }
    }
    // Outputs of different workers are different arrays.
    template <class P> void distinct(const char* what, P const* t, bool per_row)
    {
        if (!ok() || !t) return;
        for (uint32_t q = 0; q < W; ++q)
            for (uint32_t o = 0; o < q; ++o)
                if (t[q] && t[q] == t[o] && (!per_row || (rows[q] && rows[o]))) {
                    rc = host_fail(ctx, SLIMDP_ERR_INVALID_ARG, "%s: %s[%u] is %s[%u]", who, what, o, what, q);
                    return;
                }
    }
    void workspace(void* ws, uint64_t have, uint64_t need)
    {
        if (!ok() || need == 0) return;
        if (!ws || have < need)
            rc = host_fail(ctx, SLIMDP_ERR_WORKSPACE, "%s: needs a workspace of %llu bytes, got %llu", who, (unsigned long long)need,
                           (unsigned long long)(ws ? have : 0));
        else if (reinterpret_cast<uintptr_t>(ws) % 16) rc = host_fail(ctx, SLIMDP_ERR_INVALID_ARG, "%s: workspace is not aligned to 16 bytes", who);
    }
    // Bytes of some matrices of this many columns.
    uint64_t bytes(uint64_t cols, uint64_t matrices) const
    {
        uint64_t b = 0;
        for (uint32_t q = 0; q < W; ++q) b += rows[q] * cols * esize * matrices;
        return b;
    }
    template <class P> InTab in(P const* t) const
    {
        InTab r;
        for (int q = 0; q < MAXW_T; ++q) r.p[q] = t && q < (int)W ? t[q] : nullptr;
        return r;
    }
    template <class P> OutTab out(P const* t) const
    {
        OutTab r;
        for (int q = 0; q < MAXW_T; ++q) r.p[q] = t && q < (int)W ? t[q] : nullptr;
        return r;
    }
    template <class F> int launched(const char* name, F&& f)
    {
        OnDevice dev(v.device);
        if (dev.e != hipSuccess) return rc = host_fail(ctx, SLIMDP_ERR_HIP, "%s: hipSetDevice: %s", who, hipGetErrorString(dev.e));
        f();
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) rc = host_fail(ctx, SLIMDP_ERR_HIP, "%s: %s", name, hipGetErrorString(e));
        return rc;
    }
};

template <class F> void with_type(uint32_t dtype, F&& f)
{
    if (dtype == SLIMDP_F32) f(float{});
    else if (dtype == SLIMDP_F16) f(_Float16{});
    else f(__bf16{});
}

inline uint64_t ceil_div(uint64_t a, uint64_t b) { return (a + b - 1) / b; }
inline uint64_t most_rows(uint32_t n_workers, const uint64_t* rows)
{
    uint64_t m = 0;
    for (uint32_t q = 0; q < n_workers; ++q) m = std::max(m, rows[q]);
    return m;
}
bool shape_ok(uint32_t n_workers, const uint64_t* rows)
{
    return n_workers && n_workers <= SLIMDP_MAX_WORKERS && rows && most_rows(n_workers, rows) <= SLIMDP_MAX_ROWS;
}

// Workers that the rows would make if all had as many as the largest: what a launch's blocks are shared between (a worker without rows needs none).
uint64_t crowd(uint32_t n_workers, const uint64_t* rows)
{
    uint64_t all = 0;
    for (uint32_t q = 0; q < n_workers; ++q) all += rows[q];
    return std::max<uint64_t>(1, ceil_div(all, std::max<uint64_t>(1, most_rows(n_workers, rows))));
}

// Vectors that a block of the sums over rows takes of a row.
uint32_t column_lanes(uint64_t cols, size_t es)
{
    const uint64_t n = ceil_div(cols, 16 / es);
    return n <= 8 ? 8 : n <= 16 ? 16 : n <= 32 ? 32 : 64;
}
// Rows of a slab of the sums over rows: as many slabs as give the chip eight blocks a compute unit (of 256), of four rows or more for
// every group of a block's threads.
uint64_t slab_rows(uint32_t W, const uint64_t* rows, uint64_t cols, size_t es)
{
    const uint32_t lx = column_lanes(cols, es);
    const uint64_t most = most_rows(W, rows), across = ceil_div(cols, lx * (16 / es)) * crowd(W, rows);
    const uint64_t slabs = std::max<uint64_t>(1, std::min<uint64_t>(2048 / across, ceil_div(most, 4 * 256 / lx)));
    return std::max<uint64_t>(1, ceil_div(most, slabs));
}
uint64_t column_ws(uint32_t W, const uint64_t* rows, uint64_t cols, size_t es, int arrays)
{
    const uint64_t slabs = ceil_div(most_rows(W, rows), slab_rows(W, rows, cols, es));
    return slabs <= 1 ? 0 : W * slabs * arrays * cols * 4;
}

// Layer norm's backward pass in one: threads a row, and blocks a worker (256 blocks of 1024 threads, or four times as many of 256, fill
// the chip; four rows a group at least, so that the sums that the blocks write are few beside the rows).  tpr 0: rows too long to
// be held beside their sums, two passes.
struct NormBackShape { uint32_t tpr, block; uint64_t blocks; };
NormBackShape norm_back_shape(uint32_t W, const uint64_t* rows, uint64_t cols, size_t es)
{
    const uint64_t most = most_rows(W, rows), n = ceil_div(cols, 16 / es);
    const uint32_t tpr = n <= 8 ? 8 : n <= 16 ? 16 : n <= 32 ? 32 : n <= 128 ? 64 : n <= 512 ? 256 : n <= 1024 ? 512 : n <= 2048 ? 1024 : 0;
    if (!tpr) return {0, 0, 0};
    const uint32_t block = tpr <= 64 ? 256 : 1024, groups = block / tpr;
    const uint64_t fill = std::max<uint64_t>(1, (block == 256 ? 1024 : 256) / crowd(W, rows));
    return {tpr, block, std::max<uint64_t>(1, std::min(fill, ceil_div(most, 4 * groups)))};
}

void column_sums(Call& c, const ColumnSumArgs& s)
{
    c.launched("k_column_sums", [&] {
        const dim3 grid((uint32_t)ceil_div(s.cols, 16), s.arrays, c.W);
        if (s.slabs <= 128) hipLaunchKernelGGL(k_column_sums<16>, grid, dim3(256), 0, c.v.stream, s);
        else hipLaunchKernelGGL(k_column_sums<64>, grid, dim3(1024), 0, c.v.stream, s);
    });
}

// ws: for the slabs' sums; nullptr where no sums are asked for.
template <bool NORM> int column_grads(Call& c, ColumnArgs a, uint32_t dtype, int act, bool sums, void* ws)
{
    constexpr int ARR = NORM ? 2 : 1;
    a.rows = c.tab;
    a.slab = (uint32_t)slab_rows(c.W, c.rows, a.cols, c.esize);
    a.slabs = (uint32_t)std::max<uint64_t>(1, ceil_div(c.most, a.slab));
    a.partial = sums && a.slabs > 1 ? static_cast<float*>(ws) : nullptr;
    with_type(dtype, [&](auto z) {
        typedef decltype(z) T;
        const bool nt = c.bytes(a.cols, 3) > STREAM_BYTES;
        const uint32_t lx = column_lanes(a.cols, c.esize);
        auto launch = [&](auto kernel, auto kernel_nt) {
            c.launched("k_column_grads", [&] {
                const dim3 grid((uint32_t)ceil_div(a.cols, lx * Vec<T>::N), a.slabs, c.W);
                if (nt) hipLaunchKernelGGL(kernel_nt, grid, dim3(256), 0, c.v.stream, a);
                else hipLaunchKernelGGL(kernel, grid, dim3(256), 0, c.v.stream, a);
            });
        };
#define SLIMDP_COLUMNS(ACT)                                                                                      \
    do {                                                                                                         \
        if (lx == 8) launch(k_column_grads<T, NORM, ACT, 8, 0>, k_column_grads<T, NORM, ACT, 8, 1>);             \
        else if (lx == 16) launch(k_column_grads<T, NORM, ACT, 16, 0>, k_column_grads<T, NORM, ACT, 16, 1>);     \
        else if (lx == 32) launch(k_column_grads<T, NORM, ACT, 32, 0>, k_column_grads<T, NORM, ACT, 32, 1>);     \
        else launch(k_column_grads<T, NORM, ACT, 64, 0>, k_column_grads<T, NORM, ACT, 64, 1>);                   \
    } while (0)
        if constexpr (NORM) launch(k_column_grads<T, true, ACT_NONE, 64, 0>, k_column_grads<T, true, ACT_NONE, 64, 1>);      // long rows only
        else {
            if (act == ACT_NONE) SLIMDP_COLUMNS(ACT_NONE);
            else if (act == ACT_RELU) SLIMDP_COLUMNS(ACT_RELU);
            else if (act == ACT_GELU) SLIMDP_COLUMNS(ACT_GELU);
            else if (act == ACT_GELU_TANH) SLIMDP_COLUMNS(ACT_GELU_TANH);
            else SLIMDP_COLUMNS(ACT_SILU);
        }
#undef SLIMDP_COLUMNS
    });
    if (c.ok() && a.partial) {
        column_sums(c, ColumnSumArgs{a.partial, a.out0, a.out1, c.tab, a.cols, a.slab, a.slabs, (uint32_t)ARR, a.accumulate});
    }
    return c.rc;
}

// ---------------------------------------------------------------------------------------
// products
// ---------------------------------------------------------------------------------------
// How a product is cut: the kernel, its tile and the pieces of the sum, by the sizes and the type (and, for the copies into the LDS, the
// operands' layout; the workspace is asked for as if that did not matter, the larger of both).
struct Product {
    uint64_t M, N, K;
    uint32_t W;
    const uint64_t* rows;
    size_t es;
    bool forward, rows_of_k;     // both operands with k running;  K is the number of rows
    double results = 0;          // elements of all results
    bool uneven = false;         // sums of different lengths

    // Small calls wait for the host: what the cuts share is found once, and so is a cut.
    Product(uint64_t m, uint64_t n, uint64_t k, uint32_t w, const uint64_t* r, size_t e, int which)
        : M(m), N(n), K(k), W(w), rows(r), es(e), forward(which == 0), rows_of_k(which == 2)
    {
        for (uint32_t q = 0; q < W; ++q) {
            results += (double)(rows_of_k ? M : rows[q]) * (double)N;
            uneven |= rows_of_k && rows[q] != rows[0];
        }
    }
    struct Cut { uint32_t bm, bn; uint64_t tiles, splits, piece; double us; };
    uint64_t tiles(uint32_t t) const { return ceil_div(M, t) * ceil_div(N, t); }
    // Sixteen-bit types, as measured: `slots` blocks run at a time over the 256 compute units, `step` us for a step of all of them (less
    // where there is one block to a unit at most), `ends` us to begin and to write, and where the sum is cut the pieces' way to memory and back at
    // 4 TB/s.  Products of 8192 x 8192 x 8192 and 8 x 2048 x 4096 x 4096, bf16: 1.45 us a step with 256 x 256, 0.95 with two of 128 x 128.
    struct Kernel { uint32_t tile, slots; double step, alone, ends; };
    Cut cut(const Kernel& k, uint64_t want, uint64_t all) const
    {
        const uint64_t bk = 128 / es, steps = ceil_div(K, bk), per = std::max<uint64_t>(1, ceil_div(steps, want));
        const uint64_t splits = std::max<uint64_t>(1, ceil_div(steps, per)), blocks = blocks_of(all, steps, per, splits);
        const double step = blocks <= 256 ? k.alone : k.step;
        // blocks of workers with shorter sums fill the last round up: what all of them take counts, not whole rounds of the longest
        const double rounds = uneven ? std::max(1.0, (double)all / (double)per / k.slots) : (double)ceil_div(blocks, k.slots);
        double us = rounds * ((double)per * step + k.ends);
        if (splits > 1) us += 4.0 + results * (double)splits * 8.0 / 4e6;
        return {k.tile, k.tile, tiles(k.tile), splits, per * bk, us};
    }
    // Steps of all the workers' tiles, those without a step counted as one.
    uint64_t steps_of_all(uint32_t bm, uint32_t bn, uint64_t bk) const
    {
        uint64_t n = 0;
        for (uint32_t q = 0; q < W; ++q) n += rows_of_k ? std::max<uint64_t>(1, ceil_div(rows[q], bk)) : ceil_div(rows[q], bm);
        return n * ceil_div(N, bn) * (rows_of_k ? ceil_div(M, bm) : ceil_div(K, bk));
    }
    // Blocks of all workers; of sums of different lengths as many whole ones as their steps make.
    uint64_t blocks_of(uint64_t all, uint64_t steps, uint64_t per, uint64_t splits) const
    {
        return uneven ? ceil_div(all, per) : all / std::max<uint64_t>(1, steps) * splits;
    }
    Cut best(const Kernel& big, const Kernel& small) const
    {
        const uint64_t all_big = steps_of_all(big.tile, big.tile, 128 / es), all_small = steps_of_all(small.tile, small.tile, 128 / es);
        Cut b = cut(big, 1, all_big);
        for (const uint64_t want : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64}) {
            const Cut c = cut(big, want, all_big), d = cut(small, want, all_small);
            if (c.us < b.us) b = c;
            if (d.us < b.us) b = d;
        }
        return b;
    }
    // by copies into the LDS: sixteen-bit types
    const Cut& copies() const { return once(copies_, [&] { return best({256, 256, 1.45, 1.45, 12.0}, {128, 512, 0.95, 0.65, 8.0}); }); }
    // rows shorter than a vector, and what the copies do not reach: element by element
    const Cut& elements() const
    {
        const Kernel k = {64, 1024, 2.0, 0.7, 6.0};
        return once(elements_, [&] { return best(k, k); });
    }
    // Binary32.  A block's step is 32 of k.  One block to a compute unit takes `alone` us for it, several share the unit at `step` each;
    // `begin` us a block of 64 x 64 for what is no step, 18 TB/s for what all blocks read together (the caches' rate), and where the sum
    // is cut a second launch and the pieces' way to memory and back at 4 TB/s.  Fitted to the times of 5,800 products of 1 to 16,384 rows, 16 to 8192
    // in and out, forward and backward, one to eight workers, with every tile and 1 to 48 pieces: the cut that these constants choose takes
    // 1.6 % more than the fastest on average (up to a third more of calls of 12 to 70 us).
    struct Tile { uint32_t bm, bn; double step, alone; };
    const Cut& tiles32() const { return once(tiles32_, [&] { return find32(); }); }
    Cut find32() const
    {
        static const Tile list[] = {{64, 64, 0.42, 0.47}, {128, 32, 0.44, 0.6}, {32, 64, 0.24, 0.47}, {32, 32, 0.135, 0.16}, {16, 64, 0.18, 0.18}, {64, 16, 0.18, 0.18}};
        const uint64_t steps = ceil_div(K, 32);
        Cut b{};
        for (const Tile& t : list) {
            const uint64_t all = steps_of_all(t.bm, t.bn, 32), tiles = rows_of_k ? W * ceil_div(M, t.bm) * ceil_div(N, t.bn) : all / std::max<uint64_t>(1, steps);
            const double area = t.bm * t.bn / 4096.0;
            uint64_t last = 0;
            for (const uint64_t want : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48}) {
                const uint64_t per = std::max<uint64_t>(1, ceil_div(steps, want)), splits = std::max<uint64_t>(1, ceil_div(steps, per));
                if (splits == last) continue;
                last = splits;
                if (tiles * splits > (1ull << 24) && (splits > 1 || t.bm * t.bn < 4096)) break;
                const double n = (double)blocks_of(all, steps, per, splits) / 256.0, whole = std::ceil(n), each = (double)per;
                double us = std::max({each * t.alone, (whole <= 8 ? whole : n) * (each * t.step + 0.09 * area), n * each * (t.bm + t.bn) * 32768.0 / 18e6});
                if (splits > 1) us += 6.0 + results * (double)splits * 8.0 / 4e6;
                if (!b.bm || us < b.us) b = {t.bm, t.bn, tiles, splits, per * 32, us};
            }
        }
        return b;
    }
    // The blocks of every worker: only those that have work.
    uint64_t number(const Cut& c, GemmArgs& a) const
    {
        uint64_t blocks = 0;
        a.spread = uneven;
        const uint64_t across = ceil_div(N, c.bn), down = ceil_div(M, c.bm);
        for (uint32_t q = 0; q < W; ++q) {
            a.first[q] = (uint32_t)blocks;
            blocks += across * (rows_of_k ? down * std::max<uint64_t>(1, ceil_div(rows[q], c.piece)) : ceil_div(rows[q], c.bm) * c.splits);
        }
        for (uint32_t q = W; q <= MAXW_T; ++q) a.first[q] = (uint32_t)blocks;
        a.blocks = (uint32_t)blocks;
        a.each = a.first[1];
        for (uint32_t q = 2; q <= W; ++q)
            if (a.first[q] != q * a.each) a.each = 0;
        return blocks;
    }
    // ... of rows that no vector fits in
    bool narrow() const { return std::min(N, rows_of_k ? M : K) < 4; }
    bool few() const { return es == 2 && forward && M <= 64 && ceil_div(N, 16) * W >= 64; }
    static uint64_t bytes(const Cut& c, const Product& p) { return c.splits > 1 ? p.W * c.splits * p.M * p.N * 4 : 0; }
    uint64_t ws() const
    {
        if (few()) return 0;
        if (es == 2) return std::max(bytes(elements(), *this), bytes(copies(), *this));
        return bytes(narrow() ? elements() : tiles32(), *this);
    }

private:
    template <class F> static const Cut& once(Cut& c, F&& f)
    {
        if (!c.bm) c = f();
        return c;
    }
    mutable Cut copies_{}, elements_{}, tiles32_{};
};

// What a grid can number, whichever the tile; asked before a call's first launch.
void tiles_fit(Call& c, const Product& p)
{
    if (c.ok() && p.tiles(64) > SLIMDP_MAX_TILES)
        c.rc = host_fail(c.ctx, SLIMDP_ERR_OUT_OF_RANGE, "%s: a result of %llu x %llu has more than %llu tiles of 64 x 64", c.who,
                         (unsigned long long)p.M, (unsigned long long)p.N, (unsigned long long)SLIMDP_MAX_TILES);
}

// How the tile kernel takes sixteen-bit operands: not at all (2: rows shorter than a vector, or distances that do not fit its offsets), through
// registers (1), or copied into the LDS as they lie (0: whole vectors on their own alignment).
template <bool AK, bool BK> int staging(const Call& c, const GemmArgs& a, const Product& p)
{
    auto of = [&](const InTab& t, uint64_t ld, uint64_t run) {
        if (run < 8 || ld > (1u << 21)) return 2;
        if (ld % 8 || run % 8) return 1;
        for (uint32_t q = 0; q < c.W; ++q)
            if (reinterpret_cast<uintptr_t>(t.p[q]) % 16) return 1;
        return 0;
    };
    return p.es == 2 ? std::max(of(a.a, a.lda, AK ? p.M : p.K), of(a.b, a.ldb, BK ? p.N : p.K)) : 2;
}

// A grid of so many blocks: one dimension numbers 2^32 threads.
dim3 over_two(uint64_t blocks)
{
    constexpr uint64_t ACROSS = 1u << 20;
    return dim3((uint32_t)std::min(blocks, ACROSS), (uint32_t)ceil_div(blocks, ACROSS));
}

// The second launch of a product whose sum was cut.
template <class T, int EPI> int joined(Call& c, const GemmArgs& a, const Product& p)
{
    if (c.ok() && a.splits > 1)
        c.launched("k_gemm_join", [&] {
            hipLaunchKernelGGL((k_gemm_join<T, EPI>), dim3((uint32_t)ceil_div(p.N, 1024), (uint32_t)std::min<uint64_t>(p.M, 1024), c.W),
                               dim3(256), 0, c.v.stream, a);
        });
    return c.rc;
}

template <bool AK, bool BK, int EPI> int product(Call& c, GemmArgs a, const Product& p, uint32_t dtype, void* ws)
{
    if (p.M == 0 || p.N == 0) return c.rc;
    a.rows = c.tab;
    a.M = (uint32_t)p.M; a.N = (uint32_t)p.N; a.K = (uint32_t)p.K;
    a.partial = static_cast<float*>(ws);
    a.splits = 1;
    if (dtype == SLIMDP_F32 && !p.narrow()) {
        const Product::Cut& cut = p.tiles32();
        a.splits = (uint32_t)cut.splits;
        a.k_split = (uint32_t)cut.piece;
        const uint64_t blocks = p.number(cut, a);
        auto launch = [&](auto kernel) {
            c.launched("k_gemm32", [&] { hipLaunchKernelGGL(kernel, over_two(blocks), dim3(256), 0, c.v.stream, a); });
        };
        if (cut.bm == 64 && cut.bn == 64 && std::min(cut.piece, p.K) <= 256) launch(k_gemm32<AK, BK, EPI, 64, 64, 2, 2, false>);
        else if (cut.bm == 64 && cut.bn == 64) launch(k_gemm32<AK, BK, EPI, 64, 64, 2, 2, true>);
        else if (cut.bm == 128) launch(k_gemm32<AK, BK, EPI, 128, 32, 4, 1, true>);
        else if (cut.bm == 32 && cut.bn == 64) launch(k_gemm32<AK, BK, EPI, 32, 64, 1, 4, true>);
        else if (cut.bm == 32) launch(k_gemm32<AK, BK, EPI, 32, 32, 2, 2, true>);
        else if (cut.bm == 16) launch(k_gemm32<AK, BK, EPI, 16, 64, 1, 4, true>);
        else launch(k_gemm32<AK, BK, EPI, 64, 16, 4, 1, true>);
        return joined<float, EPI>(c, a, p);
    }
    if constexpr (!AK && !BK) {
        // few rows against many: 16 rows of weights a block
        if (p.few()) {
            auto of = [&](auto z) {
                typedef decltype(z) T;
                auto launch = [&](auto kernel) {
                    c.launched("k_gemm_few", [&] {
                        hipLaunchKernelGGL(kernel, dim3((uint32_t)ceil_div(p.N, 16), 1, c.W), dim3(512), 0, c.v.stream, a);
                    });
                };
                if (p.M <= 16) launch(k_gemm_few<T, 1, EPI>);
                else if (p.M <= 32) launch(k_gemm_few<T, 2, EPI>);
                else launch(k_gemm_few<T, 4, EPI>);
            };
            if (dtype == SLIMDP_F16) of(_Float16{}); else of(__bf16{});
            return c.rc;
        }
    }
    const int stage = staging<AK, BK>(c, a, p);
    const Product::Cut& cut = stage < 2 ? p.copies() : p.elements();
    a.splits = (uint32_t)cut.splits;
    a.k_split = (uint32_t)cut.piece;
    const uint64_t blocks = p.number(cut, a);
    with_type(dtype, [&](auto z) {
        typedef decltype(z) T;
        if constexpr (sizeof(T) == 2) {
            auto launch = [&](auto kernel) {
                c.launched("k_gemm_tiles", [&] { hipLaunchKernelGGL(kernel, over_two(blocks), dim3(256), 0, c.v.stream, a); });
            };
            if (stage == 0 && cut.bm == 256) launch(k_gemm_tiles<T, AK, BK, EPI, 256, 256, 2, 2, 1, true>);
            else if (stage == 0) launch(k_gemm_tiles<T, AK, BK, EPI, 128, 128, 2, 2, 2, true>);
            else if (stage == 1 && cut.bm == 256) launch(k_gemm_tiles<T, AK, BK, EPI, 256, 256, 2, 2, 1, false>);
            else if (stage == 1) launch(k_gemm_tiles<T, AK, BK, EPI, 128, 128, 2, 2, 2, false>);
        }
        if (stage == 2)
            c.launched("k_gemm", [&] {
                hipLaunchKernelGGL((k_gemm<T, AK, BK, EPI>), dim3((uint32_t)cut.tiles, 1, c.W * a.splits), dim3(256), 0, c.v.stream, a);
            });
        joined<T, EPI>(c, a, p);
    });
    return c.rc;
}

Product forward_product(uint32_t W, const uint64_t* rows, uint64_t in, uint64_t out, size_t es)
{
    return Product(most_rows(W, rows), out, in, W, rows, es, 0);
}
Product input_product(uint32_t W, const uint64_t* rows, uint64_t in, uint64_t out, size_t es)
{
    return Product(most_rows(W, rows), in, out, W, rows, es, 1);
}
Product weight_product(uint32_t W, const uint64_t* rows, uint64_t in, uint64_t out, size_t es)
{
    return Product(out, in, most_rows(W, rows), W, rows, es, 2);
}

}  // namespace

extern "C" {

int slimdp_layer_norm(slimdp_ctx* ctx, uint32_t n_workers, const uint64_t* rows, uint64_t cols, uint32_t dtype, const void* const* x,
                      uint64_t ldx, const float* const* weight, const float* const* bias, float eps, void* const* y, uint64_t ldy,
                      float* const* mean, float* const* rstd)
{
    Call c;
    if (c.begin(ctx, "slimdp_layer_norm", n_workers, rows, dtype)) return c.rc;
    c.size("cols", cols, SLIMDP_MAX_NORM_COLS);
    c.matrix("x", x, ldx, cols, c.esize);
    c.matrix("y", y, ldy, cols, c.esize);
    c.params("weight", weight, 4, true);
    c.params("bias", bias, 4, true);
    c.matrix("mean", mean, 1, 1, 4, true);
    c.matrix("rstd", rstd, 1, 1, 4, true);
    c.apart("y", y, "x", x, ldx == ldy);
    c.distinct("y", y, true);
    c.distinct("mean", mean, true);
    c.distinct("rstd", rstd, true);
    c.apart("mean", mean, "rstd", rstd);
    if (c.ok() && !(eps > 0.0f && std::isfinite(eps))) c.rc = host_fail(ctx, SLIMDP_ERR_INVALID_ARG, "slimdp_layer_norm: eps must be positive and finite");
    if (!c.ok() || c.most == 0) return c.rc;
    const bool nt = c.bytes(cols, 2) > STREAM_BYTES;
    const NormArgs a{c.in(x), c.in(weight), c.in(bias), c.out(y), c.out(mean), c.out(rstd), c.tab, ldx, ldy, (uint32_t)cols, eps};
    with_type(dtype, [&](auto z) {
        typedef decltype(z) T;
        const uint64_t n = ceil_div(cols, Vec<T>::N);
        // eight blocks of 256 threads a compute unit (of 256), a block's next row under way while it sums the present one
        auto launch = [&](auto kernel, auto kernel_nt, uint32_t tpr) {
            const uint32_t block = std::max(tpr, 256u), groups = block / tpr;
            const uint64_t want = ceil_div(c.most, groups), cap = std::max<uint64_t>(1, 2048 * 256 / block / crowd(c.W, rows));
            c.launched("k_norm", [&] {
                const dim3 grid((uint32_t)std::min(want, cap), c.W);
                if (nt) hipLaunchKernelGGL(kernel_nt, grid, dim3(block), 0, c.v.stream, a);
                else hipLaunchKernelGGL(kernel, grid, dim3(block), 0, c.v.stream, a);
            });
        };
#define SLIMDP_NORM(TPR, NC) launch(k_norm<T, TPR, NC, 0>, k_norm<T, TPR, NC, 1>, TPR)
        if (n <= 8) SLIMDP_NORM(8, 1);
        else if (n <= 16) SLIMDP_NORM(16, 1);
        else if (n <= 32) SLIMDP_NORM(32, 1);
        else if (n <= 64) SLIMDP_NORM(64, 1);
        else if (n <= 128) SLIMDP_NORM(64, 2);
        else if (n <= 256) SLIMDP_NORM(256, 1);
        else if (n <= 512) SLIMDP_NORM(256, 2);
        else if (n <= 1024) SLIMDP_NORM(256, 4);
        else if (n <= 2048) SLIMDP_NORM(1024, 2);
        else if (n <= 4096) SLIMDP_NORM(1024, 4);
        else if (n <= 8192) SLIMDP_NORM(1024, 8);
        else if constexpr (Vec<T>::N == 4) SLIMDP_NORM(1024, 16);
#undef SLIMDP_NORM
    });
    return c.rc;
}

uint64_t slimdp_layer_norm_workspace_bytes(uint32_t n_workers, const uint64_t* rows, uint64_t cols, uint32_t dtype)
{
    if (!shape_ok(n_workers, rows) || cols == 0 || cols > SLIMDP_MAX_NORM_COLS || dtype > SLIMDP_BF16) return 0;
    const size_t es = dtype == SLIMDP_F32 ? 4 : 2;
    const NormBackShape s = norm_back_shape(n_workers, rows, cols, es);
    if (s.tpr) return s.blocks > 1 ? n_workers * s.blocks * 2 * cols * 4 : 0;
    return column_ws(n_workers, rows, cols, es, 2);
}

int slimdp_layer_norm_backward(slimdp_ctx* ctx, uint32_t n_workers, const uint64_t* rows, uint64_t cols, uint32_t dtype,
                               const void* const* dy, uint64_t lddy, const void* const* x, uint64_t ldx, const float* const* weight,
                               const float* const* mean, const float* const* rstd, void* const* dx, uint64_t lddx,
                               float* const* dweight, float* const* dbias, uint32_t flags, void* workspace, uint64_t workspace_bytes)
{
    Call c;
    if (c.begin(ctx, "slimdp_layer_norm_backward", n_workers, rows, dtype)) return c.rc;
    if (flags & ~SLIMDP_GRAD_ACCUMULATE)
        return host_fail(ctx, SLIMDP_ERR_INVALID_ARG, "slimdp_layer_norm_backward: unknown flag bits 0x%x", flags);
    const bool sums = dweight || dbias;
    c.size("cols", cols, SLIMDP_MAX_NORM_COLS);
    c.matrix("dy", dy, lddy, cols, c.esize);
    c.matrix("x", x, ldx, cols, c.esize);
    c.matrix("mean", mean, 1, 1, 4);
    c.matrix("rstd", rstd, 1, 1, 4);
    c.matrix("dx", dx, lddx, cols, c.esize, true);
    c.params("weight", weight, 4, true);
    c.params("dweight", dweight, 4, true);
    c.params("dbias", dbias, 4, true);
    c.apart("dx", dx, "dy", dy, lddx == lddy);
    c.apart("dx", dx, "x", x, lddx == ldx);
    c.distinct("dx", dx, true);
    c.distinct("dweight", dweight, false);
    c.distinct("dbias", dbias, false);
    c.apart("dweight", dweight, "dbias", dbias, false, false);
    if (sums) c.workspace(workspace, workspace_bytes, slimdp_layer_norm_workspace_bytes(n_workers, rows, cols, dtype));
    if (!c.ok()) return c.rc;
    const NormBackArgs a{c.in(dy), c.in(x), c.in(weight), c.in(mean), c.in(rstd), c.out(dx), c.tab, lddy, ldx, lddx, (uint32_t)cols};
    const int accumulate = (flags & SLIMDP_GRAD_ACCUMULATE) != 0;
    const NormBackShape shape = norm_back_shape(c.W, rows, cols, c.esize);
    if (shape.tpr) {
        if (!sums && c.most == 0) return c.rc;
        const bool nt = c.bytes(cols, 3) > STREAM_BYTES;
        const NormBackSums o{c.out(dweight), c.out(dbias), sums && shape.blocks > 1 ? static_cast<float*>(workspace) : nullptr, accumulate};
        with_type(dtype, [&](auto z) {
            typedef decltype(z) T;
            auto launch = [&](auto kernel, auto kernel_nt) {
                c.launched("k_norm_back", [&] {
                    const dim3 grid((uint32_t)shape.blocks, c.W);
                    if (nt) hipLaunchKernelGGL(kernel_nt, grid, dim3(shape.block), 0, c.v.stream, a, o);
                    else hipLaunchKernelGGL(kernel, grid, dim3(shape.block), 0, c.v.stream, a, o);
                });
            };
            const uint64_t n = ceil_div(cols, Vec<T>::N);
#define SLIMDP_NORM_BACK(TPR, NC, BT) launch(k_norm_back<T, TPR, NC, BT, 0>, k_norm_back<T, TPR, NC, BT, 1>)
            if (shape.tpr == 8) SLIMDP_NORM_BACK(8, 1, 256);
            else if (shape.tpr == 16) SLIMDP_NORM_BACK(16, 1, 256);
            else if (shape.tpr == 32) SLIMDP_NORM_BACK(32, 1, 256);
            else if (shape.tpr == 64 && n <= 64) SLIMDP_NORM_BACK(64, 1, 256);
            else if (shape.tpr == 64) SLIMDP_NORM_BACK(64, 2, 256);
            else if (shape.tpr == 256 && n <= 256) SLIMDP_NORM_BACK(256, 1, 1024);
            else if (shape.tpr == 256) SLIMDP_NORM_BACK(256, 2, 1024);
            else if (shape.tpr == 512) SLIMDP_NORM_BACK(512, 2, 1024);
            else SLIMDP_NORM_BACK(1024, 2, 1024);
#undef SLIMDP_NORM_BACK
        });
        if (c.ok() && o.partial) column_sums(c, ColumnSumArgs{o.partial, o.dweight, o.dbias, c.tab, (uint32_t)cols, shape.block / shape.tpr, (uint32_t)shape.blocks, 2, accumulate});
        return c.rc;
    }
    if (sums) {      // before dx, which may overwrite dy or x
        ColumnArgs s{};
        s.a = a.dy; s.b = a.x; s.mean = a.mean; s.rstd = a.rstd;
        s.out0 = c.out(dweight); s.out1 = c.out(dbias);
        s.lda = lddy; s.ldb = ldx; s.cols = (uint32_t)cols;
        s.accumulate = accumulate;
        if (column_grads<true>(c, s, dtype, ACT_NONE, true, workspace)) return c.rc;
    }
    if (!dx || c.most == 0) return c.rc;
    with_type(dtype, [&](auto z) {
        typedef decltype(z) T;
        c.launched("k_norm_back_rows", [&] {
            hipLaunchKernelGGL(k_norm_back_rows<T>, dim3((uint32_t)std::min<uint64_t>(c.most, 65536), c.W), dim3(256), 0, c.v.stream, a);
        });
    });
    return c.rc;
}

uint64_t slimdp_linear_workspace_bytes(uint32_t n_workers, const uint64_t* rows, uint64_t in, uint64_t out, uint32_t dtype, uint32_t pass)
{
    if (!shape_ok(n_workers, rows) || in == 0 || in > SLIMDP_MAX_FEATURES || out == 0 || out > SLIMDP_MAX_FEATURES || dtype > SLIMDP_BF16 ||
        pass > SLIMDP_LINEAR_BACKWARD)
        return 0;
    const size_t es = dtype == SLIMDP_F32 ? 4 : 2;
    if (pass == SLIMDP_LINEAR_FORWARD) return forward_product(n_workers, rows, in, out, es).ws();
    if (pass == SLIMDP_LINEAR_EPILOGUE_BACKWARD) return column_ws(n_workers, rows, out, es, 1);
    return std::max(input_product(n_workers, rows, in, out, es).ws(), weight_product(n_workers, rows, in, out, es).ws());
}

int slimdp_linear(slimdp_ctx* ctx, uint32_t n_workers, const uint64_t* rows, uint64_t in, uint64_t out, uint32_t dtype,
                  const void* const* x, uint64_t ldx, const void* const* weight, uint64_t ldw, const float* const* bias,
                  uint32_t activation, const void* const* residual, uint64_t ldr, void* const* y, uint64_t ldy, void* const* z,
                  uint64_t ldz, void* workspace, uint64_t workspace_bytes)
{
    Call c;
    if (c.begin(ctx, "slimdp_linear", n_workers, rows, dtype)) return c.rc;
    if (activation >= ACTS) return host_fail(ctx, SLIMDP_ERR_INVALID_ARG, "slimdp_linear: unknown activation %u", activation);
    c.size("in", in, SLIMDP_MAX_FEATURES);
    c.size("out", out, SLIMDP_MAX_FEATURES);
    c.matrix("x", x, ldx, in, c.esize);
    c.matrix("weight", weight, ldw, in, c.esize);
    c.params("bias", bias, 4, true);
    c.matrix("residual", residual, ldr, out, c.esize, true);
    c.matrix("y", y, ldy, out, c.esize);
    c.matrix("z", z, ldz, out, c.esize, true);
    c.apart("y", y, "x", x);
    c.apart("z", z, "x", x);
    c.apart("y", y, "weight", weight);
    c.apart("z", z, "weight", weight);
    c.apart("z", z, "y", y);
    c.apart("z", z, "residual", residual);
    c.apart("y", y, "residual", residual, ldy == ldr);
    c.distinct("y", y, true);
    c.distinct("z", z, true);
    c.workspace(workspace, workspace_bytes, slimdp_linear_workspace_bytes(n_workers, rows, in, out, dtype, SLIMDP_LINEAR_FORWARD));
    const Product p = forward_product(c.W, rows, in, out, c.esize);
    tiles_fit(c, p);
    if (!c.ok()) return c.rc;
    GemmArgs a{};
    a.a = c.in(x); a.b = c.in(weight); a.bias = c.in(bias); a.residual = c.in(residual);
    a.c = c.out(y); a.z = c.out(z);
    a.lda = ldx; a.ldb = ldw; a.ldc = ldy; a.ldr = ldr; a.ldz = ldz;
    a.act = (int)activation;
    return product<false, false, 0>(c, a, p, dtype, workspace);
}

int slimdp_linear_epilogue_backward(slimdp_ctx* ctx, uint32_t n_workers, const uint64_t* rows, uint64_t out, uint32_t dtype,
                                    const void* const* dy, uint64_t lddy, const void* const* z, uint64_t ldz, uint32_t activation,
                                    void* const* dz, uint64_t lddz, float* const* dbias, uint32_t flags, void* workspace,
                                    uint64_t workspace_bytes)
{
    Call c;
    if (c.begin(ctx, "slimdp_linear_epilogue_backward", n_workers, rows, dtype)) return c.rc;
    if (activation >= ACTS) return host_fail(ctx, SLIMDP_ERR_INVALID_ARG, "slimdp_linear_epilogue_backward: unknown activation %u", activation);
    if (flags & ~SLIMDP_GRAD_ACCUMULATE)
        return host_fail(ctx, SLIMDP_ERR_INVALID_ARG, "slimdp_linear_epilogue_backward: unknown flag bits 0x%x", flags);
    c.size("out", out, SLIMDP_MAX_FEATURES);
    c.matrix("dy", dy, lddy, out, c.esize);
    c.matrix("z", z, ldz, out, c.esize, activation == ACT_NONE);
    c.matrix("dz", dz, lddz, out, c.esize, true);
    c.params("dbias", dbias, 4, true);
    c.apart("dz", dz, "dy", dy, lddz == lddy);
    c.apart("dz", dz, "z", z, lddz == ldz);
    c.distinct("dz", dz, true);
    c.distinct("dbias", dbias, false);
    if (dbias)
        c.workspace(workspace, workspace_bytes, slimdp_linear_workspace_bytes(n_workers, rows, 1, out, dtype, SLIMDP_LINEAR_EPILOGUE_BACKWARD));
    if (!c.ok() || (!dz && !dbias)) return c.rc;
    ColumnArgs s{};
    s.a = c.in(dy); s.b = c.in(z); s.dz = c.out(dz); s.out1 = c.out(dbias);
    s.lda = lddy; s.ldb = ldz; s.lddz = lddz; s.cols = (uint32_t)out;
    s.accumulate = (flags & SLIMDP_GRAD_ACCUMULATE) != 0;
    return column_grads<false>(c, s, dtype, (int)activation, dbias != nullptr, workspace);
}

int slimdp_linear_backward(slimdp_ctx* ctx, uint32_t n_workers, const uint64_t* rows, uint64_t in, uint64_t out, uint32_t dtype,
                           const void* const* dz, uint64_t lddz, const void* const* x, uint64_t ldx, const void* const* weight,
                           uint64_t ldw, void* const* dx, uint64_t lddx, float* const* dweight, uint32_t flags, void* workspace,
                           uint64_t workspace_bytes)
{
    Call c;
    if (c.begin(ctx, "slimdp_linear_backward", n_workers, rows, dtype)) return c.rc;
    if (flags & ~SLIMDP_GRAD_ACCUMULATE)
        return host_fail(ctx, SLIMDP_ERR_INVALID_ARG, "slimdp_linear_backward: unknown flag bits 0x%x", flags);
    c.size("in", in, SLIMDP_MAX_FEATURES);
    c.size("out", out, SLIMDP_MAX_FEATURES);
    c.matrix("dz", dz, lddz, out, c.esize);
    c.matrix("x", x, ldx, in, c.esize, !dweight);
    c.matrix("weight", weight, ldw, in, c.esize, !dx);
    c.matrix("dx", dx, lddx, in, c.esize, true);
    c.params("dweight", dweight, 4, true);
    c.apart("dx", dx, "dz", dz);
    c.apart("dx", dx, "x", x);
    c.apart("dx", dx, "weight", weight);
    c.distinct("dx", dx, true);
    c.distinct("dweight", dweight, false);
    const Product pi = input_product(n_workers, rows, in, out, c.esize), pw = weight_product(n_workers, rows, in, out, c.esize);
    if (c.ok() && dweight)
        for (uint32_t q = 0; q < n_workers; ++q)
            if (!dweight[q]) c.rc = host_fail(ctx, SLIMDP_ERR_INVALID_ARG, "slimdp_linear_backward: dweight[%u] is NULL", q);
    if (dx) tiles_fit(c, pi);
    if (dweight) tiles_fit(c, pw);
    c.workspace(workspace, workspace_bytes, std::max(dx ? pi.ws() : 0, dweight ? pw.ws() : 0));
    if (!c.ok()) return c.rc;
    if (dx) {
        GemmArgs a{};
        a.a = c.in(dz); a.b = c.in(weight); a.c = c.out(dx);
        a.lda = lddz; a.ldb = ldw; a.ldc = lddx;
        if (product<false, true, 1>(c, a, pi, dtype, workspace)) return c.rc;
    }
    if (dweight) {
        GemmArgs a{};
        a.a = c.in(dz); a.b = c.in(x); a.c = c.out(dweight);
        a.lda = lddz; a.ldb = ldx; a.ldc = in;
        a.k_is_rows = 1;
        a.accumulate = (flags & SLIMDP_GRAD_ACCUMULATE) != 0;
        product<true, true, 2>(c, a, pw, dtype, workspace);
    }
    return c.rc;
}

int slimdp_distill_loss(slimdp_ctx* ctx, uint32_t n_workers, const uint64_t* rows, uint64_t vocab, uint32_t dtype,
                        const void* const* logits, uint64_t ldl, uint64_t top, const uint32_t* const* index, const float* const* value,
                        uint64_t ldt, float temperature, const float* const* row_weight, float* const* loss, float* const* lse,
                        void* const* dlogits, uint64_t lddl)
{
    Call c;
    if (c.begin(ctx, "slimdp_distill_loss", n_workers, rows, dtype)) return c.rc;
    c.size("vocab", vocab, SLIMDP_MAX_VOCAB);
    if (c.ok() && top > SLIMDP_MAX_TEACHER)
        c.rc = host_fail(ctx, SLIMDP_ERR_OUT_OF_RANGE, "slimdp_distill_loss: top exceeds %u", SLIMDP_MAX_TEACHER);
    c.matrix("logits", logits, ldl, vocab, c.esize);
    if (top) {
        c.matrix("index", index, ldt, top, 4);
        c.matrix("value", value, ldt, top, 4);
    }
    c.matrix("row_weight", row_weight, 1, 1, 4, true);
    c.matrix("loss", loss, 1, 1, 4, true);
    c.matrix("lse", lse, 1, 1, 4, true);
    c.matrix("dlogits", dlogits, lddl, vocab, c.esize, true);
    c.apart("dlogits", dlogits, "logits", logits, lddl == ldl);
    c.distinct("dlogits", dlogits, true);
    c.distinct("loss", loss, true);
    c.distinct("lse", lse, true);
    c.apart("loss", loss, "lse", lse);
    if (c.ok() && !(temperature > 0.0f && std::isfinite(temperature) && std::isfinite(LOG2E / temperature)))
        c.rc = host_fail(ctx, SLIMDP_ERR_INVALID_ARG, "slimdp_distill_loss: temperature must be positive and finite");
    if (!c.ok() || c.most == 0) return c.rc;
    const DistillArgs a{c.in(logits), c.in(top ? index : nullptr), c.in(top ? value : nullptr), c.in(row_weight), c.out(loss), c.out(lse),
                        c.out(dlogits), c.tab, ldl, ldt, lddl, (uint32_t)vocab, (uint32_t)top, temperature, c.v.status};
    const uint64_t rows_bytes = c.bytes(vocab, 2);
    with_type(dtype, [&](auto z) {
        typedef decltype(z) T;
        const uint64_t n = ceil_div(vocab, Vec<T>::N);
        auto launch = [&](auto kernel, uint32_t block) {
            c.launched("k_distill", [&] {
                hipLaunchKernelGGL(kernel, dim3((uint32_t)std::min<uint64_t>(c.most, 65536), c.W), dim3(block), 0, c.v.stream, a);
            });
        };
        // the smallest block that holds the row, without a second entry for any thread where the lists are short.  Logits and gradients
        // pass the caches by where they do not fit them: 4 x 1024 rows of 128,000 bf16 (2.1 GB) 533 -> 496 us with stores, 552 without
        // loads that do; but 8 x 4096 rows of 1,000 (131 MB) 62 -> 70.
        const bool nt = rows_bytes > STREAM_BYTES;
#define SLIMDP_DISTILL_NT(BT, HELD, MINE)                                                         \
    do { if (nt) launch(k_distill<T, BT, HELD, MINE, 1>, BT); else launch(k_distill<T, BT, HELD, MINE, 0>, BT); } while (0)
#define SLIMDP_DISTILL(BT, HELD)                                                                  \
    do {                                                                                          \
        if (top <= BT) SLIMDP_DISTILL_NT(BT, HELD, 1);                                            \
        else SLIMDP_DISTILL_NT(BT, HELD, (int)(SLIMDP_MAX_TEACHER + BT - 1) / BT);                \
    } while (0)
        if (!dlogits && n <= 2048) SLIMDP_DISTILL(256, 0);
        else if (!dlogits || n > 16384) SLIMDP_DISTILL(512, 0);
        else if (n <= 512) SLIMDP_DISTILL(128, 4);
        else if (n <= 1024) SLIMDP_DISTILL(256, 4);
        else if (n <= 2048) SLIMDP_DISTILL(256, 8);
        else if (n <= 4096) SLIMDP_DISTILL(512, 8);
        else if (n <= 8192) SLIMDP_DISTILL(512, 16);
        else SLIMDP_DISTILL_NT(1024, 16, 1);
#undef SLIMDP_DISTILL
#undef SLIMDP_DISTILL_NT
    });
    return c.rc;
}

}  // extern "C"
