// Matrix products in binary32 by tiles that pass through registers.  Included only by slimdp_train.hip.
#pragma once
#include "slimdp_linear.h"

namespace slimdp {

constexpr uint32_t GEMM32_BK = 32;

// One operand's tile of a step: X rows (or columns) of the product by 32 of k.
//   k running:  X rows of 128 bytes in the LDS, their eight vectors exchanged by the row's number
//   KROWS:      32 rows of X elements as they lie in memory, their pieces of 16 elements exchanged by every fourth row's number
// so that what a wave reads at once lies in different banks.  A vector's place in memory is any that a float may have.
template <bool KROWS, uint32_t X> struct Tile32 {
    static constexpr uint32_t BYTES = X * 128, LOADS = X < 32 ? 1 : X / 32, PER_ROW = X / 4;
    static constexpr uint32_t TURN = X / 16 > 4 ? 3 : X / 16 - 1;

    const float* base[LOADS];          // the thread's vectors of a step at k = 0, rows and columns outside the matrix replaced by the last
    uint64_t ld;
    uint32_t x[LOADS], k[LOADS];       // their place in the tile
    uint32_t down[KROWS ? LOADS : 1];  // elements by which a vector taken from the row's end is moved

    __device__ __forceinline__ void init(const void* pp, uint64_t ldd, uint32_t x0, uint32_t limit)
    {
        const float* p = static_cast<const float*>(pp);
        ld = ldd;
#pragma unroll
        for (uint32_t i = 0; i < LOADS; ++i) {
            const uint32_t v = (threadIdx.x + 256u * i) % (X * 8);
            if (KROWS) {
                k[i] = v / PER_ROW;
                x[i] = v % PER_ROW * 4;
                const uint32_t c = x0 + x[i], at = min(c, limit - 4);
                base[i] = p + (uint64_t)k[i] * ld + at;
                down[i] = c < limit ? c - at : 0u;
            } else {
                x[i] = v >> 3;
                k[i] = (v & 7u) * 4;
                base[i] = p + (uint64_t)min(x0 + x[i], limit - 1) * ld + k[i];
            }
        }
    }
    // Vector i of the whole step at kb, and of any step: from a place inside the matrix (K: the piece's end, Kall: the row's).
    __device__ __forceinline__ raw4 load(uint32_t i, uint32_t kb) const { return load_raw<float>(base[i] + (KROWS ? kb * ld : kb)); }
    __device__ __forceinline__ raw4 load(uint32_t i, uint32_t kb, uint32_t K, uint32_t Kall) const
    {
        if (KROWS) return load_raw<float>(base[i] + ((int64_t)min(kb + k[i], K - 1) - (int64_t)k[i]) * (int64_t)ld);
        return load_raw<float>(base[i] + ((int64_t)min(kb + k[i], Kall - 4) - (int64_t)k[i]));
    }
    __device__ __forceinline__ void write(uint32_t i, raw4 v, char* lds, uint32_t kb, uint32_t K, bool broken) const
    {
        const uint32_t at = kb + k[i];
        if (KROWS) {
            if (down[i]) v = move_down<float>(v, down[i]);
            if (broken && at >= K) v = raw4{0, 0, 0, 0};
            *reinterpret_cast<raw4*>(lds + k[i] * (X * 4) + ((x[i] ^ ((k[i] >> 2 & TURN) << 4)) << 2)) = v;
        } else {
            if (broken) {
                if (at < K && at + 4 > K) v = move_down<float>(v, at + 4 - K);
                if (at >= K) v = raw4{0, 0, 0, 0};
            }
            *reinterpret_cast<raw4*>(lds + x[i] * 128 + ((k[i] >> 2 ^ (x[i] >> 1 & 7u)) << 4)) = v;
        }
    }
    // What a lane holds of 16 rows (xx .. xx + 15) by 16 of k for four instructions: row lane & 15, four of k from 4 * (lane >> 4).
    static __device__ __forceinline__ raw4 fragment(const char* lds, uint32_t xx, uint32_t half)
    {
        const uint32_t lane = threadIdx.x & 63u, r = xx + (lane & 15u), g = half * 4 + (lane >> 4);
        if (!KROWS) return *reinterpret_cast<const raw4*>(lds + r * 128 + ((g ^ (r >> 1 & 7u)) << 4));
        const char* q = lds + g * 4 * (X * 4) + ((r ^ ((g & TURN) << 4)) << 2);
        raw4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = *reinterpret_cast<const uint32_t*>(q + e * (X * 4));
        return v;
    }
};

// BM x BN of C a block of WM x WN waves, 32 of k a step, in 16 x 16 accumulators.  The matrix unit takes 1,024 cycles for a step of a
// wave of a 64 x 64 tile, so everything else has time beside it: a step's vectors are asked for three steps ahead, wait in registers for two,
// and go to the other half of the LDS while a step is multiplied; fragments are read half a step ahead; one barrier a step, in its middle.
// Reads, copies and loads are put between the products one by one, and loads are made without a condition but in the last steps.  Operands
// with rows of k stay as they lie (a kernel that turned them over in registers took 741 us for the weight's gradient of 2048 x 4096 x 4096, this
// one 524).
//
// LONG: every 256 of k the sums go over to a second set, so that no chain of additions is longer than 13 steps (2048 x 4096 x 2048: error 3.0e-7 of
// the result's size, 1.15e-6 in one chain, which is what a library product has).  The second set takes 16 registers of 64 x 64's
// waves, three instead of four a SIMD: sums of 256 and less do without (8 x 40 x 1040 x 7692's weight gradient, which its stores bound,
// 117 us instead of 127; 2048 x 4096 x 4096 the same either way).
//
// Bound by the matrix unit: 2048 x 4096 x 4096 522 us (132 TFLOP/s; a library product 531 on that machine, 465 on another), 1024 x 1024 x 1024
// 25 us (24).  Tiles are no larger than 64 x 64 or 128 x 32 because more blocks leave less of the last round empty (1529 x 832 x 3119: 92 us
// with 128 x 64, 78 with 64 x 64), and narrower where the result is or where it ends a little behind a tile (11,202 x 2480 x 321: 167 us with
// 128 x 32, 195 with 32 x 64): 13,286 x 6638 x 16 80 us with 64 x 16 (155 with the square tiles of an earlier kernel); 24 x 3592 x 4608 22 us
// with 32 x 64.  Few rows are bound by memory, and so is what has few of k.
// grid: a.blocks, over two dimensions where one does not number them
template <bool AK, bool BK_, int EPI, uint32_t BM, uint32_t BN, uint32_t WM, uint32_t WN, bool LONG>
__global__ __launch_bounds__(256, LONG && BM * BN == 4096 ? 3 : 4) void k_gemm32(GemmArgs a)
{
    constexpr uint32_t MT = BM / WM, NT = BN / WN, FM = MT / 16, FN = NT / 16, BK = GEMM32_BK;
    typedef Tile32<AK, BM> TA;
    typedef Tile32<BK_, BN> TB;
    constexpr uint32_t LA = TA::LOADS, LB = TB::LOADS;
    __shared__ __attribute__((aligned(1024))) char lds[2 * (TA::BYTES + TB::BYTES)];

    const uint32_t unit = blockIdx.y * gridDim.x + blockIdx.x;
    if (unit >= a.blocks) return;
    const Share of = share_of(a, unit);
    const uint32_t q = of.q;
    const uint32_t M = a.k_is_rows ? a.M : a.rows.n[q], N = a.N, Kall = a.k_is_rows ? a.rows.n[q] : a.K;
    const uint32_t across = (N + BN - 1) / BN, down = (M + BM - 1) / BM, tiles = across * down;
    // Blocks go round the eight dies in turn: of every worker a die gets consecutive tiles (workers may differ in what a tile takes), and
    // takes them eight rows of tiles at a time, so that what its blocks read at one time lies in few rows and columns.
    const uint32_t mine = unit - of.begin, die = mine & 7u;
    const uint32_t place_in = die * (of.count >> 3) + min(die, of.count & 7u) + (mine >> 3);
    const uint32_t split = place_in / tiles, tt = place_in % tiles;
    const uint32_t group = tt / (8 * across), in_group = tt % (8 * across), high = min(8u, down - group * 8);
    const uint32_t m0 = (group * 8 + in_group % high) * BM, n0 = in_group / high * BN;
    const uint32_t k0 = min(Kall, split * a.k_split), K = min(Kall, k0 + a.k_split), steps = (K - k0 + BK - 1) / BK;
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, wm = wave / WN, wn = wave % WN;

    f32x4 acc[FM][FN], sum[LONG ? FM : 1][LONG ? FN : 1];
    auto carry = [&]() {
        if constexpr (LONG)
#pragma unroll
            for (uint32_t i = 0; i < FM; ++i)
#pragma unroll
                for (uint32_t j = 0; j < FN; ++j) {
                    sum[i][j] += acc[i][j];
                    acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
                }
    };
#pragma unroll
    for (uint32_t i = 0; i < FM; ++i)
#pragma unroll
        for (uint32_t j = 0; j < FN; ++j) {
            acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
            if constexpr (LONG) sum[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
    if (steps) {
        TA ta;
        TB tb;
        ta.init(a.a.p[q], a.lda, m0, M);
        tb.init(a.b.p[q], a.ldb, n0, N);
        raw4 ra[2][LA], rb[2][LB], fa[2][FM], fb[2][FN];
        auto place = [&](uint32_t s) { return lds + (s & 1u) * (TA::BYTES + TB::BYTES); };
        auto load = [&](uint32_t s, auto r) {
            constexpr uint32_t R = decltype(r)::value;
#pragma unroll
            for (uint32_t i = 0; i < LA; ++i) ra[R][i] = ta.load(i, k0 + s * BK, K, Kall);
#pragma unroll
            for (uint32_t i = 0; i < LB; ++i) rb[R][i] = tb.load(i, k0 + s * BK, K, Kall);
        };
        auto read = [&](uint32_t s, auto h, uint32_t i) {
            constexpr uint32_t H = decltype(h)::value;
            const char* at = place(s);
            if (i < FM) fa[H][i] = TA::fragment(at, wm * MT + i * 16, H);
            else fb[H][i - FM] = TB::fragment(at + TA::BYTES, wn * NT + (i - FM) * 16, H);
        };
        constexpr std::integral_constant<uint32_t, 0> c0{};
        constexpr std::integral_constant<uint32_t, 1> c1{};
        auto barrier = [&]() {
            asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
            __builtin_amdgcn_sched_barrier(0);
        };
        // The products of half a step, with the given operations between them one by one.
        constexpr uint32_t P = FM * FN * 4;
        auto products = [&](auto h, auto count, auto&& op) {
            constexpr uint32_t H = decltype(h)::value, C = decltype(count)::value, EACH = (C + P - 1) / P;
#pragma unroll
            for (uint32_t n = 0; n < P; ++n) {
#pragma unroll
                for (uint32_t o = n * EACH; o < (n + 1) * EACH && o < C; ++o) op(o);
                const uint32_t e = n / (FM * FN), i = n / FN % FM, j = n % FN;
                // B first: a lane then holds four consecutive columns of one row of C
                acc[i][j] = Mma<float>::part(fb[H][j], fa[H][i], acc[i][j], (int)e);
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        // Step s; r: which registers hold the step after it.  FULL: that step and the one three ahead exist.
        auto step = [&](uint32_t s, auto r, auto full) {
            constexpr uint32_t R = decltype(r)::value;
            constexpr bool FULL = decltype(full)::value;
            const bool more = FULL || s + 1 < steps;
            const uint32_t kb = k0 + (s + 1) * BK;
            const bool broken = !FULL && kb + BK > K;
            char* to = place(s + 1);
            constexpr std::integral_constant<uint32_t, FM + FN + (FULL ? 2 * (LA + LB) : 0)> first_ops{};
            products(c0, first_ops, [&](uint32_t o) {
                if (o < FM + FN) { read(s, c1, o); return; }
                o -= FM + FN;
                if (o & 1u) {                   // ... and its registers take the step three ahead
                    o >>= 1;
                    if (o < LA) ra[R][o] = ta.load(o, kb + 2 * BK);
                    else rb[R][o - LA] = tb.load(o - LA, kb + 2 * BK);
                } else {
                    o >>= 1;
                    if (o < LA) ta.write(o, ra[R][o], to, kb, K, false);
                    else tb.write(o - LA, rb[R][o - LA], to + TA::BYTES, kb, K, false);
                }
            });
            if (!FULL && more) {
#pragma unroll
                for (uint32_t i = 0; i < LA; ++i) ta.write(i, ra[R][i], to, kb, K, broken);
#pragma unroll
                for (uint32_t i = 0; i < LB; ++i) tb.write(i, rb[R][i], to + TA::BYTES, kb, K, broken);
                if (s + 3 < steps) load(s + 3, r);
            }
            barrier();
            constexpr std::integral_constant<uint32_t, FM + FN> second_ops{};
            products(c1, second_ops, [&](uint32_t o) { if (more) read(s + 1, c0, o); });
        };
        load(0, c0);
        if (steps > 1) load(1, c1);
#pragma unroll
        for (uint32_t i = 0; i < LA; ++i) ta.write(i, ra[0][i], place(0), k0, K, k0 + BK > K);
#pragma unroll
        for (uint32_t i = 0; i < LB; ++i) tb.write(i, rb[0][i], place(0) + TA::BYTES, k0, K, k0 + BK > K);
        if (steps > 2) load(2, c0);
        barrier();
#pragma unroll
        for (uint32_t i = 0; i < FM + FN; ++i) read(0, c0, i);
        uint32_t s = 0;
        // steps whose next ones and those three ahead are whole
#pragma unroll 1
        for (; s + 5 < steps; s += 2) {
            step(s, c1, std::true_type{});
            step(s + 1, c0, std::true_type{});
            if ((s & 6u) == 6u) carry();
        }
#pragma unroll 1
        for (; s < steps; s += 2) {
            step(s, c1, std::false_type{});
            if (s + 1 < steps) step(s + 1, c0, std::false_type{});
        }
    }
    if constexpr (LONG) {
        carry();
#pragma unroll
        for (uint32_t i = 0; i < FM; ++i)
#pragma unroll
            for (uint32_t j = 0; j < FN; ++j) acc[i][j] = sum[i][j];
    }
#pragma unroll
    for (uint32_t i = 0; i < FM; ++i) {
        const uint32_t m = m0 + wm * MT + i * 16 + (lane & 15u);
        if (m >= M) continue;
#pragma unroll
        for (uint32_t j = 0; j < FN; ++j) {
            const uint32_t n = n0 + wn * NT + j * 16 + (lane >> 4) * 4;
            if (n >= N) continue;
            const float v[4] = {acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]};
            if (a.splits == 1) epilogue4<float, EPI>(a, q, m, n, N, v);
            else store4(a.partial + (((size_t)q * a.splits + split) * a.M + m) * N + n, N - n, v);
        }
    }
}

}  // namespace slimdp
