// Matrix products of sixteen-bit elements by tiles that go from memory to the LDS without passing through registers.
// Included only by slimdp_train.hip.
#pragma once
#include "slimdp_linear.h"

namespace slimdp {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t raw2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) void lds_void;
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

template <class T> __device__ __forceinline__ f32x16 mma32(raw4 a, raw4 b, f32x16 c);
template <> __device__ __forceinline__ f32x16 mma32<_Float16>(raw4 a, raw4 b, f32x16 c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
template <> __device__ __forceinline__ f32x16 mma32<__bf16>(raw4 a, raw4 b, f32x16 c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

constexpr uint32_t GEMM_BK = 64;

// Starts the copy of a vector a lane, from r at the lane's offset to the LDS at place + 16 * lane.  Written as assembly so that the
// compiler, which cannot tell one place in the LDS from another, does not wait for every copy under way before each read that turns rows
// over (products with such an operand: 2.0 to 2.4 us a step instead of 1.5); the kernel waits by itself.  place and r come from scalar
// instructions; a write of m0 is one instruction ahead of its use (the compiler keeps nothing in m0 of its own here: reads of the LDS need none).
__device__ __forceinline__ void copy_to_lds(raw4 r, uint32_t place, uint32_t offset)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" :: "s"(place), "v"(offset), "s"(r) : "memory");
}

// One operand's tile of a step: X rows (or columns) of the product by 64 of k, as it lies in memory.
//   k running:      X rows of 128 bytes (whole lines), their eight vectors exchanged by the row's number
//   KROWS:          64 rows of 2 X bytes, their pieces of 64 bytes exchanged by two or three bits of the row's number
// so that what a wave reads at once lies in different banks.  The copy into the LDS writes a wave's 64 vectors one after the
// other, so the exchange is made by what each lane asks for.  Vectors outside the matrix are asked for behind the descriptor's end, and
// arrive as zeros.
//
// DIRECT: by copies from memory to the LDS, for operands whose vectors lie on their own alignment.  Otherwise through registers, a
// step ahead of the LDS, from any address: loads past an edge are made from the last row or vector inside, and what they bring to rows and
// columns that are not kept does no harm; a last step that k does not fill is written by itself, with zeros (tail).
template <bool KROWS, uint32_t X, uint32_t WAVES, bool DIRECT, class T> struct Tile {
    static constexpr uint32_t BYTES = X * 2 * GEMM_BK, LOADS = BYTES / 1024 / WAVES;
    static constexpr uint32_t OUT = 0x80000000u;
    static constexpr uint32_t PER_ROW = X / 8, ROWS_A_LOAD = 64 / PER_ROW;           // KROWS: vectors of a row, rows of a load

    static constexpr uint32_t PART = LOADS * 1024;   // a wave's copies of a tile

    const char* base;            // first row (k running) or first column (KROWS) of the tile
    uint32_t off[LOADS], k[LOADS];
    uint64_t step;
    // through registers
    raw4 reg[DIRECT ? 1 : LOADS];
    uint32_t down[DIRECT || !KROWS ? 1 : LOADS];     // elements by which a vector taken from the row's end is to be moved
    bool edge;                                       // ... of any lane of the block
    const T* p;
    uint64_t ld;
    uint32_t x0, limit;

    static __device__ __forceinline__ uint32_t turn(uint32_t k) { return ((k & 3u) | ((k >> 1) & 4u)) & (X / 32 - 1); }
    // Vector i of a lane: row of the tile in the LDS, and where it begins in it, in elements.
    static __device__ __forceinline__ void place_of(uint32_t i, uint32_t& r, uint32_t& e)
    {
        const uint32_t lane = threadIdx.x & 63u, piece = (threadIdx.x >> 6) * LOADS + i;
        if (KROWS) {
            r = piece * ROWS_A_LOAD + lane / PER_ROW;
            e = ((lane % PER_ROW) ^ (turn(r) << 2)) * 8;
        } else {
            r = piece * 8 + (lane >> 3);
            e = ((lane & 7u) ^ ((r >> 1) & 7u)) * 8;
        }
    }

    // full: whether there is a whole step
    __device__ __forceinline__ void init(const void* pp, uint64_t ldd, uint32_t x, uint32_t lim, uint32_t k0, bool full)
    {
        p = static_cast<const T*>(pp);
        ld = ldd;
        x0 = x;
        limit = lim;
        const uint32_t left = limit - x0;
        edge = left < X && limit % 8;
        base = reinterpret_cast<const char*>(p + (KROWS ? (uint64_t)k0 * ld + x0 : (uint64_t)x0 * ld + k0));
        step = KROWS ? GEMM_BK * ld * 2 : GEMM_BK * 2;
        if (!DIRECT && !full) {
            base = reinterpret_cast<const char*>(p);
            step = 0;
        }
#pragma unroll
        for (uint32_t i = 0; i < LOADS; ++i) {
            uint32_t r, e;
            place_of(i, r, e);
            if (DIRECT) {
                off[i] = (KROWS ? e : r) < left ? (uint32_t)(r * ld * 2) + e * 2 : OUT;
                k[i] = KROWS ? r : e;
            } else if (KROWS) {
                // the last vector inside where the tile's columns end (it may begin before the tile: then x0 >= 8 - left)
                const bool inside = e + 8 <= left;
                down[i] = !inside && e < left ? e + 8 - left : 0u;
                off[i] = full ? (uint32_t)(r * ld * 2) + (inside ? e : left >= 8 ? left - 8 : 0u) * 2 : 0u;
                if (!inside && left < 8) down[i] = 0;
            } else {
                off[i] = full ? (uint32_t)(min(r, left - 1) * ld * 2) + e * 2 : 0u;
            }
        }
        if (!DIRECT && KROWS && left < 8) {
            // fewer columns than a vector are left: take it from before the tile
            base -= (full ? 8 - left : 0) * 2;
#pragma unroll
            for (uint32_t i = 0; i < LOADS; ++i) {
                uint32_t r, e;
                place_of(i, r, e);
                down[i] = e == 0 ? 8 - left : 0u;
            }
        }
    }
    __device__ __forceinline__ void load(uint32_t i) { reg[i] = load_raw<T>(reinterpret_cast<const T*>(base + off[i])); }
    // Vector i into its place (place: this wave's part, in bytes from the LDS's start).
    __device__ __forceinline__ void write(uint32_t i, char* lds, uint32_t place)
    {
        raw4 v = reg[i];
        if constexpr (KROWS)
            if (edge && down[i]) v = move_down<T>(v, down[i]);
        *reinterpret_cast<raw4*>(lds + place + i * 1024 + (threadIdx.x & 63u) * 16) = v;
    }
    // The step that begins at kb and that k does not fill.
    __device__ __forceinline__ void tail(char* lds, uint32_t place, uint32_t kb, uint32_t K) const
    {
#pragma unroll 1
        for (uint32_t i = 0; i < LOADS; ++i) {
            uint32_t r, e;
            place_of(i, r, e);
            const uint32_t kk = kb + (KROWS ? r : e), x = x0 + (KROWS ? e : r);
            raw4 v = {0, 0, 0, 0};
            if (kk < K && x < limit) v = KROWS ? load_clip(p + (uint64_t)kk * ld, x, limit) : load_clip(p + (uint64_t)x * ld, kk, K);
            *reinterpret_cast<raw4*>(lds + place + i * 1024 + (threadIdx.x & 63u) * 16) = v;
        }
    }
    // Copy i of the tile at k0 + the steps made so far; kleft: how much of k is left from there.  place: this wave's part.
    __device__ __forceinline__ void fetch(uint32_t i, uint32_t place, uint32_t kleft) const
    {
        const uint64_t at = reinterpret_cast<uint64_t>(base);
        const raw4 r = {(uint32_t)at, (uint32_t)(at >> 32) & 0xFFFFu, OUT, 0x00020000u};
        copy_to_lds(r, place + i * 1024, k[i] < kleft ? off[i] : OUT);
    }
    __device__ __forceinline__ void next() { base += step; }
    // What a lane holds of 32 rows (x .. x + 31) by 16 of k for one instruction: row lane & 31, eight of k from 8 * (lane >> 5).
    static __device__ __forceinline__ raw4 fragment(const char* lds, uint32_t x, uint32_t ks)
    {
        const uint32_t lane = threadIdx.x & 63u;
        if (!KROWS) {
            const uint32_t r = x + (lane & 31u), c = ks * 2 + (lane >> 5);
            return *reinterpret_cast<const raw4*>(lds + r * 128 + ((c ^ ((r >> 1) & 7u)) << 4));
        } else {
            // sixteen lanes read four rows of sixteen elements and get them turned over
            const uint32_t g = lane >> 4, i = lane & 15u;
            const uint32_t kr = ks * 16 + (g >> 1) * 8 + (i >> 2), b = (x + (g & 1u) * 16 + (i & 3u) * 4) * 2;
            const char* p = lds + kr * (X * 2);
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + (b ^ (turn(kr) << 6))));
            const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + 4 * (X * 2) + (b ^ (turn(kr) << 6))));
            const raw2 l = __builtin_bit_cast(raw2, lo), h = __builtin_bit_cast(raw2, hi);
            return raw4{l.x, l.y, h.x, h.y};
        }
    }
};

// What becomes of a column of eight consecutive places in ROWS rows of the sum (first row m, dm apart): everything that is read for them
// is asked for before the first is used.  Rows outside the product are neither read nor written.
template <class T, int EPI, int ROWS>
__device__ __forceinline__ void epilogue8(const GemmArgs& a, char* c, const T* res, T* z, const float (&bias)[8], uint32_t m, uint32_t dm, uint32_t M,
                                          uint32_t n, uint32_t N, float (&v)[ROWS][8])
{
    const bool whole = n + 8 <= N;
    if constexpr (EPI == 2) {
        float* out = reinterpret_cast<float*>(c);
        if (a.accumulate) {
            float old[ROWS][8];
#pragma unroll
            for (int r = 0; r < ROWS; ++r)
                if (m + r * dm < M) load_params<8>(out + (size_t)(m + r * dm) * a.ldc, n, N, old[r]);
#pragma unroll
            for (int r = 0; r < ROWS; ++r)
#pragma unroll
                for (int i = 0; i < 8; ++i) v[r][i] += old[r][i];
        }
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            if (m + r * dm >= M) continue;
            float* o = out + (size_t)(m + r * dm) * a.ldc + n;
#pragma unroll
            for (int i = 0; i < 8; i += 4) {
                if (whole) {
                    raw4 w;
#pragma unroll
                    for (int j = 0; j < 4; ++j) w[j] = __float_as_uint(v[r][i + j]);
                    store_raw<float>(o + i, w);
                } else {
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (n + i + j < N) o[i + j] = v[r][i + j];
                }
            }
        }
    } else {
        raw4 add[ROWS];
        if (EPI == 0 && res)
#pragma unroll
            for (int r = 0; r < ROWS; ++r)
                if (m + r * dm < M) add[r] = load_clip(res + (size_t)(m + r * dm) * a.ldr, n, N);
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            if (m + r * dm >= M) continue;
            if constexpr (EPI == 0) {
#pragma unroll
                for (int i = 0; i < 8; ++i) v[r][i] += bias[i];
                if (z) store_clip(z + (size_t)(m + r * dm) * a.ldz, n, N, pack<T>(v[r]));
                act_values(v[r], a.act);
                if (res) {
                    float f[8];
                    unpack<T>(add[r], f);
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[r][i] += f[i];
                }
            }
            store_clip(reinterpret_cast<T*>(c) + (size_t)(m + r * dm) * a.ldc, n, N, pack<T>(v[r]));
        }
    }
}

// BM x BN of C a block of WM x WN waves, 64 of k a step.  A step is four products' worth (16 of k each), in which a wave multiplies
// what it has in registers while it reads the next from the LDS.  B's part of a step is in registers after the first quarter; its place
// in the LDS is then free for the step after next, while A has three places in turn: every copy has one and a half steps to arrive.  (With
// two places for either, filled at the end of a step and waited for at the end of the next, the wait took a quarter of the time.)
// Reads and copies are put between the products one by one: the compiler by itself puts the products first and then waits for the reads.
// Sums leave through the LDS, WM parts one after the other, so that memory sees whole rows.
// BLOCKS share a compute unit: one of 256 x 256, or two of 128 x 128.
// grid: a.blocks, over two dimensions where one does not number them; which tile a block takes goes by the die it runs
// on (see below).
template <class T, bool AK, bool BK_, int EPI, uint32_t BM, uint32_t BN, uint32_t WM, uint32_t WN, uint32_t BLOCKS, bool DIRECT>
__global__ __launch_bounds__(WM * WN * 64, BLOCKS) void k_gemm_tiles(GemmArgs a)
{
    constexpr uint32_t WAVES = WM * WN, MT = BM / WM, NT = BN / WN, FM = MT / 32, FN = NT / 32;
    typedef Tile<AK, BM, WAVES, DIRECT, T> TA;
    typedef Tile<BK_, BN, WAVES, DIRECT, T> TB;
    constexpr uint32_t PLACES = 3 * TA::BYTES + 2 * TB::BYTES, ROW = BN * 4 + 16, OUT_BYTES = MT * ROW;
    constexpr uint32_t LDS = PLACES > OUT_BYTES ? PLACES : OUT_BYTES;
    __shared__ __attribute__((aligned(1024))) char lds[LDS];

    // Blocks go round the eight dies in turn: a die gets consecutive tiles (of consecutive workers), and takes them eight rows of
    // tiles at a time, so that what its blocks read at one time lies in few rows and columns.  Where a tile of one worker takes longer than
    // another's (a.spread) every die gets its share of every worker instead.  Only tiles that exist are numbered: a worker without rows
    // leaves no die idle (16,384 x 4096 x 4096 bf16, one worker of eight has all the rows: 450 us; 2,770 where every worker had the tiles of the largest).
    const uint32_t id = blockIdx.y * gridDim.x + blockIdx.x;
    if (id >= a.blocks) return;
    auto dealt = [](uint32_t n, uint32_t count) {
        const uint32_t die = n & 7u;
        return die * (count >> 3) + min(die, count & 7u) + (n >> 3);
    };
    const uint32_t unit = a.spread ? id : dealt(id, a.blocks);
    const Share of = share_of(a, unit);
    const uint32_t q = of.q, local = a.spread ? dealt(unit - of.begin, of.count) : unit - of.begin;
    const uint32_t M = a.k_is_rows ? a.M : a.rows.n[q], N = a.N, Kall = a.k_is_rows ? a.rows.n[q] : a.K;
    const uint32_t across = (N + BN - 1) / BN, down = (M + BM - 1) / BM, tiles = across * down;
    const uint32_t split = local / tiles, tt = local % tiles;
    const uint32_t group = tt / (8 * across), in_group = tt % (8 * across), high = min(8u, down - group * 8);
    const uint32_t m0 = (group * 8 + in_group % high) * BM, n0 = in_group / high * BN;
    const uint32_t k0 = min(Kall, split * a.k_split), K = min(Kall, k0 + a.k_split);
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, wm = wave / WN, wn = wave % WN;

    TA ta;
    TB tb;
    const uint32_t whole = (K - k0) / GEMM_BK, steps = (K - k0 + GEMM_BK - 1) / GEMM_BK;
    ta.init(a.a.p[q], a.lda, m0, M, k0, whole != 0);
    tb.init(a.b.p[q], a.ldb, n0, N, k0, whole != 0);
    f32x16 acc[FM][FN];
#pragma unroll
    for (uint32_t i = 0; i < FM; ++i)
#pragma unroll
        for (uint32_t j = 0; j < FN; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;
    raw4 fa[2][FM], fb[4][FN];
    if (k0 < K) {
        const uint32_t first = DIRECT ? (uint32_t)(uintptr_t)(lds_void*)lds : 0u, mine = __builtin_amdgcn_readfirstlane(wave);
        const uint32_t first_b = first + 3 * TA::BYTES, my_a = first + mine * TA::PART, my_b = first_b + mine * TB::PART;
        const char* const lds_b = lds + 3 * TA::BYTES;
        // what is left of k where the next copies begin; behind the end zeros are copied, so that every step waits for the same number
        auto left = [&](uint32_t kb) { return kb < K ? K - kb : 0u; };
        auto read_a = [&](uint32_t tile, uint32_t ks, uint32_t i) { fa[ks & 1][i] = TA::fragment(lds + tile, wm * MT + i * 32, ks); };
        auto read_b = [&](uint32_t tile, uint32_t ks, uint32_t j) { fb[ks][j] = TB::fragment(lds_b + tile, wn * NT + j * 32, ks); };
        // A quarter of a step: the products of ks, with the reads of A's next quarter, of B's from kb on and the copies between them.
        // B first in the product: a lane then holds four consecutive columns of one row of C at a time.
        auto quarter = [&](auto ks, uint32_t a_tile, uint32_t b_tile, auto bs, auto nb, auto na_copies, auto nb_copies, uint32_t a_place, uint32_t b_place,
                           uint32_t kleft) {
            constexpr uint32_t KS = decltype(ks)::value, RB = decltype(nb)::value * FN, R = RB + FM, CA = decltype(na_copies)::value, CB = decltype(nb_copies)::value;
            constexpr uint32_t P = FM * FN, EACH = (R + CA + CB + P - 1) / P;
#pragma unroll
            for (uint32_t p = 0; p < P; ++p) {
#pragma unroll
                for (uint32_t o = p * EACH; o < (p + 1) * EACH; ++o) {
                    if (o < FM) read_a(a_tile, (KS + 1) & 3u, o);
                    else if (o < R) read_b(b_tile, decltype(bs)::value + (o - FM) / FN, (o - FM) % FN);
                    else if (o < R + CA) {
                        if constexpr (DIRECT) ta.fetch(o - R, a_place, kleft);
                        else { ta.write(o - R, lds, a_place); ta.load(o - R); }
                    } else if (o < R + CA + CB) {
                        if constexpr (DIRECT) tb.fetch(o - R - CA, b_place, kleft);
                        else { tb.write(o - R - CA, lds, b_place); tb.load(o - R - CA); }
                    }
                }
                acc[p / FN][p % FN] = mma32<T>(fb[KS][p % FN], fa[KS & 1][p / FN], acc[p / FN][p % FN]);
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        constexpr std::integral_constant<uint32_t, 0> c0{};
        constexpr std::integral_constant<uint32_t, 1> c1{};
        constexpr std::integral_constant<uint32_t, 2> c2{};
        constexpr std::integral_constant<uint32_t, 3> c3{};
        constexpr std::integral_constant<uint32_t, TA::LOADS> copies_a{};
        constexpr std::integral_constant<uint32_t, TB::LOADS> copies_b{};
        // through registers: where the next loads come from, the last whole step's place once there is no other
        uint32_t loaded = 0;
        auto onward = [&]() {
            if (++loaded < whole) {
                ta.next();
                tb.next();
            }
        };
        auto load_all = [&]() {
#pragma unroll
            for (uint32_t i = 0; i < TA::LOADS; ++i) ta.load(i);
#pragma unroll
            for (uint32_t i = 0; i < TB::LOADS; ++i) tb.load(i);
            onward();
        };
        auto write_tail = [&](uint32_t step, uint32_t a_place, uint32_t b_place) {
            if (step == whole && step < steps) {
                ta.tail(lds, a_place, k0 + step * GEMM_BK, K);
                tb.tail(lds, b_place, k0 + step * GEMM_BK, K);
            }
        };
        if constexpr (!DIRECT) load_all();
#pragma unroll
        for (uint32_t st = 0; st < 2; ++st) {
            if constexpr (DIRECT) {
#pragma unroll
                for (uint32_t i = 0; i < TA::LOADS; ++i) ta.fetch(i, my_a + st * TA::BYTES, left(k0 + st * GEMM_BK));
#pragma unroll
                for (uint32_t i = 0; i < TB::LOADS; ++i) tb.fetch(i, my_b + st * TB::BYTES, left(k0 + st * GEMM_BK));
                ta.next();
                tb.next();
            } else {
#pragma unroll
                for (uint32_t i = 0; i < TA::LOADS; ++i) ta.write(i, lds, my_a + st * TA::BYTES);
#pragma unroll
                for (uint32_t i = 0; i < TB::LOADS; ++i) tb.write(i, lds, my_b + st * TB::BYTES);
                load_all();
                write_tail(st, my_a + st * TA::BYTES, my_b + st * TB::BYTES);
            }
        }
        if constexpr (DIRECT) asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" :: "n"(TA::LOADS + TB::LOADS) : "memory");
        else __syncthreads();
#pragma unroll
        for (uint32_t i = 0; i < FM; ++i) read_a(0, 0, i);
#pragma unroll
        for (uint32_t j = 0; j < 2 * FN; ++j) read_b(0, j / FN, j % FN);
        uint32_t a_now = 0, a_next = TA::BYTES, a_after = 2 * TA::BYTES, b_now = 0;
        for (uint32_t kb = k0; kb < K; kb += GEMM_BK) {
            const uint32_t more = left(kb + 2 * GEMM_BK);
            quarter(c0, a_now, b_now, c2, c2, c0, c0, 0, 0, 0);
            asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");          // every wave has its part of B in registers
            __builtin_amdgcn_sched_barrier(0);
            quarter(c1, a_now, 0, c0, c0, copies_a, c0, my_a + a_after, 0, more);
            quarter(c2, a_now, 0, c0, c0, c0, copies_b, 0, my_b + b_now, more);
            // the next step's tiles have arrived, and every wave has read all of this one's
            if constexpr (DIRECT) {
                ta.next();
                tb.next();
                asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" :: "n"(TA::LOADS + TB::LOADS) : "memory");
            } else {
                onward();
                write_tail((kb - k0) / GEMM_BK + 2, my_a + a_after, my_b + b_now);
                asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
            }
            __builtin_amdgcn_sched_barrier(0);
            b_now ^= TB::BYTES;
            quarter(c3, a_next, b_now, c0, c2, c0, c0, 0, 0, 0);
            const uint32_t t = a_now;
            a_now = a_next;
            a_next = a_after;
            a_after = t;
        }
        if constexpr (DIRECT) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");          // no copy may land in what follows
    }
    char* out = static_cast<char*>(a.c.p[q]);
    const T* res = EPI == 0 ? static_cast<const T*>(a.residual.p[q]) : nullptr;
    T* z = EPI == 0 ? static_cast<T*>(a.z.p[q]) : nullptr;
    float bias[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (EPI == 0 && a.bias.p[q] && n0 + threadIdx.x % (BN / 8) * 8 < N)
        load_params<8>(static_cast<const float*>(a.bias.p[q]), n0 + threadIdx.x % (BN / 8) * 8, N, bias);
#pragma unroll
    for (uint32_t part = 0; part < WM; ++part) {
        __syncthreads();
        if (wm == part) {
#pragma unroll
            for (uint32_t i = 0; i < FM; ++i)
#pragma unroll
                for (uint32_t j = 0; j < FN; ++j)
#pragma unroll
                    for (uint32_t e = 0; e < 4; ++e) {
                        char* p = lds + (i * 32 + (lane & 31u)) * ROW + (wn * NT + j * 32 + e * 8 + (lane >> 5) * 4) * 4;
                        *reinterpret_cast<f32x4*>(p) = f32x4{acc[i][j][4 * e], acc[i][j][4 * e + 1], acc[i][j][4 * e + 2], acc[i][j][4 * e + 3]};
                    }
        }
        __syncthreads();
        constexpr uint32_t ROWS = 4, LANES = BN / 8, DM = WAVES * 64 / LANES;
        const uint32_t n = n0 + threadIdx.x % LANES * 8;
        if (n >= N) continue;
#pragma unroll 1
        for (uint32_t r = threadIdx.x / LANES; r < MT; r += ROWS * DM) {
            float v[ROWS][8];
#pragma unroll
            for (uint32_t i = 0; i < ROWS; ++i) {
                const char* p = lds + (r + i * DM) * ROW + threadIdx.x % LANES * 32;
                const f32x4 x = *reinterpret_cast<const f32x4*>(p), y = *reinterpret_cast<const f32x4*>(p + 16);
#pragma unroll
                for (int e = 0; e < 4; ++e) { v[i][e] = x[e]; v[i][4 + e] = y[e]; }
            }
            const uint32_t m = m0 + part * MT + r;
            if (a.splits > 1) {
                GemmArgs b = a;
                b.accumulate = 0;
                b.ldc = N;
                epilogue8<T, 2, ROWS>(b, reinterpret_cast<char*>(a.partial + ((size_t)q * a.splits + split) * a.M * N), nullptr, nullptr, bias, m, DM, M, n, N, v);
            } else epilogue8<T, EPI, ROWS>(a, out, res, z, bias, m, DM, M, n, N, v);
        }
    }
}

}  // namespace slimdp
