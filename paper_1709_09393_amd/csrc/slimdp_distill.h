// Distillation from a teacher's top logits: loss of every row and gradient of the student's logits.  Included only by slimdp_train.hip.
#pragma once
#include "slimdp_act.h"
#include "slimdp_host.h"
#include "slimdp_train.h"

namespace slimdp {

constexpr int TEACHER_MAX = SLIMDP_MAX_TEACHER;

struct DistillArgs {
    InTab logits, index, value, row_weight;
    OutTab loss, lse, dlogits;
    RowTab rows;
    uint64_t ldl, ldt, lddl;
    uint32_t vocab, top;
    float tau;
    uint32_t* status;
};

// Per row, with s = logits / tau over the vocabulary, q = softmax(s), v = value / tau of the row's valid entries and p = softmax(v):
//     lse = log sum exp(s),   loss = w tau^2 sum_j p_j (log p_j - (s[index_j] - lse)),   dlogits = w tau (q - sum over j at v of p_j)
//
// One block of BT threads a row, which takes MINE of the teacher's entries a thread.  HELD > 0: the row stays in registers, HELD vectors of sixteen bytes a thread, so that it is read
// once and written once; the sum's exponentials are taken as the vectors arrive (against each thread's own largest value so far),
// the gradient's as they leave, and neither waits for the other's memory.  HELD = 0: rows that no block holds, read twice, and calls that ask for no
// gradient (nothing is kept then: 128,000 columns of bf16, 4,096 rows: 192 us instead of 294).  NT: streams pass the caches by.
// The largest logit is held finite: one of +inf has an infinite exponential then, no NaN, and lse is infinite.
// Exponentials are powers of two of (x - largest) * (log2 e / tau): the difference first, so that logits far from zero (a mask of the
// type's lowest value over a whole row among them) lose nothing to the product's rounding, and the teacher's likewise: a value whose quotient
// by a temperature below 1 is beyond the type's range is still a value.
//
// The teacher's entries are subtracted by the threads that own their places: every thread has a list of the entries in its vectors.
// An entry that appears twice counts twice: the first of equal indices carries the sum, added in the order of the entries, and
// the others nothing, so that no order of threads shows in the result.
template <class T, int BT, int HELD, int MINE, int NT>
__global__ __launch_bounds__(BT) void k_distill(DistillArgs a)
{
    constexpr int V = Vec<T>::N, WAVES = BT / 64, ROOM = BT * MINE;
    __shared__ float tp[ROOM];                       // p of every entry; then what its place loses
    __shared__ uint32_t ti[ROOM];
    __shared__ uint16_t follow[ROOM];
    __shared__ uint32_t head[BT];
    __shared__ uint32_t held_slots[BT];              // bit: the list has an entry in vector (number mod 32) of the thread
    __shared__ float slots[5][WAVES];
    const uint32_t q = blockIdx.y, rows = a.rows.n[q], vocab = a.vocab, top = a.top, t = threadIdx.x, wave = t >> 6;
    const T* logits = static_cast<const T*>(a.logits.p[q]);
    const uint32_t* index = static_cast<const uint32_t*>(a.index.p[q]);
    const float* value = static_cast<const float*>(a.value.p[q]);
    const float* row_weight = static_cast<const float*>(a.row_weight.p[q]);
    T* dlogits = static_cast<T*>(a.dlogits.p[q]);
    const float inv_tau = 1.0f / a.tau, scale2 = inv_tau * LOG2E;
    const float INF = __builtin_inff(), MOST = __FLT_MAX__;
    // whole vectors, and behind the last of them one element a thread
    const uint32_t main = vocab / V * V, last = main + t;
    const bool has_last = last < vocab;
    auto owner_of = [&](uint32_t i) { return i < main ? i / V % BT : i - main; };
    auto put = [&](float v, float* s) { if ((t & 63u) == 0) s[wave] = v; };
    auto sum_of = [&](const float* s) {
        float v = s[0];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) v += s[w];
        return v;
    };
    auto max_of = [&](const float* s) {
        float v = s[0];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) v = fmaxf(v, s[w]);
        return v;
    };
    for (uint32_t r = blockIdx.x; r < rows; r += gridDim.x) {
        const T* row = logits + (size_t)r * a.ldl;
        raw4 x[HELD ? HELD : 1];
        if constexpr (HELD > 0) {
#pragma unroll
            for (int j = 0; j < HELD; ++j) {
                const uint32_t c = ((uint32_t)j * BT + t) * V;
                if (c < main) x[j] = load_raw<T, NT>(row + c);
            }
        }
        const float x_last = has_last ? (float)row[last] : 0.0f;
        const float w = row_weight ? row_weight[r] : 1.0f;
        // the teacher's distribution, and the student's logits at its entries
        float vmax = -INF, logit[MINE], mine[MINE];
        uint32_t at[MINE];
        head[t] = 0xFFFFu;
        held_slots[t] = 0;
#pragma unroll
        for (int k = 0; k < MINE; ++k) {
            const uint32_t j = k * BT + t;
            at[k] = 0xFFFFFFFFu;
            mine[k] = -INF;
            logit[k] = 0.0f;
            if (j >= top) continue;
            at[k] = index[(size_t)r * a.ldt + j];
            if (at[k] < vocab) {
                mine[k] = value[(size_t)r * a.ldt + j];
                logit[k] = (float)row[at[k]];
            } else {
                if (at[k] != 0xFFFFFFFFu) atomicOr(a.status, STATUS_TEACHER);
                at[k] = 0xFFFFFFFFu;
            }
            vmax = fmaxf(vmax, mine[k] == mine[k] ? mine[k] : INF);              // a NaN must not look like no entry
        }
        put(wave_max_f(vmax), slots[0]);
        __syncthreads();
        vmax = max_of(slots[0]);
        const bool live = vmax != -INF && w != 0.0f;
        float mass = 0.0f;
#pragma unroll
        for (int k = 0; k < MINE; ++k)
            if (live && at[k] != 0xFFFFFFFFu) {
                mine[k] = (mine[k] - vmax) / a.tau;
                mass += expf(mine[k]);
            }
        put(wave_sum_f(mass), slots[1]);
        __syncthreads();
        const float log_mass = logf(sum_of(slots[1]));
#pragma unroll
        for (int k = 0; k < MINE; ++k) {
            const uint32_t j = k * BT + t;
            if (j >= top) continue;
            mine[k] = live ? mine[k] - log_mass : -INF;                        // log p
            ti[j] = at[k];
            tp[j] = at[k] != 0xFFFFFFFFu ? expf(mine[k]) : 0.0f;
            if (live && dlogits && at[k] != 0xFFFFFFFFu) {
                const uint32_t owner = owner_of(at[k]);
                follow[j] = (uint16_t)atomicExch(&head[owner], j);
                if (at[k] < main) atomicOr(&held_slots[owner], 1u << (at[k] / (V * BT) & 31u));
            }
        }
        // the student's largest logit and sum of exponentials
        float m = -INF, sum = 0.0f;
        auto take = [&](raw4 v) {
            float f[V], big = -INF;
            unpack<T>(v, f);
#pragma unroll
            for (int i = 0; i < V; ++i) big = fmaxf(big, f[i]);
            big = fminf(big, MOST);
            if (big > m) {
                sum *= __builtin_amdgcn_exp2f((m - big) * scale2);             // the first time: 0 * 0
                m = big;
            }
            const float ref = m == -INF ? 0.0f : m;
#pragma unroll
            for (int i = 0; i < V; ++i) sum += __builtin_amdgcn_exp2f((f[i] - ref) * scale2);
        };
        if (has_last) {
            m = fminf(fmaxf(x_last, -INF), MOST);
            sum = __builtin_amdgcn_exp2f((x_last - (m == -INF ? 0.0f : m)) * scale2);
        }
        if constexpr (HELD > 0) {
#pragma unroll
            for (int j = 0; j < HELD; ++j)
                if (((uint32_t)j * BT + t) * V < main) take(x[j]);
        } else {
            for (uint32_t c = t * V; c < main; c += BT * V) take(load_raw<T>(row + c));
        }
        const float wave_m = wave_max_f(m);
        sum = m == -INF ? sum : sum * __builtin_amdgcn_exp2f((m - wave_m) * scale2);      // nothing but -inf seen: 0, or NaN
        put(wave_m, slots[2]);
        put(wave_sum_f(sum), slots[3]);
        __syncthreads();
        m = max_of(slots[2]);
        if (m == -INF) m = 0.0f;
        sum = 0.0f;
#pragma unroll
        for (int i = 0; i < WAVES; ++i) {
            const float wm = slots[2][i], ws = slots[3][i];
            sum += wm == -INF ? ws : ws * __builtin_amdgcn_exp2f((wm - m) * scale2);
        }
        const float log_sum = logf(sum), lse = m * inv_tau + log_sum;
        float loss = 0.0f;
#pragma unroll
        for (int k = 0; k < MINE; ++k) {
            const uint32_t j = k * BT + t;
            if (!live || j >= top || at[k] == 0xFFFFFFFFu) continue;
            const float p = tp[j];
            if (p != 0.0f) loss += p * (mine[k] - ((logit[k] - m) * inv_tau - log_sum));
        }
        put(wave_sum_f(loss), slots[4]);
        // equal indices: whoever finds another one in the list of their place
        float lost[MINE];
#pragma unroll
        for (int k = 0; k < MINE; ++k) {
            const uint32_t j = k * BT + t;
            lost[k] = 0.0f;
            if (!live || !dlogits || j >= top || at[k] == 0xFFFFFFFFu) continue;
            uint32_t same = 0, before = 0;
            for (uint32_t e = head[owner_of(at[k])]; e != 0xFFFFu; e = follow[e])
                if (ti[e] == at[k]) {
                    ++same;
                    before += e < j;
                }
            lost[k] = before ? 0.0f : tp[j];
            if (before || same == 1) continue;
            if (same <= 8) {                         // the next larger one of the list, again and again
                uint32_t last = j;
                for (uint32_t i = 1; i < same; ++i) {
                    uint32_t least = 0xFFFFu;
                    for (uint32_t e = head[owner_of(at[k])]; e != 0xFFFFu; e = follow[e])
                        if (ti[e] == at[k] && e > last && e < least) least = e;
                    lost[k] += tp[least];
                    last = least;
                }
            } else
                for (uint32_t e = j + 1; e < top; ++e)
                    if (ti[e] == at[k]) lost[k] += tp[e];
        }
        __syncthreads();
        if (t == 0) {
            if (a.loss.p[q]) static_cast<float*>(a.loss.p[q])[r] = live ? w * a.tau * a.tau * sum_of(slots[4]) : 0.0f;
            if (a.lse.p[q]) static_cast<float*>(a.lse.p[q])[r] = lse;
        }
        if (!dlogits) continue;
#pragma unroll
        for (int k = 0; k < MINE; ++k)
            if (live && k * BT + t < top) tp[k * BT + t] = w * a.tau * lost[k];
        __syncthreads();
        T* out = dlogits + (size_t)r * a.lddl;
        const float scale = w * a.tau / sum;
        const uint32_t touched = held_slots[t], list = head[t];
        auto give = [&](raw4 v, uint32_t c, uint32_t j) {
            float f[V];
            unpack<T>(v, f);
#pragma unroll
            for (int i = 0; i < V; ++i) f[i] = scale * __builtin_amdgcn_exp2f((f[i] - m) * scale2);
            if (touched >> (j & 31u) & 1u)
                for (uint32_t e = list; e != 0xFFFFu; e = follow[e]) {
                    const uint32_t o = ti[e] - c;
                    const float p = tp[e];
#pragma unroll
                    for (int i = 0; i < V; ++i)
                        if (o == (uint32_t)i) f[i] -= p;
                }
            store_raw<T, NT>(out + c, live ? pack<T>(f) : raw4{0, 0, 0, 0});
        };
        if constexpr (HELD > 0) {
#pragma unroll
            for (int j = 0; j < HELD; ++j) {
                const uint32_t c = ((uint32_t)j * BT + t) * V;
                if (c < main) give(x[j], c, j);
            }
        } else {
            uint32_t j = 0;
            for (uint32_t c = t * V; c < main; c += BT * V, ++j) give(load_raw<T>(row + c), c, j);
        }
        if (has_last) {
            float f = scale * __builtin_amdgcn_exp2f((x_last - m) * scale2);
            for (uint32_t e = list; e != 0xFFFFu; e = follow[e])
                if (ti[e] == last) f -= tp[e];
            out[last] = live ? (T)f : (T)0.0f;
        }
        __syncthreads();                             // lists and sums are written anew for the next row
    }
}

}  // namespace slimdp
