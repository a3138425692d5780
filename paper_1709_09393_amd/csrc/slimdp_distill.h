// Distillation from a teacher's top logits: loss of every row and gradient of the student's logits.  Included only by slimdp_train.hip.
#pragma once
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
// One block of 256 threads a row; the logits are read twice, the second time from the caches.
// An entry that appears twice counts twice; the first of equal indices carries the sum of all, so that one thread
// writes each place and the sum's order is that of the list.
template <class T>
__global__ __launch_bounds__(256) void k_distill(DistillArgs a)
{
    constexpr int V = Vec<T>::N, BT = 256;
    __shared__ float tp[TEACHER_MAX];
    __shared__ uint32_t ti[TEACHER_MAX];
    __shared__ float slots[6][BT / 64];
    const uint32_t q = blockIdx.y, rows = a.rows.n[q], vocab = a.vocab, top = a.top, t = threadIdx.x;
    const T* logits = static_cast<const T*>(a.logits.p[q]);
    const uint32_t* index = static_cast<const uint32_t*>(a.index.p[q]);
    const float* value = static_cast<const float*>(a.value.p[q]);
    const float* row_weight = static_cast<const float*>(a.row_weight.p[q]);
    T* dlogits = static_cast<T*>(a.dlogits.p[q]);
    const float inv_tau = 1.0f / a.tau;
    auto block_max = [&](float v, float* s) {
        v = wave_max_f(v);
        if ((t & 63u) == 0) s[t >> 6] = v;
        __syncthreads();
        return fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3]));
    };
    for (uint32_t r = blockIdx.x; r < rows; r += gridDim.x) {
        const T* row = logits + (size_t)r * a.ldl;
        const float w = row_weight ? row_weight[r] : 1.0f;
        // the teacher's distribution
        float vmax = -__builtin_inff();
        for (uint32_t j = t; j < top; j += BT) {
            uint32_t i = index[(size_t)r * a.ldt + j];
            float v = -__builtin_inff();
            if (i < vocab) v = value[(size_t)r * a.ldt + j] * inv_tau;
            else {
                if (i != 0xFFFFFFFFu) atomicOr(a.status, 4u);
                i = 0xFFFFFFFFu;
            }
            ti[j] = i;
            tp[j] = v;
            vmax = fmaxf(vmax, v);
        }
        vmax = block_max(vmax, slots[0]);
        const bool some = vmax != -__builtin_inff();
        float mass = 0.0f;
        if (some)
            for (uint32_t j = t; j < top; j += BT)
                if (ti[j] != 0xFFFFFFFFu) mass += expf(tp[j] - vmax);
        mass = group_sum<BT>(mass, slots[1]);
        // the student's largest logit and sum of exponentials
        float top_s = -__builtin_inff();
        for (uint32_t c = t * V; c < vocab; c += BT * V) {
            float f[V];
            unpack<T>(load_clip(row, c, vocab), f);
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (c + i < vocab) top_s = fmaxf(top_s, f[i]);
        }
        top_s = block_max(top_s, slots[2]) * inv_tau;
        if (top_s == -__builtin_inff()) top_s = 0.0f;
        float sum = 0.0f;
        for (uint32_t c = t * V; c < vocab; c += BT * V) {
            float f[V];
            unpack<T>(load_clip(row, c, vocab), f);
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (c + i < vocab) sum += expf(f[i] * inv_tau - top_s);
        }
        sum = group_sum<BT>(sum, slots[3]);
        const float lse = top_s + logf(sum), log_mass = logf(mass);
        float loss = 0.0f;
        if (some && w != 0.0f)
            for (uint32_t j = t; j < top; j += BT) {
                if (ti[j] == 0xFFFFFFFFu) continue;
                const float l = tp[j] - vmax - log_mass, p = expf(l);
                if (p != 0.0f) loss += p * (l - ((float)row[ti[j]] * inv_tau - lse));
            }
        loss = group_sum<BT>(loss, slots[4]);
        if (t == 0) {
            if (a.loss.p[q]) static_cast<float*>(a.loss.p[q])[r] = some && w != 0.0f ? w * a.tau * a.tau * loss : 0.0f;
            if (a.lse.p[q]) static_cast<float*>(a.lse.p[q])[r] = lse;
        }
        if (dlogits) {
            T* out = dlogits + (size_t)r * a.lddl;
            const float scale = w * a.tau;
            const bool live = some && w != 0.0f;
            // each entry's final value, taken before the row may be overwritten (dlogits may be logits)
            float mine[(TEACHER_MAX + BT - 1) / BT];
#pragma unroll
            for (int k = 0; k < (TEACHER_MAX + BT - 1) / BT; ++k) {
                const uint32_t j = k * BT + t;
                mine[k] = 0.0f;
                if (!live || j >= top || ti[j] == 0xFFFFFFFFu) continue;
                float p = 0.0f;
                for (uint32_t o = 0; o < top; ++o)
                    if (ti[o] == ti[j]) p += expf(tp[o] - vmax - log_mass);
                mine[k] = scale * (expf((float)row[ti[j]] * inv_tau - lse) - p);
            }
            __syncthreads();
            for (uint32_t c = t * V; c < vocab; c += BT * V) {
                float f[V];
                unpack<T>(load_clip(row, c, vocab), f);
#pragma unroll
                for (int i = 0; i < V; ++i) f[i] = live ? scale * expf(f[i] * inv_tau - lse) : 0.0f;
                store_clip(out, c, vocab, pack<T>(f));
            }
            __syncthreads();
            if (live)
#pragma unroll
                for (int k = 0; k < (TEACHER_MAX + BT - 1) / BT; ++k) {
                    const uint32_t j = k * BT + t;
                    if (j < top && ti[j] != 0xFFFFFFFFu) out[ti[j]] = (T)mine[k];      // equal indices: the same value
                }
        }
        __syncthreads();
    }
}

}  // namespace slimdp
