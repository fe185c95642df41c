// Draws from scores: a unit's action out of eight, an env's next level out of a bank; the log-probability and entropy
// of actions and their gradient.
#pragma once
#include "tabx_rows.h"

#pragma clang fp contract(off)

namespace tabx {

constexpr int kChoices = TABX_NUM_ACTIONS;

struct ChoiceArgs {
    const void    *logits;
    const uint8_t *action_mask, *controlled, *actions;
    TabxSampling   how;
    const float   *uniform;
    uint8_t       *actions_out;
    float         *log_prob, *entropy;
    const float   *grad_log_prob, *grad_entropy;
    void          *grad_logits;
    int64_t        rows, stride, grad_stride;
    int32_t        type, grad_type;
    float          inv_temperature, log2e_by_temperature;
    double         inv_temperature64;
};

// A row's eight scores; what is not allowed, and NaN, is -infinity.
__device__ __forceinline__ void load_choices(float (&l)[kChoices], const ChoiceArgs &a, int64_t r)
{
    f32x4 lo, hi;
    const int64_t at = r * a.stride;
    if (a.type == TABX_F32) {
        lo = load_four<TABX_F32>((const float *)a.logits + at);
        hi = load_four<TABX_F32>((const float *)a.logits + at + 4);
    } else if (a.type == TABX_BF16) {
        lo = load_four<TABX_BF16>((const __bf16 *)a.logits + at);
        hi = load_four<TABX_BF16>((const __bf16 *)a.logits + at + 4);
    } else {
        lo = load_four<TABX_F16>((const _Float16 *)a.logits + at);
        hi = load_four<TABX_F16>((const _Float16 *)a.logits + at + 4);
    }
    const float v[kChoices] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
#pragma unroll
    for (int i = 0; i < kChoices; ++i) l[i] = v[i] == v[i] ? v[i] : -INFINITY;
    if (a.action_mask && a.action_mask[r] == 0) l[TABX_ACT_ATTACK] = -INFINITY;
}

__device__ __forceinline__ float largest(const float (&l)[kChoices])
{
    float top = l[0];
#pragma unroll
    for (int i = 1; i < kChoices; ++i) top = fmaxf(top, l[i]);
    return top;
}

// (l - top) times a factor, where an infinite top is as far from itself as a finite one: not at all.
template <typename F>
__device__ __forceinline__ F below_top(float l, float top, F factor)
{
    return l == top ? (F)0 : ((F)l - (F)top) * factor;
}

// Weights exp((l - top) / temperature) in 32 bits, as powers of two: the exponent t is off by three roundings, so a weight
// w = 2^t by at most (2.1 |t| + 2) 2^-24 w, which is below 3.2 * 2^-24 whatever t is.
__device__ __forceinline__ void weigh(float (&w)[kChoices], const float (&l)[kChoices], float top, const ChoiceArgs &a)
{
#pragma unroll
    for (int i = 0; i < kChoices; ++i) w[i] = __builtin_amdgcn_exp2f(below_top(l[i], top, a.log2e_by_temperature));
}

// The sum of the weights but one that is 1: so small a sum as the others may have keeps its bits.
__device__ __forceinline__ float sum_of_others(const float (&w)[kChoices], const float (&l)[kChoices], float top)
{
    float others = 0.0f;
    bool first = true;
#pragma unroll
    for (int i = 0; i < kChoices; ++i) {
        const bool one = first && l[i] == top;
        others += one ? 0.0f : w[i];
        first = first && !one;
    }
    return others;
}

// The choice that `uniform` points to among the kept ones.  Every decision compares sums of weights; `close` says that
// two of them were within `margin`, so that the decision is not certain.  All selects, no branches: the lanes' rows differ.
template <typename F>
__device__ __forceinline__ int pick(const float (&l)[kChoices], const F (&w)[kChoices], float top, const TabxSampling &how,
                                    float uniform, F margin, bool &close)
{
    F kept[kChoices];
#pragma unroll
    for (int i = 0; i < kChoices; ++i) kept[i] = w[i];
    const bool some = how.top_k > 0 && how.top_k < kChoices;
    if (some) {
        int rank[kChoices];                        // how many come before it
#pragma unroll
        for (int i = 0; i < kChoices; ++i) rank[i] = i;
#pragma unroll
        for (int i = 0; i < kChoices; ++i)
#pragma unroll
            for (int j = i + 1; j < kChoices; ++j) {
                const int later = l[j] > l[i] ? 1 : 0;
                rank[i] += later;
                rank[j] -= later;
            }
#pragma unroll
        for (int i = 0; i < kChoices; ++i) kept[i] = rank[i] < how.top_k ? kept[i] : (F)0;
    }
    if (how.top_p < 1.0f) {
        F among = (F)0, ahead[kChoices];
#pragma unroll
        for (int i = 0; i < kChoices; ++i) {
            among += kept[i];
            ahead[i] = (F)0;
        }
#pragma unroll
        for (int i = 0; i < kChoices; ++i)
#pragma unroll
            for (int j = i + 1; j < kChoices; ++j) {
                const bool later = l[j] > l[i];
                ahead[i] += later ? kept[j] : (F)0;
                ahead[j] += later ? (F)0 : kept[i];
            }
        const F most = (F)how.top_p * among;
#pragma unroll
        for (int i = 0; i < kChoices; ++i) {
            close = close || (kept[i] > (F)0 && fabs(ahead[i] - most) <= margin);
            kept[i] = ahead[i] < most ? kept[i] : (F)0;
        }
    }
    if (how.min_p > 0.0f) {
#pragma unroll
        for (int i = 0; i < kChoices; ++i) {
            close = close || (l[i] != top && fabs(w[i] - (F)how.min_p) <= margin);
            kept[i] = w[i] >= (F)how.min_p ? kept[i] : (F)0;
        }
    }
    F total = (F)0;
#pragma unroll
    for (int i = 0; i < kChoices; ++i) total += kept[i];
    const float u = uniform > 0.0f ? fminf(uniform, 0x1.fffffep-1f) : 0.0f;
    const F at = (F)u * total;
    // the first whose running sum exceeds `at`: as many as do not come before it
    F upto = (F)0;
    int choice = 0;
#pragma unroll
    for (int i = 0; i < kChoices; ++i) {
        upto += kept[i];
        close = close || fabs(upto - at) <= margin;
        choice += upto > at ? 0 : 1;
    }
    return choice;
}

// One lane per row.  What a row is made of is 64 bytes at most, so the launch is bound by HBM or, below a few ten thousand
// rows, by its own latency.  The draw is decided in 32 bits where no comparison is closer than the weights are exact, and
// in 64 bits else (once in ten thousand rows).  A sum of eight weights is off by 26 * 2^-24 from the weights and by 28 * 2^-24
// from its own additions (seven, each of half a step below 8), its product with `uniform` by another 4 * 2^-24: 112 * 2^-24
// on both sides of a comparison, under the margin of 2^-17.
__global__ __launch_bounds__(256) void tabx_sample_actions_kernel(const ChoiceArgs a)
{
    for (int64_t r = (int64_t)blockIdx.x * 256 + threadIdx.x; r < a.rows; r += (int64_t)gridDim.x * 256) {
        if (a.controlled && a.controlled[r] == 0) continue;
        const float uniform = a.uniform[r];
        float l[kChoices];
        load_choices(l, a, r);
        const float top = largest(l);
        int choice = TABX_ACT_NOOP;
        float log_prob = 0.0f;
        if (a.how.temperature == 0.0f) {
#pragma unroll
            for (int i = kChoices - 1; i >= 0; --i) choice = l[i] == top ? i : choice;
            choice = top > -INFINITY ? choice : TABX_ACT_NOOP;
        } else if (top > -INFINITY) {
            float w[kChoices];
            weigh(w, l, top, a);
            bool close = false;
            choice = pick<float>(l, w, top, a.how, uniform, 0x1p-17f, close);
            if (close) {
                double w64[kChoices];
#pragma unroll
                for (int i = 0; i < kChoices; ++i) w64[i] = exp(below_top(l[i], top, a.inv_temperature64));
                choice = pick<double>(l, w64, top, a.how, uniform, -1.0, close);
            }
            float taken = 0.0f;
#pragma unroll
            for (int i = 0; i < kChoices; ++i) taken = choice == i ? l[i] : taken;
            log_prob = below_top(taken, top, a.inv_temperature) - log1pf(sum_of_others(w, l, top));
        }
        a.actions_out[r] = (uint8_t)choice;
        if (a.log_prob) a.log_prob[r] = log_prob;
    }
}

// p_i and log p_i of a row, the entropy, and log p_a; nothing allowed: false.
struct Shares {
    float p[kChoices], log_p[kChoices], entropy, taken, rest;   // rest: sum of p over the actions not taken
};

__device__ __forceinline__ bool shares(Shares &s, const ChoiceArgs &a, int64_t r)
{
    float l[kChoices];
    load_choices(l, a, r);
    const float top = largest(l);
    if (!(top > -INFINITY)) return false;
    weigh(s.p, l, top, a);
    const float others = sum_of_others(s.p, l, top);
    const float log_sum = log1pf(others), inv = 1.0f / (1.0f + others);
    const int act = a.actions[r] < kChoices ? a.actions[r] : TABX_ACT_NOOP;
    s.entropy = 0.0f;
    s.taken = 0.0f;
    s.rest = 0.0f;
#pragma unroll
    for (int i = 0; i < kChoices; ++i) {
        s.log_p[i] = below_top(l[i], top, a.inv_temperature) - log_sum;
        s.p[i] *= inv;
        s.entropy -= s.p[i] > 0.0f ? s.p[i] * s.log_p[i] : 0.0f;
        s.taken = act == i ? s.log_p[i] : s.taken;
        s.rest += act == i ? 0.0f : s.p[i];
    }
    return true;
}

__global__ __launch_bounds__(256) void tabx_log_prob_kernel(const ChoiceArgs a)
{
    for (int64_t r = (int64_t)blockIdx.x * 256 + threadIdx.x; r < a.rows; r += (int64_t)gridDim.x * 256) {
        if (a.controlled && a.controlled[r] == 0) continue;
        Shares s;
        const bool some = shares(s, a, r);
        a.log_prob[r] = some ? s.taken : 0.0f;
        if (a.entropy) a.entropy[r] = some ? s.entropy : 0.0f;
    }
}

template <int TYPE>
__device__ __forceinline__ void store_choices(void *data, int64_t at, f32x4 lo, f32x4 hi)
{
    typename Element<TYPE>::one *to = (typename Element<TYPE>::one *)data + at;
    store_four<TYPE>(to, lo);
    store_four<TYPE>(to + 4, hi);
}

__global__ __launch_bounds__(256) void tabx_log_prob_grad_kernel(const ChoiceArgs a)
{
    for (int64_t r = (int64_t)blockIdx.x * 256 + threadIdx.x; r < a.rows; r += (int64_t)gridDim.x * 256) {
        float g[kChoices];
#pragma unroll
        for (int i = 0; i < kChoices; ++i) g[i] = 0.0f;
        Shares s;
        if ((!a.controlled || a.controlled[r] != 0) && shares(s, a, r)) {
            const float gl = a.grad_log_prob && s.taken > -INFINITY ? a.grad_log_prob[r] : 0.0f;
            const float ge = a.grad_entropy ? a.grad_entropy[r] : 0.0f;
            const int act = a.actions[r] < kChoices ? a.actions[r] : TABX_ACT_NOOP;
#pragma unroll
            for (int i = 0; i < kChoices; ++i) {
                const float toward = act == i ? s.rest : -s.p[i];
                const float even = s.p[i] > 0.0f ? s.p[i] * (s.log_p[i] + s.entropy) : 0.0f;
                g[i] = (gl * toward - ge * even) * a.inv_temperature;
            }
        }
        const f32x4 lo = {g[0], g[1], g[2], g[3]}, hi = {g[4], g[5], g[6], g[7]};
        const int64_t at = r * a.grad_stride;
        if (a.grad_type == TABX_F32) store_choices<TABX_F32>(a.grad_logits, at, lo, hi);
        else if (a.grad_type == TABX_BF16) store_choices<TABX_BF16>(a.grad_logits, at, lo, hi);
        else store_choices<TABX_F16>(a.grad_logits, at, lo, hi);
    }
}

} // namespace tabx
