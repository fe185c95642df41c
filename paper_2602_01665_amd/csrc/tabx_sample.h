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
    int32_t        stream;         // the gradient goes past the caches
    float          inv_temperature, log2e_by_temperature;
    double         inv_temperature64;
};

// A row's eight scores, in 32 bits; what is not allowed, and NaN, is -infinity.
struct Scores {
    float l[kChoices], top;
};

__device__ __forceinline__ Scores load_scores(const ChoiceArgs &a, int64_t r)
{
    f32x4 lo, hi;
    const int64_t at = r * a.stride;
    const bool attack = !a.action_mask || a.action_mask[r] != 0;
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
    Scores s = {{lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w}, -INFINITY};
    static_assert(TABX_ACT_ATTACK == 5 && kChoices == 8, "");
    s.l[TABX_ACT_ATTACK] = attack ? s.l[TABX_ACT_ATTACK] : -INFINITY;
#pragma unroll
    for (int i = 0; i < kChoices; ++i) {
        s.l[i] = fmaxf(s.l[i], -INFINITY);         // of a number and NaN, the number
        s.top = fmaxf(s.top, s.l[i]);
    }
    if (s.top == INFINITY) {                       // the infinite ones share the draw: as if they were 0 and the others nothing
#pragma unroll
        for (int i = 0; i < kChoices; ++i) s.l[i] = s.l[i] == INFINITY ? 0.0f : -INFINITY;
        s.top = 0.0f;
    }
    return s;
}

// Weights exp((l - top) / temperature) in 32 bits, as powers of two: the exponent t is off by three roundings, so a weight
// w = 2^t by at most (2.1 |t| + 2) 2^-24 w, which is below 3.2 * 2^-24 whatever t is.
struct Weights8 {
    float t[kChoices], w[kChoices];
    // The sum of the weights but one that is 1: so small a sum as the others may have keeps its bits.
    float others;
};

__device__ __forceinline__ Weights8 weigh(const Scores &s, const ChoiceArgs &a)
{
    Weights8 r;
    r.others = 0.0f;
    bool first = true;
#pragma unroll
    for (int i = 0; i < kChoices; ++i) {
        r.t[i] = (s.l[i] - s.top) * a.log2e_by_temperature;
        r.w[i] = __builtin_amdgcn_exp2f(r.t[i]);
        const bool one = first && s.l[i] == s.top;
        r.others += one ? 0.0f : r.w[i];
        first = first && !one;
    }
    return r;
}

// (Bits are put together: a choice between the scores would become one between their addresses, and the scores would
// move to LDS, which cost these launches 11 us.)
__device__ __forceinline__ float score_of_choice(const Scores &s, int choice)
{
    uint32_t bits = 0;
#pragma unroll
    for (int i = 0; i < kChoices; ++i) bits |= choice == i ? __float_as_uint(s.l[i]) : 0u;
    return __uint_as_float(bits);
}

constexpr float kLn2 = 0.693147180559945f;

// log(1 + x) for x >= 0: the logarithm of the rounded sum, and what the rounding took, over the sum.
__device__ __forceinline__ float log_of_sum(float others)
{
    const float sum = 1.0f + others;
    return fmaf(others - (sum - 1.0f), __builtin_amdgcn_rcpf(sum), kLn2 * __builtin_amdgcn_logf(sum));
}

__host__ __device__ __forceinline__ float usable_uniform(float u) { return u > 0.0f ? fminf(u, 0x1.fffffep-1f) : 0.0f; }

constexpr float kMargin = 0x1p-16f;

// The same settings as the kernel takes them.  The largest weight is 1 and all together are at most kChoices: up to a top_p of
// one by that many the second is never kept, and no comparison needs to find out.
inline TabxSampling settings_of(TabxSampling how)
{
    if (how.top_p <= 1.0f / kChoices) how.top_k = 1, how.top_p = 1.0f;
    return how;
}

// The choice that `uniform` points to among the kept ones.  Every decision compares weights or sums of them; `spare` becomes
// the least that a difference which decided one had beyond its margin.  Two weights or sums that a filter compares are as
// exact as they are large, and so is their margin; the draw's is that of the sum of all.  All selects, no branches: the
// lanes' rows differ.
template <bool FILTER>
__host__ __device__ __forceinline__ int pick(const Scores &s, const float (&w)[kChoices], const TabxSampling &how, float uniform,
                                             float &spare)
{
    spare = 1.0f;
    float kept[kChoices];
#pragma unroll
    for (int i = 0; i < kChoices; ++i) kept[i] = w[i];
    if (FILTER && how.top_k > 0 && how.top_k < kChoices) {
        int rank[kChoices];                        // how many come before it
#pragma unroll
        for (int i = 0; i < kChoices; ++i) rank[i] = i;
#pragma unroll
        for (int i = 0; i < kChoices; ++i)
#pragma unroll
            for (int j = i + 1; j < kChoices; ++j) {
                const int later = s.l[j] > s.l[i] ? 1 : 0;
                rank[i] += later;
                rank[j] -= later;
            }
#pragma unroll
        for (int i = 0; i < kChoices; ++i) kept[i] = rank[i] < how.top_k ? kept[i] : 0.0f;
    }
    if (FILTER && how.top_p < 1.0f) {
        // What comes before it is less than top_p of all where it and what comes after are more than the rest of all: sums
        // of few small weights, which keep their bits where top_p is close to one.
        float tail[kChoices], among = 0.0f;
#pragma unroll
        for (int i = 0; i < kChoices; ++i) {
            tail[i] = kept[i];
            among += kept[i];
        }
#pragma unroll
        for (int i = 0; i < kChoices; ++i)
#pragma unroll
            for (int j = i + 1; j < kChoices; ++j) {
                const bool later = s.l[j] > s.l[i];
                tail[i] += later ? 0.0f : kept[j];
                tail[j] += later ? kept[i] : 0.0f;
            }
        const float rest = (1.0f - how.top_p) * among;
#pragma unroll
        for (int i = 0; i < kChoices; ++i) {
            const float over = tail[i] - rest;
            spare = fminf(spare, fmaf(-kMargin, tail[i], fabsf(over)));
            kept[i] = over > 0.0f ? kept[i] : 0.0f;
        }
    }
    if (FILTER && how.min_p > 0.0f) {
#pragma unroll
        for (int i = 0; i < kChoices; ++i) {
            const float over = w[i] - how.min_p;
            spare = fminf(spare, s.l[i] != s.top ? fmaf(-kMargin, w[i], fabsf(over)) : spare);
            kept[i] = over >= 0.0f ? kept[i] : 0.0f;
        }
    }
    float total = 0.0f;
#pragma unroll
    for (int i = 0; i < kChoices; ++i) total += kept[i];
    float left = usable_uniform(uniform) * total, nearest = 1.0f;
    // the first whose running sum exceeds that: as many as do not come before it
    int choice = 0;
#pragma unroll
    for (int i = 0; i < kChoices; ++i) {
        left -= kept[i];
        nearest = fminf(nearest, fabsf(left));
        choice += left < 0.0f ? 0 : 1;
    }
    spare = fminf(spare, nearest - kMargin);
    return choice;
}

// v of another lane.
__device__ __forceinline__ float of_lane(float v, int lane)
{
    return __int_as_float(__builtin_amdgcn_ds_bpermute(lane * 4, __float_as_int(v)));
}

// v of lane I of each eight.
template <int I>
__device__ __forceinline__ double of_eight(double v)
{
    const uint64_t b = (uint64_t)__double_as_longlong(v);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_ds_swizzle((int)(uint32_t)b, I << 5 | 0x18);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_ds_swizzle((int)(uint32_t)(b >> 32), I << 5 | 0x18);
    return __longlong_as_double((long long)((uint64_t)hi << 32 | lo));
}

// The same in 64 bits for the row of lane `source`, by the eight lanes it is one of: lane j has choice j mod 8.  (Each lane for
// its own row, the few wavefronts that need it would be the last to finish, a thousand instructions after the others.
// 327680 rows: 9.3 us.)
template <bool FILTER>
__device__ __forceinline__ int pick_exactly(const Scores &s, const TabxSampling &how, float uniform, double inv_temperature,
                                            int source)
{
    const int j = (int)threadIdx.x & 7, eight = (int)threadIdx.x & 56;
    const float top = of_lane(s.top, source);
    float l[kChoices], mine;
#pragma unroll
    for (int i = 0; i < kChoices; ++i) {
        l[i] = of_lane(s.l[i], source);
        mine = i == 0 || j == i ? l[i] : mine;
    }
    const double own = exp(((double)mine - (double)top) * inv_temperature);
    double w[kChoices] = {of_eight<0>(own), of_eight<1>(own), of_eight<2>(own), of_eight<3>(own),
                          of_eight<4>(own), of_eight<5>(own), of_eight<6>(own), of_eight<7>(own)};
    if constexpr (FILTER) {
        uint32_t ahead = 0;                        // which come before it
#pragma unroll
        for (int i = 0; i < kChoices; ++i) ahead |= l[i] > mine || (i < j && l[i] == mine) ? 1u << i : 0u;
        const bool few = how.top_k == 0 || __builtin_popcount(ahead) < how.top_k;
        const uint32_t among = (uint32_t)(__ballot(few) >> eight);
        double before = 0.0, most = 0.0;
#pragma unroll
        for (int i = 0; i < kChoices; ++i) {
            before += ahead >> i & 1 ? w[i] : 0.0;
            most += among >> i & 1 ? w[i] : 0.0;
        }
        const bool enough = how.top_p >= 1.0f || before < (double)how.top_p * most;
        const uint32_t kept = (uint32_t)(__ballot(few && enough && own >= (double)how.min_p) >> eight);
#pragma unroll
        for (int i = 0; i < kChoices; ++i) w[i] = kept >> i & 1 ? w[i] : 0.0;
    }
    double at = 0.0, upto = 0.0;
#pragma unroll
    for (int i = 0; i < kChoices; ++i) at += w[i];
    at *= (double)usable_uniform(of_lane(uniform, source));
    int choice = 0;
#pragma unroll
    for (int i = 0; i < kChoices; ++i) {
        upto += w[i];
        choice += upto > at ? 0 : 1;
    }
    return choice;
}

// One lane per row.  The draw is decided in 32 bits where no comparison is closer than the weights are exact, and in 64
// bits else.  In steps of 2^-24:
//   - a sum of eight weights is off by 26 from the weights and by 28 from its own additions (seven, each of half a step below
//     8), the weights before one by as much again, `uniform` times a sum by another 4: below 200 on both sides of the draw's
//     comparison, under the margin of 256;
//   - a weight that min_p or top_p may leave out wrongly moves these sums by itself: eight below 2^-22 by 32, still under the
//     margin, and one above that is off by 49 of itself, a sum of it and those that come after it by 59 of itself, (1 - top_p)
//     times the sum of all by 57 of itself: under the margin of 256 of itself.
// A draw is so close once in some thousand rows, and so is a filter, but where the scores make ties of them: eight equal ones
// and a top_p of one half send every row to the 64 bits, one of each eight lanes' at a time (655360 rows 37 us; 235 with one
// of the wavefront's).
// FILTER: top_k, top_p or min_p leave something out.  655360 rows of nine f32, 28 MB: 7.7 us; 327680 of bf16, half of them
// controlled, all filters: 6.9 us, with five wavefronts per SIMD (four, in 20 registers more: 7.6).  96 rows: 2.3 us, 6.8 from
// call to call.
template <bool FILTER>
__global__ __launch_bounds__(256, 5) void tabx_sample_actions_kernel(const ChoiceArgs a)
{
    for (int64_t first = (int64_t)blockIdx.x * 256; first < a.rows; first += (int64_t)gridDim.x * 256) {
        const bool there = first + (int)threadIdx.x < a.rows;
        const int64_t r = there ? first + (int)threadIdx.x : a.rows - 1;
        const bool on = there && (!a.controlled || a.controlled[r] != 0);
        const float uniform = a.uniform[r];
        const Scores s = load_scores(a, r);
        int choice = TABX_ACT_NOOP;
        float log_prob = 0.0f;
        if (a.how.temperature == 0.0) {
#pragma unroll
            for (int i = kChoices - 1; i >= 0; --i) choice = s.l[i] == s.top ? i : choice;
            choice = s.top > -INFINITY ? choice : TABX_ACT_NOOP;
        } else {
            const bool some = s.top > -INFINITY;
            const Weights8 w = weigh(s, a);
            float spare;
            choice = pick<FILTER>(s, w.w, a.how, uniform, spare);
            uint64_t close = __ballot(on && some && spare <= 0.0f);
            uint32_t left = (uint32_t)(close >> ((int)threadIdx.x & 56)) & 255;   // of this lane's eight rows
            while (close != 0) {
                const int source = ((int)threadIdx.x & 56) + (left != 0 ? __builtin_ctz(left) : 0);
                const int exact = pick_exactly<FILTER>(s, a.how, uniform, a.inv_temperature64, source);
                choice = left != 0 && ((int)threadIdx.x & 63) == source ? exact : choice;
                left &= left - 1;
                close = __ballot(left != 0);
            }
            choice = some ? choice : TABX_ACT_NOOP;
            log_prob = some ? (score_of_choice(s, choice) - s.top) * a.inv_temperature - log_of_sum(w.others) : 0.0f;
        }
        if (on) {
            a.actions_out[r] = (uint8_t)choice;
            if (a.log_prob) a.log_prob[r] = log_prob;
        }
    }
}

// With Z = sum w = 1 + others and L = log Z: log p_i = ln2 t_i - L and entropy = L - ln2 sum w_i t_i / Z, so nothing is
// done to each choice that the sum has not got already.  Where t is below every exponent of a 32-bit number, w is zero
// and t only has to be finite.  All of it in 32 bits, with the hardware's exponential, logarithm and reciprocal: what comes out
// is off by 4e-8 of itself on average, where 64 bits rounded once would be by 2.5e-8, and one more rounding is all that the
// gradients of a network take from it.
struct Taken {
    float log_prob, t, log_sum, inv_sum, mean_t;   // of the action, and its t; L; 1 / Z; sum p_i t_i
    int   action;
};

__device__ __forceinline__ Taken take_action(const Scores &s, Weights8 &w, int action, const ChoiceArgs &a)
{
    Taken k;
    k.action = action < kChoices ? action : TABX_ACT_NOOP;
    k.log_sum = log_of_sum(w.others);
    k.inv_sum = __builtin_amdgcn_rcpf(1.0f + w.others);
    const float below = score_of_choice(s, k.action) - s.top;
    k.log_prob = below * a.inv_temperature - k.log_sum;
    k.t = below * a.log2e_by_temperature;
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < kChoices; ++i) {
        w.t[i] = fmaxf(w.t[i], -200.0f);
        sum = fmaf(w.w[i], w.t[i], sum);
    }
    k.mean_t = sum * k.inv_sum;
    return k;
}

// Bound by HBM: 2621440 rows of f32 21.5 us, 5.1 TB/s (half of them controlled 19.5: a line holds four rows).
__global__ __launch_bounds__(256) void tabx_log_prob_kernel(const ChoiceArgs a)
{
    for (int64_t r = (int64_t)blockIdx.x * 256 + threadIdx.x; r < a.rows; r += (int64_t)gridDim.x * 256) {
        if (a.controlled && a.controlled[r] == 0) continue;
        const int act = a.actions[r];
        const Scores s = load_scores(a, r);
        Weights8 w = weigh(s, a);
        const Taken k = take_action(s, w, act, a);
        const bool some = s.top > -INFINITY;
        a.log_prob[r] = some ? k.log_prob : 0.0f;
        if (a.entropy) a.entropy[r] = some ? fmaf(-kLn2, k.mean_t, k.log_sum) : 0.0f;
    }
}

template <int TYPE, bool STREAM>
__device__ __forceinline__ void store_choices(void *data, int64_t at, f32x4 lo, f32x4 hi)
{
    typename Element<TYPE>::one *to = (typename Element<TYPE>::one *)data + at;
    store_four<TYPE, STREAM>(to, lo);
    store_four<TYPE, STREAM>(to + 4, hi);
}

template <bool STREAM>
__device__ __forceinline__ void store_gradient(const float (&g)[kChoices], const ChoiceArgs &a, int64_t r)
{
    const f32x4 lo = {g[0], g[1], g[2], g[3]}, hi = {g[4], g[5], g[6], g[7]};
    const int64_t at = r * a.grad_stride;
    if (a.grad_type == TABX_F32) store_choices<TABX_F32, STREAM>(a.grad_logits, at, lo, hi);
    else if (a.grad_type == TABX_BF16) store_choices<TABX_BF16, STREAM>(a.grad_logits, at, lo, hi);
    else store_choices<TABX_F16, STREAM>(a.grad_logits, at, lo, hi);
}

// Bound by HBM.  Rows that are not controlled are written by the same store as the others, in whole lines: written by a
// store of their own, or with only the rows that are controlled dealt to the lanes, it is 5 to 6 us more (2621440 rows of
// f32, half of them controlled, 30 us; all of them 37 us, 5.2 TB/s).
__global__ __launch_bounds__(256) void tabx_log_prob_grad_kernel(const ChoiceArgs a)
{
    for (int64_t r = (int64_t)blockIdx.x * 256 + threadIdx.x; r < a.rows; r += (int64_t)gridDim.x * 256) {
        float g[kChoices];
#pragma unroll
        for (int i = 0; i < kChoices; ++i) g[i] = 0.0f;
        if (!a.controlled || a.controlled[r] != 0) {
            const int act = a.actions[r];
            const float grad_log_prob = a.grad_log_prob ? a.grad_log_prob[r] : 0.0f;
            const float grad_entropy = a.grad_entropy ? a.grad_entropy[r] : 0.0f;
            const Scores s = load_scores(a, r);
            Weights8 w = weigh(s, a);
            const Taken k = take_action(s, w, act, a);
            if (s.top > -INFINITY) {
                // g_i = w_i (towards + apart + along t_i) for the choices not taken
                const float by = k.inv_sum * a.inv_temperature;
                const float gl = k.log_prob > -INFINITY ? grad_log_prob : 0.0f;
                const float apart = grad_entropy * kLn2 * k.mean_t * by, along = -grad_entropy * kLn2 * by;
                const float both = fmaf(-gl, by, apart);
                // 1 - p of the action, from the others where the action has the largest weight
                const float own = __builtin_amdgcn_exp2f(k.t), rest = k.t == 0.0f ? w.others : 1.0f + w.others - own;
                const float mine = fmaf(gl * rest, by, own * fmaf(along, fmaxf(k.t, -200.0f), apart));
#pragma unroll
                for (int i = 0; i < kChoices; ++i) {
                    const float v = k.action == i ? mine : w.w[i] * fmaf(along, w.t[i], both);
                    g[i] = s.l[i] > -INFINITY ? v : 0.0f;   // (zero times a gradient that is not finite would be none)
                }
            }
        }
        if (a.stream) store_gradient<true>(g, a, r);
        else store_gradient<false>(g, a, r);
    }
}

} // namespace tabx
