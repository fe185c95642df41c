// Draws of levels: one table of scores per env, or one for all of them.
//
// A workgroup holds a table in registers, four consecutive levels per thread and tile.  A level's score becomes a
// 32-bit number that is in order like the score, and with its index behind it a 46-bit one that no two levels share;
// what top_k and top_p leave is then "all levels from a threshold up", found eight bits at a time from histograms in
// LDS of how many levels, or how much weight, each value of the eight bits has.  Weights are whole multiples of
// 2^-scale, so that their sums do not depend on the order of the additions.  The running sums of what is kept lie in
// LDS; each env then looks for its level in them by bisection.
#pragma once
#include "tabx_rows.h"

#pragma clang fp contract(off)

namespace tabx {

struct LevelArgs {
    const void    *scores;
    const uint8_t *level_mask, *env_mask;
    TabxSampling   how;
    const float   *uniform;
    int32_t       *next_level;
    int64_t        stride;         // 0: one table for all envs
    int32_t        envs, levels, type;
    int32_t        scale;          // bits after the point of a weight
    double         inv_temperature;
};

constexpr int kIndexBits = 14;
static_assert(TABX_SAMPLE_MAX_LEVELS == 1 << kIndexBits, "a level's index fits behind its score");

// Monotone in the score; 0 for a level that cannot be drawn (-infinity and NaN included).
__device__ __forceinline__ uint32_t score_key(float v)
{
    v += 0.0f;                                     // -0 is +0
    const uint32_t b = __float_as_uint(v);
    return v > -INFINITY ? b ^ ((b >> 31) ? 0xffffffffu : 0x80000000u) : 0u;
}

__device__ __forceinline__ float score_of(uint32_t key)
{
    return __uint_as_float(key ^ ((key >> 31) ? 0x80000000u : 0xffffffffu));
}

__device__ __forceinline__ uint64_t level_weight(uint32_t key, float top, const LevelArgs &a)
{
    if (key == 0) return 0;
    const float l = score_of(key);
    const double d = l == top ? 0.0 : ((double)l - (double)top) * a.inv_temperature;
    return (uint64_t)(ldexp(exp(d), a.scale) + 0.5);
}

// Sum over the workgroup, in all threads.
template <typename T, int THREADS>
__device__ __forceinline__ T group_sum(T v, T *slots)
{
#pragma unroll
    for (int d = 1; d < 64; d *= 2) v += __shfl_xor(v, d);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) slots[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) v += slots[w];
    return v;
}

template <int THREADS>
__device__ __forceinline__ uint32_t group_max(uint32_t v, uint64_t *slots)
{
#pragma unroll
    for (int d = 1; d < 64; d *= 2) v = max(v, (uint32_t)__shfl_xor((int)v, d));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) slots[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) v = max(v, (uint32_t)slots[w]);
    return v;
}

// Running sum over the workgroup's threads: what the threads before this one have, and the whole sum.
template <int THREADS>
__device__ __forceinline__ uint64_t group_scan(uint64_t v, uint64_t *slots, uint64_t &total)
{
    const int lane = (int)threadIdx.x & 63;
    uint64_t upto = v;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const uint64_t before = __shfl_up(upto, d);
        if (lane >= d) upto += before;
    }
    __syncthreads();
    if (lane == 63) slots[threadIdx.x >> 6] = upto;
    __syncthreads();
    uint64_t ahead = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) {
        if (w < (int)(threadIdx.x >> 6)) ahead += slots[w];
        total += slots[w];
    }
    return ahead + upto - v;
}

struct LevelShared {
    uint64_t slots[16];
    uint64_t mass[256];
    uint32_t count[256];
    uint32_t digit;                // the eight bits the threshold has
    uint64_t above;                // count or weight of the levels beyond them
    uint64_t within;               // ... and of those that share them
};

// The weights of a thread's levels: in registers, or from the scores again where there are too many of them.
template <int ITEMS>
struct Weights {
    static constexpr bool kStored = ITEMS <= 8;
    uint64_t w[kStored ? ITEMS : 1];
    float    top;
    __device__ __forceinline__ void take(const uint32_t (&key)[ITEMS], const LevelArgs &a)
    {
        if (kStored) {
#pragma unroll
            for (int i = 0; i < ITEMS; ++i) w[kStored ? i : 0] = level_weight(key[i], top, a);
        }
    }
    __device__ __forceinline__ uint64_t of(int i, uint32_t key, const LevelArgs &a) const
    {
        if (kStored) return w[kStored ? i : 0];
        __builtin_amdgcn_sched_barrier(0);         // one after the other: side by side they would not fit the registers
        return level_weight(key, top, a);
    }
};

// The composite of the level that is the last to be kept.  want: how many levels (MASS false), or the weight that
// the levels before a kept one stay under (MASS true; > 0).  Only composites >= floor compete.
template <int THREADS, int ITEMS, bool MASS>
__device__ __forceinline__ uint64_t threshold(uint32_t (&key)[ITEMS], const Weights<ITEMS> &weight, uint64_t floor,
                                              uint64_t want, const LevelArgs &a, LevelShared &sh)
{
    uint64_t prefix = 0;
    // 48 bits from the top, the two highest of them always zero
#pragma unroll 1
    for (int shift = 40; shift >= 0; shift -= 8) {
        for (int b = (int)threadIdx.x; b < 256; b += THREADS) sh.count[b] = 0, sh.mass[b] = 0;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int j = ((i / 4) * THREADS + (int)threadIdx.x) * 4 + i % 4;
            if (ITEMS > 8) asm volatile("" : "+v"(key[i]));   // (the numbers of all levels at once would not fit either)
            const uint64_t c = (uint64_t)key[i] << kIndexBits | (uint32_t)((1 << kIndexBits) - 1 - j);
            if (key[i] != 0 && c >= floor && (c >> (shift + 8)) == (prefix >> (shift + 8))) {
                const int b = (int)(c >> shift) & 255;
                atomicAdd(&sh.count[b], 1u);
                if (MASS) atomicAdd((unsigned long long *)&sh.mass[b], (unsigned long long)weight.of(i, key[i], a));
            }
        }
        __syncthreads();
        if (threadIdx.x < 64) {
            // lane n has the bins 255 - 4 n ... 252 - 4 n: falling order
            const int first = 255 - 4 * (int)threadIdx.x;
            uint64_t part[4], sum = 0;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                part[q] = MASS ? sh.mass[first - q] : sh.count[first - q];
                sum += part[q];
            }
            uint64_t before = sum;
#pragma unroll
            for (int d = 1; d < 64; d *= 2) {
                const uint64_t other = __shfl_up(before, d);
                if ((int)threadIdx.x >= d) before += other;
            }
            before -= sum;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                if (before < want && before + part[q] >= want) {
                    sh.digit = (uint32_t)(first - q);
                    sh.above = before;
                    sh.within = sh.count[first - q];
                }
                before += part[q];
            }
        }
        __syncthreads();
        prefix |= (uint64_t)sh.digit << shift;
        want -= sh.above;
        // all of them are kept, or the one there is: whatever its other bits are, it lies from here up
        const bool done = MASS ? sh.within == 1 : sh.within == want;
        __syncthreads();
        if (done) break;
    }
    return prefix;
}

// THREADS threads hold ITEMS levels each.  EACH: the running sums of single levels fit into LDS; else those of four.
template <int THREADS, int ITEMS, bool EACH>
__global__ __launch_bounds__(THREADS) void tabx_sample_levels_kernel(const LevelArgs a)
{
    __shared__ LevelShared sh;
    extern __shared__ __attribute__((aligned(16))) uint64_t running[];
    // the envs of this workgroup
    const int group = (int)(blockIdx.y * gridDim.x + blockIdx.x);
    const int env = a.stride != 0 ? group : group * THREADS + (int)threadIdx.x;
    const bool mine = (a.stride == 0 || threadIdx.x == 0) && env < a.envs && (!a.env_mask || a.env_mask[env] != 0);
    if (!__syncthreads_or(mine)) return;
    const int64_t row = a.stride * group;

    uint32_t key[ITEMS], most = 0;
#pragma unroll
    for (int t = 0; t < ITEMS / 4; ++t) {
        const int j = (t * THREADS + (int)threadIdx.x) * 4;
        f32x4 v = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
        if (j + 4 <= a.levels) {
            if (a.type == TABX_F32) v = load_four<TABX_F32>((const float *)a.scores + row + j);
            else if (a.type == TABX_BF16) v = load_four<TABX_BF16>((const __bf16 *)a.scores + row + j);
            else v = load_four<TABX_F16>((const _Float16 *)a.scores + row + j);
        } else {
#pragma unroll
            for (int q = 0; q < 3; ++q)
                if (j + q < a.levels)
                    v[q] = a.type == TABX_F32 ? ((const float *)a.scores)[row + j + q]
                         : a.type == TABX_BF16 ? (float)((const __bf16 *)a.scores)[row + j + q]
                                               : (float)((const _Float16 *)a.scores)[row + j + q];
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            key[4 * t + q] = score_key(v[q]);
            if (a.level_mask && j + q < a.levels && a.level_mask[j + q] == 0) key[4 * t + q] = 0;
            most = max(most, key[4 * t + q]);
        }
    }
    most = group_max<THREADS>(most, sh.slots);
    if (most == 0) return;                         // nothing to draw from: every env keeps what it has
    const float top = score_of(most);

    if (a.how.temperature == 0.0f) {
        uint32_t rank = 0;                         // the lowest index counts most
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int j = ((i / 4) * THREADS + (int)threadIdx.x) * 4 + i % 4;
            if (key[i] == most) rank = max(rank, (uint32_t)((1 << kIndexBits) - j));
        }
        rank = group_max<THREADS>(rank, sh.slots);
        if (mine) a.next_level[env] = (int32_t)((1 << kIndexBits) - rank);
        return;
    }

    Weights<ITEMS> weight;
    weight.top = top;
    weight.take(key, a);

    uint64_t floor = 0;
    if (a.how.top_k > 0 && a.how.top_k < a.levels) {
        uint32_t some = 0;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) some += key[i] != 0;
        some = group_sum<uint32_t, THREADS>(some, (uint32_t *)sh.slots);
        if ((uint32_t)a.how.top_k < some)
            floor = threshold<THREADS, ITEMS, false>(key, weight, 0, (uint64_t)a.how.top_k, a, sh);
    }
    if (a.how.top_p < 1.0f) {
        uint64_t sum = 0;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int j = ((i / 4) * THREADS + (int)threadIdx.x) * 4 + i % 4;
            const uint64_t c = (uint64_t)key[i] << kIndexBits | (uint32_t)((1 << kIndexBits) - 1 - j);
            if (key[i] != 0 && c >= floor) sum += weight.of(i, key[i], a);
        }
        sum = group_sum<uint64_t, THREADS>(sum, sh.slots);
        const uint64_t want = (uint64_t)ceil((double)a.how.top_p * (double)sum);
        const uint64_t least = threshold<THREADS, ITEMS, true>(key, weight, floor, want < sum ? want : sum, a, sh);
        floor = least > floor ? least : floor;
    }
    const uint64_t least = (uint64_t)(ldexp((double)a.how.min_p, a.scale) + 0.5);

    uint64_t before = 0;
#pragma unroll
    for (int t = 0; t < ITEMS / 4; ++t) {
        const int at = t * THREADS + (int)threadIdx.x;
        uint64_t kept[4], sum = 0, total;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const uint64_t c = (uint64_t)key[4 * t + q] << kIndexBits | (uint32_t)((1 << kIndexBits) - 1 - (at * 4 + q));
            kept[q] = key[4 * t + q] != 0 && c >= floor ? weight.of(4 * t + q, key[4 * t + q], a) : 0;
            if (kept[q] < least) kept[q] = 0;
            sum += kept[q];
        }
        uint64_t upto = before + group_scan<THREADS>(sum, sh.slots, total);
        before += total;
        if (EACH) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                upto += kept[q];
                running[at * 4 + q] = upto;
            }
        } else {
            running[at] = upto + sum;
        }
    }
    __syncthreads();
    if (!mine) return;

    // the first running sum beyond uniform * total
    const float u = a.uniform[env] > 0.0f ? fminf(a.uniform[env], 0x1.fffffep-1f) : 0.0f;
    uint64_t at = (uint64_t)((double)u * (double)before);
    at = at < before ? at : before - 1;
    int low = 0, high = (EACH ? ITEMS : ITEMS / 4) * THREADS - 1;
    while (low < high) {
        const int middle = (low + high) >> 1;
        if (running[middle] > at) high = middle;
        else low = middle + 1;
    }
    if (!EACH) {
        uint64_t upto = low > 0 ? running[low - 1] : 0;
        int choice = 4 * low;
        for (int q = 0; q < 4; ++q) {
            const int j = 4 * low + q;
            if (j >= a.levels) break;
            const float v = a.type == TABX_F32 ? ((const float *)a.scores)[row + j]
                          : a.type == TABX_BF16 ? (float)((const __bf16 *)a.scores)[row + j]
                                                : (float)((const _Float16 *)a.scores)[row + j];
            const uint32_t k = a.level_mask && a.level_mask[j] == 0 ? 0u : score_key(v);
            const uint64_t c = (uint64_t)k << kIndexBits | (uint32_t)((1 << kIndexBits) - 1 - j);
            const uint64_t w = level_weight(k, top, a);
            if (k != 0 && c >= floor && w >= least) upto += w;
            choice = j;
            if (upto > at) break;
        }
        low = choice;
    }
    a.next_level[env] = low;
}

} // namespace tabx
