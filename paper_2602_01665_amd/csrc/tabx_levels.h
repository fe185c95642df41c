// Draws of levels: one table of scores per env, or one for all of them.
//
// A workgroup holds a table in registers, four consecutive levels per thread and tile.  A level's score becomes a
// 32-bit number that is in order like the score, and with its index behind it a 46-bit one that no two levels share;
// what top_k and top_p leave is then "all levels from a threshold up".  The threshold is sought in two steps: a histogram
// over 256 equal ranges of the scores (how many levels, or how much weight, each has) says in which range it lies, and the
// few levels of that range are compared with each other.  Where a range holds too many (equal scores, or a few far from
// the rest), it is found eight bits of the 46-bit numbers at a time.  Weights are whole multiples of 2^-scale, so that
// their sums do not depend on the order of the additions.  The running sums of what is kept lie in LDS; each env then
// looks for its level in them by bisection.
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
    int32_t        share;          // envs of a workgroup, at most as many as it has threads (of one table for all)
    int32_t        scale;          // bits after the point of a weight
    double         log2e_by_temperature;
    float          reach;          // 44 temperatures below the largest score a weight is less than 2^-63
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

// 2^t * 2^scale for t <= 0, to the nearest whole number: the power of two nearest to 2^t, and for the rest, x = f ln2 within
// +-0.35, the series of e^x to x^13 (what is left out is below 2^-57).  It is below 2^52, so that adding 2^52 leaves it in
// the low bits.
__device__ __forceinline__ uint64_t power_of_two64(double t, int scale)
{
    t = fmax(t, -2000.0);
    const double n = rint(t), x = (t - n) * 0.69314718055994530942;
    double p = 1.0 / 6227020800.0;
    p = fma(p, x, 1.0 / 479001600.0);
    p = fma(p, x, 1.0 / 39916800.0);
    p = fma(p, x, 1.0 / 3628800.0);
    p = fma(p, x, 1.0 / 362880.0);
    p = fma(p, x, 1.0 / 40320.0);
    p = fma(p, x, 1.0 / 5040.0);
    p = fma(p, x, 1.0 / 720.0);
    p = fma(p, x, 1.0 / 120.0);
    p = fma(p, x, 1.0 / 24.0);
    p = fma(p, x, 1.0 / 6.0);
    p = fma(p, x, 0.5);
    p = fma(p, x, 1.0);
    p = fma(p, x, 1.0);
    return (uint64_t)__double_as_longlong(ldexp(p, (int)n + scale) + 0x1p52) & 0xfffffffffffffull;
}

__device__ __forceinline__ uint64_t level_weight(uint32_t key, float top, const LevelArgs &a)
{
    const float l = score_of(key);
    const double t = l == top ? 0.0 : ((double)l - (double)top) * a.log2e_by_temperature;
    const uint64_t w = power_of_two64(t, a.scale);
    return key != 0 ? w : 0;
}

// Which of 256 equal ranges below the largest score a score lies in; the last one has all that lies further off.
struct Ranges {
    float top, by;
    __device__ __forceinline__ Ranges(float top_, float bottom, float reach) : top(top_)
    {
        const float width = fminf(top - bottom, reach);
        by = width > 0.0f ? fminf(255.0f / width, 3e38f) : 0.0f;
    }
    __device__ __forceinline__ int of(uint32_t key) const
    {
        const float l = score_of(key);
        return l == top ? 0 : (int)fminf((top - l) * by, 255.0f);
    }
};

// v of the lane that the pattern names, 0 where it names none.
template <int PATTERN, int ROWS>
__device__ __forceinline__ uint64_t moved64(uint64_t v)
{
    const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)v, PATTERN, ROWS, 0xf, false);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(v >> 32), PATTERN, ROWS, 0xf, false);
    return (uint64_t)hi << 32 | lo;
}

// Running sum over the wavefront's lanes: within each sixteen of them, then of the sixteens before.
__device__ __forceinline__ uint64_t lanes_scan(uint64_t v)
{
    v += moved64<0x111, 0xf>(v);                   // row_shr 1, 2, 4, 8
    v += moved64<0x112, 0xf>(v);
    v += moved64<0x114, 0xf>(v);
    v += moved64<0x118, 0xf>(v);
    v += moved64<0x142, 0xa>(v);                   // row_bcast 15 to rows 1 and 3
    v += moved64<0x143, 0xc>(v);                   // row_bcast 31 to rows 2 and 3
    return v;
}

__device__ __forceinline__ uint64_t of_lane(uint64_t v, int lane)
{
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)v, lane);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(v >> 32), lane);
    return (uint64_t)hi << 32 | lo;
}

// Largest of v over the wavefront's lanes, in the last one.
__device__ __forceinline__ uint32_t lanes_max(uint32_t v)
{
#define TABX_LANES_MAX(PATTERN, ROWS) \
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, PATTERN, ROWS, 0xf, false));
    TABX_LANES_MAX(0x111, 0xf) TABX_LANES_MAX(0x112, 0xf) TABX_LANES_MAX(0x114, 0xf) TABX_LANES_MAX(0x118, 0xf)
    TABX_LANES_MAX(0x142, 0xa) TABX_LANES_MAX(0x143, 0xc)
#undef TABX_LANES_MAX
    return v;
}

// Largest of v, and of w, over the workgroup, in all threads.
template <int THREADS>
__device__ __forceinline__ void group_max(uint32_t &v, uint32_t &w, uint64_t *slots)
{
    const int lane = (int)threadIdx.x & 63;
    v = lanes_max(v);
    w = lanes_max(w);
    __syncthreads();
    if (lane == 63) slots[threadIdx.x >> 6] = (uint64_t)v << 32 | w;
    __syncthreads();
    const uint64_t both = lane < THREADS / 64 ? slots[lane & 15] : 0;
    v = (uint32_t)__builtin_amdgcn_readlane((int)lanes_max((uint32_t)(both >> 32)), 63);
    w = (uint32_t)__builtin_amdgcn_readlane((int)lanes_max((uint32_t)both), 63);
}

// Running sum over the workgroup's threads: what the threads before this one have, and the whole sum.
template <int THREADS>
__device__ __forceinline__ uint64_t group_scan(uint64_t v, uint64_t *slots, uint64_t &total)
{
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const uint64_t upto = lanes_scan(v);
    __syncthreads();
    if (lane == 63) slots[wave] = upto;
    __syncthreads();
    const uint64_t waves = lanes_scan(lane < THREADS / 64 ? slots[lane & 15] : 0);
    total = of_lane(waves, THREADS / 64 - 1);
    return upto - v + (wave > 0 ? of_lane(waves, wave > 0 ? wave - 1 : 0) : 0);
}

constexpr int kRivals = 256;       // most levels that are compared with each other

struct Rival {
    uint64_t number, weight;
};

struct LevelShared {
    uint64_t slots[16];
    uint64_t mass[256];
    uint32_t count[256];
    Rival    rivals[kRivals];
    uint32_t found;                // levels in the range
    int      digit;                // the range, or the eight bits, the threshold is in; -1: there is none
    uint64_t all, want;            // what is wanted in all, and what is left of it to be had there
    uint64_t within;               // how many levels it has
    uint64_t threshold;
};

__device__ __forceinline__ uint64_t level_number(uint32_t key, int j)
{
    return (uint64_t)key << kIndexBits | (uint32_t)((1 << kIndexBits) - 1 - j);
}

// Where the bins' contents, added up in falling order of the scores, reach what is wanted.  By the first wavefront.
// RISING: bin 0 has the largest scores.  MASS: weights count, else levels.  share < 1: wanted is that share of them all.
template <bool RISING, bool MASS>
__device__ __forceinline__ void cross(LevelShared &sh, uint64_t want, float share)
{
    const int lane = (int)threadIdx.x;
    uint64_t part[4], sum = 0;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const int bin = RISING ? 4 * lane + q : 255 - 4 * lane - q;
        part[q] = MASS ? sh.mass[bin] : sh.count[bin];
        sum += part[q];
    }
    const uint64_t upto = lanes_scan(sum);
    if (MASS && share < 1.0f) {
        const uint64_t all = of_lane(upto, 63);
        want = (uint64_t)ceil((double)share * (double)all);
        want = want < all ? want : all;
    }
    if (lane == 0) sh.all = want;
    uint64_t before = upto - sum;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        if (before < want && before + part[q] >= want) {
            const int bin = RISING ? 4 * lane + q : 255 - 4 * lane - q;
            sh.digit = bin;
            sh.want = want - before;
            sh.within = sh.count[bin];
        }
        before += part[q];
    }
}

// The number of the level that is the last to be kept, eight bits at a time.  want: how many levels (MASS false), or the
// weight that the levels before a kept one stay under (MASS true; > 0).  Only numbers >= floor compete.
template <int THREADS, int ITEMS, bool MASS>
__device__ __forceinline__ uint64_t threshold_by_bits(uint32_t (&key)[ITEMS], const uint64_t (&weight)[ITEMS], uint64_t floor,
                                                      uint64_t want, LevelShared &sh)
{
    uint64_t prefix = 0;
    // 48 bits from the top, the two highest of them always zero
#pragma unroll 1
    for (int shift = 40; shift >= 0; shift -= 8) {
        for (int b = (int)threadIdx.x; b < 256; b += THREADS) sh.count[b] = 0, sh.mass[b] = 0;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            if (THREADS * ITEMS > 8192) asm volatile("" : "+v"(key[i]));   // (the numbers of all levels at once would not fit either)
            const uint64_t c = level_number(key[i], ((i / 4) * THREADS + (int)threadIdx.x) * 4 + i % 4);
            if (key[i] != 0 && c >= floor && (c >> (shift + 8)) == (prefix >> (shift + 8))) {
                const int b = (int)(c >> shift) & 255;
                atomicAdd(&sh.count[b], 1u);
                if (MASS) atomicAdd((unsigned long long *)&sh.mass[b], (unsigned long long)weight[i]);
            }
        }
        __syncthreads();
        if (threadIdx.x < 64) cross<false, MASS>(sh, want, 1.0f);
        __syncthreads();
        prefix |= (uint64_t)(uint32_t)sh.digit << shift;
        want = sh.want;
        // all of them are kept, or the one there is: whatever its other bits are, it lies from here up
        const bool done = MASS ? sh.within == 1 : sh.within == want;
        __syncthreads();
        if (done) break;
    }
    return prefix;
}

// The same by ranges and rivals.  Of MASS, want is top_p times all that competes; without, top_k levels.  0: all are kept
// that have a weight.
template <int THREADS, int ITEMS, bool MASS>
__device__ __forceinline__ uint64_t threshold(uint32_t (&key)[ITEMS], const uint64_t (&weight)[ITEMS], const Ranges &ranges,
                                              uint64_t floor, const LevelArgs &a, LevelShared &sh)
{
    for (int b = (int)threadIdx.x; b < 256; b += THREADS) sh.count[b] = 0, sh.mass[b] = 0;
    if (threadIdx.x == 0) sh.found = 0, sh.digit = -1, sh.threshold = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        if (THREADS * ITEMS > 8192) asm volatile("" : "+v"(key[i]));
        if (key[i] != 0 && level_number(key[i], ((i / 4) * THREADS + (int)threadIdx.x) * 4 + i % 4) >= floor) {
            const int b = ranges.of(key[i]);
            atomicAdd(&sh.count[b], 1u);
            if (MASS) atomicAdd((unsigned long long *)&sh.mass[b], (unsigned long long)weight[i]);
        }
    }
    __syncthreads();
    if (threadIdx.x < 64) cross<true, MASS>(sh, (uint64_t)a.how.top_k, a.how.top_p);
    __syncthreads();
    const int range = sh.digit;
    const uint64_t want = sh.want;
    if (range < 0) return 0;                       // not even all of them are as many as that
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        if (THREADS * ITEMS > 8192) asm volatile("" : "+v"(key[i]));
        const uint64_t c = level_number(key[i], ((i / 4) * THREADS + (int)threadIdx.x) * 4 + i % 4);
        if (key[i] != 0 && c >= floor && ranges.of(key[i]) == range) {
            const uint64_t w = weight[i];
            if (w != 0) {                          // (one without is never drawn, wherever the threshold is)
                const uint32_t at = atomicAdd(&sh.found, 1u);
                if (at < (uint32_t)kRivals) sh.rivals[at] = Rival{c, w};
            }
        }
    }
    __syncthreads();
    const uint32_t found = sh.found;
    if (found > (uint32_t)kRivals) {
        const uint64_t all = sh.all;
        __syncthreads();
        return threshold_by_bits<THREADS, ITEMS, MASS>(key, weight, floor, all, sh);
    }
    if (threadIdx.x < found) {
        const Rival mine = sh.rivals[threadIdx.x];
        uint64_t before = 0;
#pragma unroll 4
        for (uint32_t n = 0; n < found; ++n) {
            const Rival other = sh.rivals[n];
            before += other.number > mine.number ? (MASS ? other.weight : 1) : 0;
        }
        if (before < want && before + (MASS ? mine.weight : 1) >= want) sh.threshold = mine.number;
    }
    __syncthreads();
    return sh.threshold;
}

// THREADS threads hold ITEMS levels each.  EACH: the running sums of single levels fit into LDS; else those of four.
// One table of up to 4096 levels is bound by its own latency: two trips to memory, the weights, and a dozen barriers for each
// threshold.  16384 envs, 4096 levels: 6.3 us (3.7 at temperature 0, which needs no weights), top_k 8.6, top_p 8.3, both 10.4,
// of which the vector instructions take 4.5; 5003 envs, 257 levels: 4.1.  More levels, or tables of the envs' own, are bound by
// vector instructions, most of them for the weights and for numbers of 64 bits: 4096 envs with tables of 2048 22 us (14.5 of
// instructions), with both 38 (23.9); one table of 16384 with both 28 (17.4).
template <int THREADS, int ITEMS, bool EACH>
__global__ __launch_bounds__(THREADS) void tabx_sample_levels_kernel(const LevelArgs a)
{
    __shared__ LevelShared sh;
    extern __shared__ __attribute__((aligned(16))) uint64_t running[];
    // the envs of this workgroup: one, or one for each thread
    const int group = (int)(blockIdx.y * gridDim.x + blockIdx.x);
    const int env = a.stride != 0 ? group : group * a.share + (int)threadIdx.x;
    const bool there = env < a.envs && (a.stride != 0 || (int)threadIdx.x < a.share);
    const bool wanted = there && (!a.env_mask || a.env_mask[env] != 0);
    if (a.stride != 0 && !wanted) return;
    const bool mine = wanted && (a.stride == 0 || threadIdx.x == 0);
    const float uniform = there ? a.uniform[env] : 0.0f;
    const int64_t row = a.stride * group;

    uint32_t key[ITEMS], most = 0, low_end = 0;   // low_end: the lowest key's complement
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
            low_end = max(low_end, key[4 * t + q] != 0 ? ~key[4 * t + q] : 0u);
        }
    }
    if (!__syncthreads_or(mine)) return;
    group_max<THREADS>(most, low_end, sh.slots);
    if (most == 0) return;                         // nothing to draw from: every env keeps what it has
    const float top = score_of(most);

    if (a.how.temperature == 0.0) {
        uint32_t rank = 0, none = 0;               // the lowest index counts most
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int j = ((i / 4) * THREADS + (int)threadIdx.x) * 4 + i % 4;
            if (key[i] == most) rank = max(rank, (uint32_t)((1 << kIndexBits) - j));
        }
        group_max<THREADS>(rank, none, sh.slots);
        if (mine) a.next_level[env] = (int32_t)((1 << kIndexBits) - rank);
        return;
    }

    uint64_t weight[ITEMS];
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) weight[i] = level_weight(key[i], top, a);

    const Ranges ranges(top, score_of(~low_end), a.reach);
    uint64_t floor = 0;
    if (a.how.top_k > 0 && a.how.top_k < a.levels) floor = threshold<THREADS, ITEMS, false>(key, weight, ranges, 0, a, sh);
    if (a.how.top_p < 1.0f) {
        __syncthreads();
        const uint64_t least = threshold<THREADS, ITEMS, true>(key, weight, ranges, floor, a, sh);
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
            const uint64_t c = level_number(key[4 * t + q], at * 4 + q);
            kept[q] = key[4 * t + q] != 0 && c >= floor ? weight[4 * t + q] : 0;
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
    const float u = uniform > 0.0f ? fminf(uniform, 0x1.fffffep-1f) : 0.0f;
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
            const uint64_t c = level_number(k, j);
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
