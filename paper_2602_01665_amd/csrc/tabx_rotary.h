// Rotation of pairs of a head's elements by angles that grow along several axes.
#pragma once
#include "tabx_rows.h"

#pragma clang fp contract(off)

namespace tabx {

struct RotaryArgs {
    const void *x;
    void       *y;
    const uint8_t *row_mask;
    const double  *frequency;
    const void *position[TABX_ROTARY_MAX_AXES];
    int64_t     rows, x_row, x_head, y_row, y_head;   // strides in elements
    int32_t     axis_type[TABX_ROTARY_MAX_AXES], units[TABX_ROTARY_MAX_AXES], end[TABX_ROTARY_MAX_AXES];   // end: of its pairs
    int32_t     num_axes, heads, width, pairs;
    int32_t     copies;            // the elements behind the pairs are copied (y is not x itself)
    double      sign;              // of the angles
};

// Cosine and sine of an angle given in quarter turns: the nearest whole number of them is taken off in 64 bits, what is
// left, at most pi / 4, goes through the two series up to its tenth and ninth power (the next terms are below 2^-33 and
// 2^-29), and the whole number says which of the two is which.  A position times its frequency is rounded to 64 bits
// twice, so that of 2^31 radians some 2^-21 are lost; of a thousand, nothing that 32 bits show.
__device__ __forceinline__ void quarter_turns(double quarters, float &cosine, float &sine)
{
    const double whole = __builtin_rint(quarters);
    const float a = (float)((quarters - whole) * 1.5707963267948966), s = a * a;
    const float sn = fmaf(a * s, fmaf(s, fmaf(s, fmaf(s, 2.7557319e-6f, -1.9841270e-4f), 8.3333333e-3f), -1.6666667e-1f), a);
    const float cs = fmaf(s, fmaf(s, fmaf(s, fmaf(s, fmaf(s, -2.7557319e-7f, 2.4801587e-5f), -1.3888889e-3f), 4.1666667e-2f), -0.5f), 1.0f);
    // (whole numbers beyond 2^31 keep their last two bits in what is left of them by multiples of four)
    const int turn = (int)(whole - 4.0 * __builtin_floor(whole * 0.25));
    const bool odd = turn & 1;
    const float c = odd ? sn : cs, d = odd ? cs : sn;
    cosine = (turn + 1) & 2 ? -c : c;
    sine = turn & 2 ? -d : d;
}

// Four elements (or fewer) of one kind of a pair, `step` apart.
template <int TYPE, int STEP>
__device__ __forceinline__ void load_some(f32x4 &v, const typename Element<TYPE>::one *at, int count)
{
    if (STEP == 1 && count == 4) {
        v = load_four<TYPE>(at);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = i < count ? (float)at[i * STEP] : 0.0f;
    }
}

template <int TYPE, int STEP>
__device__ __forceinline__ void store_some(typename Element<TYPE>::one *at, f32x4 v, int count)
{
    if (STEP == 1 && count == 4) {
        store_four<TYPE>(at, v);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < count) at[i * STEP] = (typename Element<TYPE>::one)v[i];
    }
}

// Four pairs (or fewer): the first elements in u, the second ones in v.
template <int TYPE, bool INTERLEAVED>
__device__ __forceinline__ void load_pairs(f32x4 &u, f32x4 &v, const typename Element<TYPE>::one *x, int first, int pairs, int count)
{
    if constexpr (!INTERLEAVED) {
        load_some<TYPE, 1>(u, x + first, count);
        load_some<TYPE, 1>(v, x + pairs + first, count);
    } else if (count == 4) {
        const f32x4 a = load_four<TYPE>(x + 2 * first), b = load_four<TYPE>(x + 2 * first + 4);
        u = __builtin_shufflevector(a, b, 0, 2, 4, 6), v = __builtin_shufflevector(a, b, 1, 3, 5, 7);
    } else {
        load_some<TYPE, 2>(u, x + 2 * first, count);
        load_some<TYPE, 2>(v, x + 2 * first + 1, count);
    }
}

template <int TYPE, bool INTERLEAVED>
__device__ __forceinline__ void store_pairs(f32x4 u, f32x4 v, typename Element<TYPE>::one *y, int first, int pairs, int count)
{
    if constexpr (!INTERLEAVED) {
        store_some<TYPE, 1>(y + first, u, count);
        store_some<TYPE, 1>(y + pairs + first, v, count);
    } else if (count == 4) {
        store_four<TYPE>(y + 2 * first, __builtin_shufflevector(u, v, 0, 4, 1, 5));
        store_four<TYPE>(y + 2 * first + 4, __builtin_shufflevector(u, v, 2, 6, 3, 7));
    } else {
        store_some<TYPE, 2>(y + 2 * first, u, count);
        store_some<TYPE, 2>(y + 2 * first + 1, v, count);
    }
}

// LANES of a wavefront share a row, each with four of its pairs, whose angles serve all of the row's heads; HEADS of them are
// on their way at a time.
template <int LANES, int TYPE, bool INTERLEAVED>
__global__ __launch_bounds__(256) void tabx_rotary_kernel(const RotaryArgs a)
{
    typedef typename Element<TYPE>::one T;
    constexpr int ROWS = 256 / LANES;              // of a workgroup at a time
    constexpr int HEADS = 4;
    const int lane = (int)threadIdx.x % LANES, first = 4 * lane;
    const int count = max(0, min(4, a.pairs - first));
    double frequency[4];
    int axis[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int p = min(first + i, a.pairs - 1);
        frequency[i] = a.frequency[p] * (a.sign * 0.63661977236758134);       // quarter turns
        axis[i] = 0;
#pragma unroll
        for (int n = 1; n < TABX_ROTARY_MAX_AXES; ++n) axis[i] += n < a.num_axes && p >= a.end[n - 1];
    }
    const int behind = a.width - 2 * a.pairs;
    for (int64_t r = (int64_t)blockIdx.x * ROWS + threadIdx.x / LANES; r < a.rows; r += (int64_t)gridDim.x * ROWS) {
        if (a.row_mask && a.row_mask[r] == 0) continue;
        const T *x = (const T *)a.x + r * a.x_row;
        T *y = (T *)a.y + r * a.y_row;
        f32x4 u[HEADS], v[HEADS];
        const auto fetch = [&](int h) {
#pragma unroll
            for (int n = 0; n < HEADS; ++n) load_pairs<TYPE, INTERLEAVED>(u[n], v[n], x + min(h + n, a.heads - 1) * a.x_head, first, a.pairs, count);
        };
        fetch(0);
        double where[TABX_ROTARY_MAX_AXES];
#pragma unroll
        for (int n = 0; n < TABX_ROTARY_MAX_AXES; ++n) {
            where[n] = 0.0;
            if (n >= a.num_axes) continue;
            const int64_t at = a.units[n] == 1 ? r : r >> 32 ? r / a.units[n] : (int64_t)((uint32_t)r / (uint32_t)a.units[n]);
            where[n] = a.axis_type[n] == TABX_I32 ? (double)((const int32_t *)a.position[n])[at] : (double)((const float *)a.position[n])[at];
        }
        float cosine[4], sine[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const double p = axis[i] == 0 ? where[0] : axis[i] == 1 ? where[1] : axis[i] == 2 ? where[2] : where[3];
            quarter_turns(p * frequency[i], cosine[i], sine[i]);
        }
        for (int h = 0; h < a.heads; h += HEADS) {
            if (h > 0) fetch(h);
#pragma unroll
            for (int n = 0; n < HEADS; ++n) {
                if (h + n >= a.heads) break;
                f32x4 s, t;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    s[i] = fmaf(u[n][i], cosine[i], -(v[n][i] * sine[i]));
                    t[i] = fmaf(u[n][i], sine[i], v[n][i] * cosine[i]);
                }
                store_pairs<TYPE, INTERLEAVED>(s, t, y + (h + n) * a.y_head, first, a.pairs, count);
            }
        }
        if (a.copies)
            for (int h = 0; h < a.heads; ++h)
                for (int j = lane; j < behind; j += LANES) y[h * a.y_head + 2 * a.pairs + j] = x[h * a.x_head + 2 * a.pairs + j];
    }
}

} // namespace tabx
