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
    int32_t     num_axes, heads, width, pairs, type, interleaved;
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

template <int TYPE>
__device__ __forceinline__ void load_some(float (&v)[4], const typename Element<TYPE>::one *at, int step, int count)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = i < count ? (float)at[i * step] : 0.0f;
}

template <int TYPE>
__device__ __forceinline__ void store_some(typename Element<TYPE>::one *at, int step, const float (&v)[4], int count)
{
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i < count) at[i * step] = (typename Element<TYPE>::one)v[i];
}

// LANES of a wavefront share a row, each with four of its pairs, whose angles serve all of the row's heads.
template <int LANES, int TYPE>
__global__ __launch_bounds__(256) void tabx_rotary_kernel(const RotaryArgs a)
{
    typedef typename Element<TYPE>::one T;
    constexpr int ROWS = 256 / LANES;              // of a workgroup at a time
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
        const T *x = (const T *)a.x + r * a.x_row;
        T *y = (T *)a.y + r * a.y_row;
        const int step = a.interleaved ? 2 : 1, other = a.interleaved ? 1 : a.pairs;
        const int from = step * first;
        for (int h = 0; h < a.heads; ++h, x += a.x_head, y += a.y_head) {
            float u[4], v[4], s[4], t[4];
            load_some<TYPE>(u, x + from, step, count);
            load_some<TYPE>(v, x + from + other, step, count);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                s[i] = fmaf(u[i], cosine[i], -(v[i] * sine[i]));
                t[i] = fmaf(u[i], sine[i], v[i] * cosine[i]);
            }
            store_some<TYPE>(y + from, step, s, count);
            store_some<TYPE>(y + from + other, step, t, count);
            if (a.copies)
                for (int j = lane; j < behind; j += LANES) y[2 * a.pairs + j] = x[2 * a.pairs + j];
        }
    }
}

} // namespace tabx
