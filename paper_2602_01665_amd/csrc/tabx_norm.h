// Layer norm of rows and its gradients.
//
// A row of W elements is held in registers by LANES lanes, PIECES pieces of four consecutive elements each (piece q
// of lane l starts at element 4 (q LANES + l)), so the mean and the sum of squared differences from it are two
// passes over registers and one over memory.
#pragma once
#include "tabx_rows.h"

#pragma clang fp contract(off)

namespace tabx {

struct NormArgs {
    const void *x;
    void       *y;                 // forward: the result; backward: the input's gradient, or nullptr
    const void *grad_y;            // backward only
    const uint8_t *row_mask;
    const float *weight, *bias;
    float      *mean, *rstd;       // forward: written; backward: read
    float      *partial;           // backward: [workgroup][2][width]
    int64_t     rows, x_stride, y_stride, g_stride;
    int32_t     width, x_type, y_type, g_type;
    float       eps, inv_width;
};

// PIECES pieces of a row that starts at `row`; zero behind its end.
template <int TYPE, int LANES, int PIECES>
__device__ __forceinline__ void load_pieces(f32x4 (&v)[PIECES], const void *data, int64_t offset, int lane, int width)
{
    typedef typename Element<TYPE>::one T;
    const T *row = (const T *)data + offset;
#pragma unroll
    for (int q = 0; q < PIECES; ++q) {
        const int j = 4 * (q * LANES + lane);
        v[q] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        if (j + 4 <= width) {
            v[q] = load_four<TYPE>(row + j);
        } else if (j < width) {
            v[q].x = (float)row[j];
            if (j + 1 < width) v[q].y = (float)row[j + 1];
            if (j + 2 < width) v[q].z = (float)row[j + 2];
        }
    }
}

template <int LANES, int PIECES>
__device__ __forceinline__ void load_row(f32x4 (&v)[PIECES], const void *data, int type, int64_t offset, int lane, int width)
{
    if (type == TABX_F32) load_pieces<TABX_F32, LANES, PIECES>(v, data, offset, lane, width);
    else if (type == TABX_BF16) load_pieces<TABX_BF16, LANES, PIECES>(v, data, offset, lane, width);
    else load_pieces<TABX_F16, LANES, PIECES>(v, data, offset, lane, width);
}

template <int TYPE, int LANES, int PIECES>
__device__ __forceinline__ void store_pieces(const f32x4 (&v)[PIECES], void *data, int64_t offset, int lane, int width)
{
    typedef typename Element<TYPE>::one T;
    T *row = (T *)data + offset;
#pragma unroll
    for (int q = 0; q < PIECES; ++q) {
        const int j = 4 * (q * LANES + lane);
        if (j + 4 <= width) {
            store_four<TYPE>(row + j, v[q]);
        } else if (j < width) {
            row[j] = (T)v[q].x;
            if (j + 1 < width) row[j + 1] = (T)v[q].y;
            if (j + 2 < width) row[j + 2] = (T)v[q].z;
        }
    }
}

template <int LANES, int PIECES>
__device__ __forceinline__ void store_row(const f32x4 (&v)[PIECES], void *data, int type, int64_t offset, int lane, int width)
{
    if (type == TABX_F32) store_pieces<TABX_F32, LANES, PIECES>(v, data, offset, lane, width);
    else if (type == TABX_BF16) store_pieces<TABX_BF16, LANES, PIECES>(v, data, offset, lane, width);
    else store_pieces<TABX_F16, LANES, PIECES>(v, data, offset, lane, width);
}

// Sum over the lanes of a row; rows of more than a wavefront meet in `slots` (one float per wavefront; a call uses
// slots that no wavefront can still be reading: those of the call before the last).
template <int LANES>
__device__ __forceinline__ float row_sum(float v, float *slots)
{
    v = lanes_sum<(LANES < 64 ? LANES : 64)>(v);
    if (LANES > 64) {
        if ((threadIdx.x & 63) == 0) slots[threadIdx.x >> 6] = v;
        __syncthreads();
        v = 0.0f;
#pragma unroll
        for (int w = 0; w < LANES / 64; ++w) v += slots[w];
    }
    return v;
}

__device__ __forceinline__ float sum_of(f32x4 v) { return (v.x + v.y) + (v.z + v.w); }

// The first columns behind the row's end are zero in registers, but not after the mean has been taken off.
__device__ __forceinline__ f32x4 inside(f32x4 v, int j, int width)
{
    if (j + 4 > width) {
        if (j >= width) v.x = 0.0f;
        if (j + 1 >= width) v.y = 0.0f;
        if (j + 2 >= width) v.z = 0.0f;
        if (j + 3 >= width) v.w = 0.0f;
    }
    return v;
}

template <int LANES, int PIECES>
__global__ __launch_bounds__(LANES > 256 ? LANES : 256) void tabx_norm_kernel(const NormArgs a)
{
    constexpr int THREADS = LANES > 256 ? LANES : 256;
    constexpr int ROWS = THREADS / LANES;          // rows a workgroup works on at a time
    __shared__ float slots[4][THREADS / 64];
    const int lane = (int)threadIdx.x % LANES;
    f32x4 w[PIECES], b[PIECES];
    const f32x4 one = {1.0f, 1.0f, 1.0f, 1.0f}, zero = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int q = 0; q < PIECES; ++q) w[q] = one, b[q] = zero;
    if (a.weight) load_pieces<TABX_F32, LANES>(w, a.weight, 0, lane, a.width);
    if (a.bias) load_pieces<TABX_F32, LANES>(b, a.bias, 0, lane, a.width);
    int turn = 0;
    for (int64_t first = (int64_t)blockIdx.x * ROWS; first < a.rows; first += (int64_t)gridDim.x * ROWS) {
        const int64_t r = first + (LANES < 256 ? (int)threadIdx.x / LANES : 0);
        const bool on = r < a.rows && (!a.row_mask || a.row_mask[r] != 0);
        if (LANES > 64 && !on) continue;           // (the same for the whole workgroup)
        f32x4 v[PIECES];
        if (on) {
            load_row<LANES>(v, a.x, a.x_type, r * a.x_stride, lane, a.width);
        } else {
#pragma unroll
            for (int q = 0; q < PIECES; ++q) v[q] = zero;
        }
        float s = 0.0f;
#pragma unroll
        for (int q = 0; q < PIECES; ++q) s += sum_of(v[q]);
        const float mean = row_sum<LANES>(s, slots[turn]) * a.inv_width;
        s = 0.0f;
#pragma unroll
        for (int q = 0; q < PIECES; ++q) {
            v[q] = inside(v[q] - mean, 4 * (q * LANES + lane), a.width);
            s += sum_of(v[q] * v[q]);
        }
        const float rstd = 1.0f / sqrtf(row_sum<LANES>(s, slots[turn + 1]) * a.inv_width + a.eps);
        turn ^= 2;
        if (!on) continue;
#pragma unroll
        for (int q = 0; q < PIECES; ++q) v[q] = v[q] * rstd * w[q] + b[q];
        store_row<LANES>(v, a.y, a.y_type, r * a.y_stride, lane, a.width);
        if (a.mean && lane == 0) {
            a.mean[r] = mean;
            a.rstd[r] = rstd;
        }
    }
}

// INPUTS: the input's gradient is wanted; WEIGHTS: the sums over rows are.  Each workgroup adds up its rows' parts of
// the weight's and the bias's gradient in registers, one column set per lane, and leaves them in a.partial.
template <int LANES, int PIECES, bool INPUTS, bool WEIGHTS>
__global__ __launch_bounds__(LANES > 256 ? LANES : 256) void tabx_norm_grad_kernel(const NormArgs a)
{
    constexpr int THREADS = LANES > 256 ? LANES : 256;
    constexpr int ROWS = THREADS / LANES;
    constexpr int WAVES = THREADS / 64;
    __shared__ float slots[4][WAVES];
    __shared__ f32x4 meet[WEIGHTS && LANES <= 64 ? WAVES : 1][WEIGHTS && LANES <= 64 ? LANES : 1];
    const int lane = (int)threadIdx.x % LANES;
    const f32x4 one = {1.0f, 1.0f, 1.0f, 1.0f}, zero = {0.0f, 0.0f, 0.0f, 0.0f};
    f32x4 w[INPUTS ? PIECES : 1], dw[PIECES], db[PIECES];
#pragma unroll
    for (int q = 0; q < PIECES; ++q) dw[q] = zero, db[q] = zero, w[INPUTS ? q : 0] = one;
    if (INPUTS && a.weight) load_row<LANES>(w, a.weight, TABX_F32, 0, lane, a.width);
    int turn = 0;
    for (int64_t first = (int64_t)blockIdx.x * ROWS; first < a.rows; first += (int64_t)gridDim.x * ROWS) {
        const int64_t r = first + (LANES < 256 ? (int)threadIdx.x / LANES : 0);
        const bool on = r < a.rows && (!a.row_mask || a.row_mask[r] != 0);
        f32x4 x[PIECES], g[PIECES];
        float rstd = 0.0f;
        if (on) {
            load_row<LANES>(x, a.x, a.x_type, r * a.x_stride, lane, a.width);
            load_row<LANES>(g, a.grad_y, a.g_type, r * a.g_stride, lane, a.width);
            const float mean = a.mean[r];
            rstd = a.rstd[r];
#pragma unroll
            for (int q = 0; q < PIECES; ++q) {
                x[q] = inside((x[q] - mean) * rstd, 4 * (q * LANES + lane), a.width);
                if (WEIGHTS) {
                    dw[q] += g[q] * x[q];
                    db[q] += g[q];
                }
            }
        } else {
#pragma unroll
            for (int q = 0; q < PIECES; ++q) x[q] = zero, g[q] = zero;
        }
        if (INPUTS) {
            float sg = 0.0f, sh = 0.0f;
#pragma unroll
            for (int q = 0; q < PIECES; ++q) {
                g[q] *= w[INPUTS ? q : 0];
                sg += sum_of(g[q]);
                sh += sum_of(g[q] * x[q]);
            }
            sg = row_sum<LANES>(sg, slots[turn]) * a.inv_width;
            sh = row_sum<LANES>(sh, slots[turn + 1]) * a.inv_width;
            turn ^= 2;
#pragma unroll
            for (int q = 0; q < PIECES; ++q) g[q] = on ? (g[q] - sg - x[q] * sh) * rstd : zero;
            if (r < a.rows) store_row<LANES>(g, a.y, a.y_type, r * a.y_stride, lane, a.width);
        }
    }
    if (!WEIGHTS) return;
    // the row groups of a wavefront, then the wavefronts
    float *const out = a.partial + (int64_t)blockIdx.x * 2 * a.width;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
#pragma unroll
        for (int q = 0; q < PIECES; ++q) {
            f32x4 v = half ? db[q] : dw[q];
            if (LANES <= 64) {
#pragma unroll
                for (int d = LANES; d < 64; d *= 2) {
                    v.x += __shfl_xor(v.x, d);
                    v.y += __shfl_xor(v.y, d);
                    v.z += __shfl_xor(v.z, d);
                    v.w += __shfl_xor(v.w, d);
                }
                __syncthreads();                   // the piece before has been read
                if ((int)(threadIdx.x & 63) < LANES) meet[LANES <= 64 ? threadIdx.x >> 6 : 0][LANES <= 64 ? lane : 0] = v;
                __syncthreads();
                if ((int)threadIdx.x >= LANES) continue;
                v = meet[0][LANES <= 64 ? lane : 0];
#pragma unroll
                for (int k = 1; k < WAVES; ++k) v += meet[LANES <= 64 ? k : 0][LANES <= 64 ? lane : 0];
            }
            const int j = 4 * (q * LANES + lane);
            float *at = out + half * a.width + j;
            if (j + 4 <= a.width) {
                store_four<TABX_F32>(at, v);
            } else if (j < a.width) {
                at[0] = v.x;
                if (j + 1 < a.width) at[1] = v.y;
                if (j + 2 < a.width) at[2] = v.z;
            }
        }
    }
}

// Adds up the workgroups' parts: 32 columns per workgroup, 32 runs of parts side by side, always in the same order.
__global__ __launch_bounds__(1024) void tabx_norm_join_kernel(const float *partial, int parts, int width, float *grad_weight,
                                                              float *grad_bias)
{
    __shared__ float meet[32][33];
    const int c = (int)threadIdx.x & 31, run = (int)threadIdx.x >> 5;
    const int j = (int)blockIdx.x * 32 + c;
    float s = 0.0f;
    if (j < 2 * width) {
#pragma unroll 8
        for (int k = run; k < parts; k += 32) s += partial[(int64_t)k * 2 * width + j];
    }
    meet[run][c] = s;
    __syncthreads();
    if (run != 0 || j >= 2 * width) return;
#pragma unroll
    for (int k = 1; k < 32; ++k) s += meet[k][c];
    float *const out = j < width ? grad_weight : grad_bias;
    if (out) out[j < width ? j : j - width] = s;
}

} // namespace tabx
