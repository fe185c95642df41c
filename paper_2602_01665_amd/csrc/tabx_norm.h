// Layer norm of rows and its gradients: the mean and the sum of squared differences from it are two passes over a row's
// registers (tabx_teams.h).
#pragma once
#include "tabx_teams.h"

#pragma clang fp contract(off)

namespace tabx {

struct NormArgs {
    const void *x;
    void       *y;                 // forward: the result; backward: the input's gradient, or nullptr
    const void *grad_y;            // backward only
    const uint8_t *row_mask;
    const float *weight, *bias;
    float      *mean, *rstd;       // forward: written; backward: read
    float      *partial;           // backward: [workgroup][2][width], or nullptr
    float      *grad_weight, *grad_bias;   // backward of a single workgroup, if `partial` is nullptr
    int64_t     rows, x_stride, y_stride, g_stride;
    int64_t     team_rows, lap;    // a team's rows are runs of at most 64 of them, `lap` rows from one run to the next
    int32_t     width, x_type, y_type, g_type;
    float       eps, inv_width;
    int32_t     stream;            // forward: the result goes past the caches
};

// Bound by HBM.  Rows go through the machine in the order of their addresses: a team has few rows, and the next
// workgroup's lie behind its own (a wavefront of 64 rows: 85 us, of 4: 76, 10v10 x 16384, half of the rows).  71 us, 5.1
// TB/s of x and y (a large copy on this card: 5.2); 64v64 x 1024, all rows, 281 us, 5.7 TB/s.
template <int LANES, int PIECES, int X_BYTES>
__global__ __launch_bounds__(threads_of(LANES)) void tabx_norm_kernel(const NormArgs a)
{
    constexpr int THREADS = threads_of(LANES);
    __shared__ float slots[4][THREADS / 64];
    const Cut<LANES, PIECES> cut(a.width);
    Walk<LANES> walk(a);
    f32x4 w[PIECES], b[PIECES];
    load_columns(w, a.weight, 1.0f, cut, a.width);
    load_columns(b, a.bias, 0.0f, cut, a.width);
    int turn = 0;
    struct Rows {
        RawRow<X_BYTES, PIECES> x;
        int64_t r;
    };
    const auto more = [&] { return walk.more([] {}); };
    const auto fetch = [&](Rows &h, bool some, const Rows &last) {
        bool own;
        h.r = some ? walk.take(walk.on, own) : last.r;
        load_raw(h.x, a.x, h.r * a.x_stride, cut, a.width);
    };
    const auto work = [&](const Rows &h) {
        f32x4 v[PIECES];
        unpack(v, h.x, a.x_type);
        f32x4 sum = cut.counted(v[PIECES - 1]);
#pragma unroll
        for (int q = 0; q < PIECES - 1; ++q) sum += v[q];
        const float mean = row_sum<LANES>(sum_of(sum), slots[turn]) * a.inv_width;
#pragma unroll
        for (int q = 0; q < PIECES; ++q) v[q] -= mean;
        const f32x4 last = cut.counted(v[PIECES - 1]);
        f32x4 squares = last * last;
#pragma unroll
        for (int q = 0; q < PIECES - 1; ++q) squares = fma4(v[q], v[q], squares);
        const float rstd = rsqrtf(fmaf(row_sum<LANES>(sum_of(squares), slots[turn + 1]), a.inv_width, a.eps));
        turn ^= 2;
        if (a.mean && cut.lane == 0) {
            a.mean[h.r] = mean;
            a.rstd[h.r] = rstd;
        }
#pragma unroll
        for (int q = 0; q < PIECES; ++q) v[q] = fma4(v[q] * rstd, w[q], b[q]);
        if (a.stream) store_row<true>(v, a.y, a.y_type, h.r * a.y_stride, cut, a.width);
        else store_row(v, a.y, a.y_type, h.r * a.y_stride, cut, a.width);
    };
    walk_through<kNormAhead<LANES>, Rows>(more, fetch, work);
}

// INPUTS: the input's gradient is wanted.  Each workgroup adds up its rows' parts of the weight's and the bias's
// gradient in registers, one column set per lane, and leaves them in a.partial (if that is given).  Bound by HBM: a
// workgroup stays, for the sake of its sums, but its teams take short runs of rows a lap apart, so that the machine goes
// through the rows in the order of their addresses all the same (200000 rows of 512 in bf16 136 us with a long run per
// team, 121 with runs of four rows, 5.1 TB/s; 85051 rows 61 and 56).
// ONCE: more is read than the memory-side cache holds, so nothing of it is kept (10v10 x 16384 without the input's
// gradient, 364 MB: 64 us, 5.7 TB/s, 69 without; 66 MB: 14.4 and 13.3; with the input's gradient it is slower, 182 us
// and 171, 200000 rows of 700).  Rows that are masked out count, as the host does not see them; a call that reads half of
// that gains too (132 MB of 265: 28.6 us and 31.3).
template <int LANES, int PIECES, int X_BYTES, int G_BYTES, bool INPUTS, bool ONCE>
__global__ __launch_bounds__(threads_of(LANES), grad_wavefronts(PIECES)) void tabx_norm_grad_kernel(const NormArgs a)
{
    constexpr int THREADS = threads_of(LANES);
    constexpr int WAVES = THREADS / 64;
    __shared__ float slots[4][WAVES];
    __shared__ f32x4 meet[LANES <= 64 ? WAVES : 1][LANES <= 64 ? LANES : 1];
    const Cut<LANES, PIECES> cut(a.width);
    const f32x4 zero = {0.0f, 0.0f, 0.0f, 0.0f};
    Walk<LANES> walk(a);
    f32x4 w[INPUTS ? PIECES : 1], dw[PIECES], db[PIECES];
    if constexpr (INPUTS) load_columns(w, a.weight, 1.0f, cut, a.width);
#pragma unroll
    for (int q = 0; q < PIECES; ++q) dw[q] = zero, db[q] = zero;
    const bool sums = !INPUTS || a.partial || a.grad_weight || a.grad_bias;
    // a row's mean and rstd are the same for a whole wavefront; without a lane's own address they would be moved to
    // scalar registers as soon as they are loaded, and waited for
    int here = 0;
    asm("v_mov_b32 %0, 0" : "=v"(here));
    int turn = 0;
    struct Rows {
        RawRow<X_BYTES, PIECES> x;
        RawRow<G_BYTES, PIECES> g;
        float   mean, rstd;
        int64_t r;
        bool    own;
    };
    const auto more = [&] {
        return walk.more([&] {
            if constexpr (INPUTS) {                // rows that are masked out have no gradient
                f32x4 none[PIECES];
#pragma unroll
                for (int q = 0; q < PIECES; ++q) none[q] = zero;
                while (walk.off) {
                    bool own;
                    store_row(none, a.y, a.y_type, walk.take(walk.off, own) * a.y_stride, cut, a.width);
                }
            }
        });
    };
    const auto fetch = [&](Rows &h, bool some, const Rows &last) {
        h.r = some ? walk.take(walk.on, h.own) : last.r;
        h.mean = (a.mean + h.r)[here];
        h.rstd = (a.rstd + h.r)[here];
        load_raw<ONCE>(h.x, a.x, h.r * a.x_stride, cut, a.width);
        load_raw<ONCE>(h.g, a.grad_y, h.r * a.g_stride, cut, a.width);
    };
    const auto work = [&](const Rows &h) {
        f32x4 x[PIECES], g[PIECES];
        unpack(x, h.x, a.x_type);
        unpack(g, h.g, a.g_type);
#pragma unroll
        for (int q = 0; q < PIECES; ++q) x[q] = (x[q] - h.mean) * h.rstd;
        const f32x4 last = cut.counted(g[PIECES - 1]);
        if (sums && (LANES >= 64 || h.own)) {
#pragma unroll
            for (int q = 0; q < PIECES; ++q) {
                const f32x4 t = q < PIECES - 1 ? g[q] : last;
                dw[q] = fma4(t, x[q], dw[q]);
                db[q] += t;
            }
        }
        if constexpr (INPUTS) {
            f32x4 total = last * w[PIECES - 1], along = total * x[PIECES - 1];
#pragma unroll
            for (int q = 0; q < PIECES; ++q) {
                g[q] *= w[q];
                if (q < PIECES - 1) {
                    total += g[q];
                    along = fma4(g[q], x[q], along);
                }
            }
            const float sg = row_sum<LANES>(sum_of(total), slots[turn]) * a.inv_width;
            const float sh = row_sum<LANES>(sum_of(along), slots[turn + 1]) * a.inv_width;
            turn ^= 2;
#pragma unroll
            for (int q = 0; q < PIECES; ++q) g[q] = (fma4(x[q], f32x4{-sh, -sh, -sh, -sh}, g[q]) - sg) * h.rstd;
            store_row(g, a.y, a.y_type, h.r * a.y_stride, cut, a.width);
        }
    };
    walk_through<kGradAhead<LANES>, Rows>(more, fetch, work);
    if (!sums) return;
    // the rows worked on side by side in a wavefront, then the wavefronts
    const int64_t part = (int64_t)blockIdx.x * 2 * a.width;
    float *const outs[2] = {a.partial ? a.partial + part : a.grad_weight, a.partial ? a.partial + part + a.width : a.grad_bias};
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        float *const out = outs[half];
        if (!out) continue;                        // (the same for all)
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
                if ((int)(threadIdx.x & 63) < LANES) meet[LANES <= 64 ? threadIdx.x >> 6 : 0][LANES <= 64 ? cut.lane : 0] = v;
                __syncthreads();
                if ((int)threadIdx.x >= LANES) continue;
                v = meet[0][LANES <= 64 ? cut.lane : 0];
#pragma unroll
                for (int k = 1; k < WAVES; ++k) v += meet[LANES <= 64 ? k : 0][LANES <= 64 ? cut.lane : 0];
            }
            float *at = out + cut.at(q);
            if (q < PIECES - 1) {
                store_four<TABX_F32>(at, v);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (cut.counts(i)) at[i] = v[i];
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
