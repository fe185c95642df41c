// Root-mean-square norm of rows behind a residual addition, to 8 bits too, and its gradients.  A row stays in registers
// from its loads to its last store (tabx_teams.h).
#pragma once
#include "tabx_teams.h"

#pragma clang fp contract(off)

namespace tabx {

struct RmsArgs {
    const void *x, *residual;      // forward; x is the sum that was normed in the backward pass
    void       *sum, *y;           // forward: y is the result; backward: the input's gradient, or nullptr
    const void *grad_y, *grad_sum; // backward only
    const uint8_t *row_mask;
    const float *weight;
    float      *scale, *rstd;      // forward: written; backward: rstd is read
    float      *partial;           // backward: [workgroup][width], or nullptr
    float      *grad_weight;       // backward of a single workgroup, if `partial` is nullptr
    int64_t     rows, x_stride, residual_stride, sum_stride, y_stride, g_stride, grad_sum_stride;
    int64_t     team_rows, lap;    // a team's rows are runs of at most 64 of them, `lap` rows from one run to the next
    int32_t     width, x_type, residual_type, sum_type, y_type, g_type;
    float       eps, inv_width;
    int32_t     stream;            // forward: the results go past the caches
};

constexpr float kLargestE4m3 = 448.0f, kLeastScale = 0x1p-126f;

// Four results of eight bits, to nearest even; their magnitudes round to 448 at the most.
template <bool STREAM>
__device__ __forceinline__ void store_four_e4m3(uint8_t *at, f32x4 v)
{
    typedef uint32_t Anywhere __attribute__((aligned(1)));
    int r = __builtin_amdgcn_cvt_pk_fp8_f32(v.x, v.y, 0, false);
    r = __builtin_amdgcn_cvt_pk_fp8_f32(v.z, v.w, r, true);
    if (STREAM) __builtin_nontemporal_store((uint32_t)r, (Anywhere *)at);
    else *(Anywhere *)at = (uint32_t)r;
}

template <bool STREAM, int LANES, int PIECES>
__device__ __forceinline__ void store_row_e4m3(const f32x4 (&v)[PIECES], void *data, int64_t offset, const Cut<LANES, PIECES> &cut,
                                               int width)
{
    uint8_t *row = (uint8_t *)data + offset;
    if constexpr (LANES == 1) {
        const int r = __builtin_amdgcn_cvt_pk_fp8_f32(v[0].z, v[0].w, __builtin_amdgcn_cvt_pk_fp8_f32(v[0].x, v[0].y, 0, false), true);
        row[0] = (uint8_t)r;
        if (width > 1) row[1] = (uint8_t)(r >> 8);
        if (width > 2) row[2] = (uint8_t)(r >> 16);
        if (width > 3) row[3] = (uint8_t)(r >> 24);
    } else {
#pragma unroll
        for (int q = 0; q < PIECES; ++q) store_four_e4m3<STREAM>(row + cut.at(q), v[q]);
    }
}

// To the type and back: what a reader of the stored value sees.
template <int PIECES>
__device__ __forceinline__ void round_to(f32x4 (&v)[PIECES], int type)
{
    if (type == TABX_BF16) {
#pragma unroll
        for (int q = 0; q < PIECES; ++q) v[q] = __builtin_convertvector(__builtin_convertvector(v[q], bf16x4), f32x4);
    } else if (type == TABX_F16) {
#pragma unroll
        for (int q = 0; q < PIECES; ++q) v[q] = __builtin_convertvector(__builtin_convertvector(v[q], f16x4), f32x4);
    }
}

// Largest over the lanes of a row, in all of them; NaN is passed over.
template <int LANES>
__device__ __forceinline__ float row_max(float v, float *slots)
{
#pragma unroll
    for (int d = 1; d < (LANES < 64 ? LANES : 64); d *= 2) v = fmaxf(v, __shfl_xor(v, d));
    if (LANES > 64) {
        if ((threadIdx.x & 63) == 0) slots[threadIdx.x >> 6] = v;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < LANES / 64; ++w) v = fmaxf(v, slots[w]);
    }
    return v;
}

// s = x + residual, y = s rstd w.  Bound by HBM: 112 us for 163840 of 327680 rows of 512 in bf16 to e4m3, 5.2 TB/s of x,
// residual, sum and y (a large copy: 5.2).  Rows go through the machine in the order of their addresses (tabx_memory.hip:
// kRmsTeams).  96 rows of 128 take 3 us, with their launch 8.5.
template <int LANES, int PIECES, int X_BYTES, int R_BYTES>
__global__ __launch_bounds__(threads_of(LANES)) void tabx_rms_kernel(const RmsArgs a)
{
    constexpr int THREADS = threads_of(LANES);
    __shared__ float slots[4][THREADS / 64];
    const Cut<LANES, PIECES> cut(a.width);
    Walk<LANES> walk(a);
    f32x4 w[PIECES];
    load_columns(w, a.weight, 1.0f, cut, a.width);
    int turn = 0;
    struct Rows {
        RawRow<X_BYTES, PIECES> x;
        RawRow<R_BYTES ? R_BYTES : 2, R_BYTES ? PIECES : 1> r;
        int64_t at;
    };
    const auto more = [&] { return walk.more([] {}); };
    const auto fetch = [&](Rows &h, bool some, const Rows &last) {
        bool own;
        h.at = some ? walk.take(walk.on, own) : last.at;
        load_raw(h.x, a.x, h.at * a.x_stride, cut, a.width);
        if constexpr (R_BYTES > 0) load_raw(h.r, a.residual, h.at * a.residual_stride, cut, a.width);
    };
    const auto work = [&](const Rows &h) {
        f32x4 v[PIECES];
        unpack(v, h.x, a.x_type);
        if constexpr (R_BYTES > 0) {
            f32x4 r[PIECES];
            unpack(r, h.r, a.residual_type);
#pragma unroll
            for (int q = 0; q < PIECES; ++q) v[q] += r[q];
        }
        if (a.sum) round_to(v, a.sum_type);
        const f32x4 last = cut.counted(v[PIECES - 1]);
        f32x4 squares = last * last;
#pragma unroll
        for (int q = 0; q < PIECES - 1; ++q) squares = fma4(v[q], v[q], squares);
        const float rstd = rsqrtf(fmaf(row_sum<LANES>(sum_of(squares), slots[turn]), a.inv_width, a.eps));
        if (a.rstd && cut.lane == 0) a.rstd[h.at] = rstd;
        // (the sum may lie where x or the residual does: not before all of the team has the row's last elements, which
        // several lanes read)
        if (a.sum) {
            if (a.stream) store_row<true>(v, a.sum, a.sum_type, h.at * a.sum_stride, cut, a.width);
            else store_row(v, a.sum, a.sum_type, h.at * a.sum_stride, cut, a.width);
        }
        if (a.y_type == TABX_E4M3) {
            // y / scale is (s w) (448 / largest |s w|): rstd is in both and need not be rounded into either.  (Elements that
            // lie in two pieces are as large in both.)
            float most = 0.0f;
#pragma unroll
            for (int q = 0; q < PIECES; ++q) {
                v[q] *= w[q];
                most = fmaxf(most, fmaxf(fmaxf(fabsf(v[q].x), fabsf(v[q].y)), fmaxf(fabsf(v[q].z), fabsf(v[q].w))));
            }
            most = row_max<LANES>(most, slots[turn + 1]);
            const float scale = fmaxf(most * rstd / kLargestE4m3, kLeastScale);        // (the least where an infinite sum made rstd 0)
            if (cut.lane == 0) a.scale[h.at] = scale;
            const bool small = !(scale > kLeastScale && most > 1e-30f);                // 448 / most might be infinite
            const float one = small ? rstd : kLargestE4m3 / most, other = small ? 1.0f / scale : 1.0f;
#pragma unroll
            for (int q = 0; q < PIECES; ++q) v[q] = v[q] * one * other;
            if (a.stream) store_row_e4m3<true>(v, a.y, h.at * a.y_stride, cut, a.width);
            else store_row_e4m3<false>(v, a.y, h.at * a.y_stride, cut, a.width);
        } else {
#pragma unroll
            for (int q = 0; q < PIECES; ++q) v[q] = v[q] * rstd * w[q];
            if (a.stream) store_row<true>(v, a.y, a.y_type, h.at * a.y_stride, cut, a.width);
            else store_row(v, a.y, a.y_type, h.at * a.y_stride, cut, a.width);
        }
        turn ^= 2;
    };
    walk_through<kNormAhead<LANES>, Rows>(more, fetch, work);
}

// With h = s rstd, g = grad_y w: grad_x = rstd (g - h mean(g h)) + grad_sum, grad_weight = sum of grad_y h.  Bound by HBM:
// 163840 of 327680 rows of 512 in bf16 with all of it 164 us (5.1 TB/s) and 4.7 for the joining launch; 42517 rows of 1000,
// f32 and f16, 84 us (5.1 TB/s).
// As the layer norm's: a workgroup stays for the sake of its sums, its teams take short runs of rows a lap apart.
// INPUTS: the input's gradient is wanted.  STREAMED: something comes along the residual stream.
template <int LANES, int PIECES, int X_BYTES, int G_BYTES, bool INPUTS, bool STREAMED>
__global__ __launch_bounds__(threads_of(LANES), grad_wavefronts(PIECES)) void tabx_rms_grad_kernel(const RmsArgs a)
{
    constexpr int THREADS = threads_of(LANES);
    constexpr int WAVES = THREADS / 64;
    __shared__ float slots[2][WAVES];
    __shared__ f32x4 meet[LANES <= 64 ? WAVES : 1][LANES <= 64 ? LANES : 1];
    const Cut<LANES, PIECES> cut(a.width);
    const f32x4 zero = {0.0f, 0.0f, 0.0f, 0.0f};
    Walk<LANES> walk(a);
    f32x4 w[INPUTS ? PIECES : 1], dw[PIECES];
    if constexpr (INPUTS) load_columns(w, a.weight, 1.0f, cut, a.width);
#pragma unroll
    for (int q = 0; q < PIECES; ++q) dw[q] = zero;
    const bool sums = !INPUTS || a.partial || a.grad_weight;
    int here = 0;                                  // keeps a row's rstd from being moved to a scalar register, and waited for
    asm("v_mov_b32 %0, 0" : "=v"(here));
    int turn = 0;
    struct Rows {
        RawRow<X_BYTES, PIECES> x;
        RawRow<G_BYTES, PIECES> g;
        RawRow<STREAMED ? X_BYTES : 2, STREAMED ? PIECES : 1> s;
        float   rstd;
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
        h.rstd = (a.rstd + h.r)[here];
        load_raw(h.x, a.x, h.r * a.x_stride, cut, a.width);
        load_raw(h.g, a.grad_y, h.r * a.g_stride, cut, a.width);
        if constexpr (STREAMED) load_raw(h.s, a.grad_sum, h.r * a.grad_sum_stride, cut, a.width);
    };
    const auto work = [&](const Rows &h) {
        f32x4 x[PIECES], g[PIECES];
        unpack(x, h.x, a.x_type);
        unpack(g, h.g, a.g_type);
#pragma unroll
        for (int q = 0; q < PIECES; ++q) x[q] *= h.rstd;
        const f32x4 last = cut.counted(g[PIECES - 1]);
        if (sums && (LANES >= 64 || h.own)) {
#pragma unroll
            for (int q = 0; q < PIECES; ++q) dw[q] = fma4(q < PIECES - 1 ? g[q] : last, x[q], dw[q]);
        }
        if constexpr (INPUTS) {
            f32x4 along = last * w[PIECES - 1] * x[PIECES - 1];
#pragma unroll
            for (int q = 0; q < PIECES; ++q) {
                g[q] *= w[q];
                if (q < PIECES - 1) along = fma4(g[q], x[q], along);
            }
            if constexpr (STREAMED && LANES > 64) {    // (grad_x may lie where grad_sum does, and several wavefronts read a
#pragma unroll                                         // row's last elements: all of them have theirs before the first store)
                for (int q = 0; q < PIECES; ++q) asm volatile("" ::"v"(h.s.v[q]) : "memory");
            }
            const float sh = row_sum<LANES>(sum_of(along), slots[turn]) * a.inv_width;
            turn ^= 1;
#pragma unroll
            for (int q = 0; q < PIECES; ++q) g[q] = fma4(x[q], f32x4{-sh, -sh, -sh, -sh}, g[q]) * h.rstd;
            if constexpr (STREAMED) {
                unpack(x, h.s, a.x_type);
#pragma unroll
                for (int q = 0; q < PIECES; ++q) g[q] += x[q];
            }
            store_row(g, a.y, a.y_type, h.r * a.y_stride, cut, a.width);
        }
    };
    walk_through<kGradAhead<LANES>, Rows>(more, fetch, work);
    if (!sums) return;
    // the rows worked on side by side in a wavefront, then the wavefronts
    float *const out = a.partial ? a.partial + (int64_t)blockIdx.x * a.width : a.grad_weight;
#pragma unroll
    for (int q = 0; q < PIECES; ++q) {
        f32x4 v = dw[q];
        if (LANES <= 64) {
#pragma unroll
            for (int d = LANES; d < 64; d *= 2) {
                v.x += __shfl_xor(v.x, d);
                v.y += __shfl_xor(v.y, d);
                v.z += __shfl_xor(v.z, d);
                v.w += __shfl_xor(v.w, d);
            }
            __syncthreads();                       // the piece before has been read
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

} // namespace tabx
