// Linear attention with a decay for each head: one tick of it, and many ticks at once.
//
// With e = exp(log_decay), of one row and head
//   S_t = e S_{t-1} + k_t v_t^T (from zero where tick t is the first of an episode),  out_t = scale q_t S_t.
// Many ticks are taken in chunks of C.  Of a chunk's ticks i, j = 0 .. C-1, with S the state before it,
//   out_i = scale (e^(i+1) q_i S [no episode has begun up to i] + sum over j <= i of the same episode of e^(i-j) (q_i k_j) v_j),
//   S'    = e^C S [none has begun] + sum over the j of the last episode of e^(C-1-j) k_j v_j^T:
// four products of matrices a chunk, in the matrix cores.  All gradients have the same form: grad_q is the attention of
// queries grad_out, keys v and values k, with S transposed; and backwards in time, where D, the gradient of the state,
// takes its part, grad_k that of queries v, keys grad_out and values q, and grad_v that of queries k, keys q and values
// grad_out.  Backwards, e has been applied to D before a chunk's last tick reads it, so the powers are e^i there and
// e^(C-j) in D'; and an episode begins behind the tick where, forwards, the next one does.
#pragma once
#include <type_traits>

#include "tabx_rows.h"

#pragma clang fp contract(off)

namespace tabx {

typedef float f32x16 __attribute__((ext_vector_type(16)));

struct Strides {
    int64_t tick, row, head;
};

struct AttentionArgs {
    const void *q, *k, *v;
    void       *out;
    Strides     qs, ks, vs, os;
    const float *log_decay;
    const uint8_t *fresh;          // [ticks][rows / units], or nullptr
    const uint8_t *controlled;     // [rows], or nullptr
    const float *state_in;         // or nullptr: zero
    float      *state_out;         // or nullptr
    float      *carried;           // [row and head][segment][keys][values]: states before each segment, or nullptr
    float      *kept;              // [row and head][segment]: what a segment leaves of the state before it; -1: an episode begins in it
    int64_t     ticks, rows, envs, works;   // works: rows x heads x segments
    int64_t     segment;           // ticks of a segment, a multiple of the chunk
    int32_t     segments, heads, units, keys, values;
    int32_t     backward;          // in time
    int32_t     exactly;           // the scale is beyond kMostScale
    float       scale_read, scale_added;   // of what is read, of what is taken in
};

// What a launch works on: one attention, or two of the same sizes side by side (blockIdx.y).
struct AttentionPair {
    AttentionArgs of[2];
};

// The way back: all that the three attentions of the gradients need.
struct AttentionGradArgs {
    const void *q, *k, *v, *grad_out;
    void       *grad_q, *grad_k, *grad_v;  // each may be nullptr
    Strides     qs, ks, vs, os, gqs, gks, gvs;
    const float *log_decay;
    const uint8_t *fresh, *controlled;
    const float *state_in, *grad_state_out;
    float      *grad_state_in;     // or nullptr
    const float *states, *grad_states;     // before each segment, forwards and backwards in time, or nullptr
    int64_t     ticks, rows, envs, works, segment;
    int32_t     segments, heads, units, keys, values;
    int32_t     exactly;           // the scale is beyond kMostScale
    float       scale;
};

// exp(log_decay) and its powers as powers of two.
__device__ __forceinline__ float log2_decay(const float *log_decay, int h)
{
    const float g = log_decay[h];
    return (g < 0.0f ? g : 0.0f) * 1.4426950408889634f;    // (NaN too is none)
}
__device__ __forceinline__ float decayed(float l2, int64_t ticks) { return ticks <= 0 ? 1.0f : __builtin_exp2f(l2 * (float)ticks); }

template <int TYPE>
__device__ __forceinline__ float element(const void *data, int64_t at)
{
    return (float)((const typename Element<TYPE>::one *)data)[at];
}

// --- one tick -----------------------------------------------------------------------------------

struct StepArgs {
    const void *q, *k, *v;
    void       *out;
    Strides     qs, ks, vs, os;
    const float *log_decay;
    const uint8_t *fresh, *controlled;
    float      *state;
    int64_t     works;             // rows x heads
    int32_t     heads, units, keys, values;
    float       scale;
};

// A state is a run of keys x values floats.  LANES lanes have a row's head (64: a whole wavefront); lane l has four
// consecutive values of every (4 LANES / VALUES)-th line of the state, so that the lanes read and write 16 bytes each of
// one run.  Bound by HBM: the state is read (also where it is forgotten) and written, once each; 1310720 heads of 32 x 32
// 2.12 ms, 5.1 TB/s; 160000 of 80 x 48 964 us; 96 rows of 4 heads 4.5 us, with the launch 10.8.  Eight lines under way in
// a lane at a time.  VALUES: the values, a multiple of four, rounded up to a power of two; lanes beyond the last value idle.
template <int TYPE, int VALUES, int LANES>
__global__ __launch_bounds__(256) void tabx_attention_step_kernel(const StepArgs a)
{
    typedef typename Element<TYPE>::one T;
    typedef f32x4 Anywhere __attribute__((aligned(4)));
    constexpr int ACROSS = VALUES / 4, LINES = LANES / ACROSS, WORKS = 256 / LANES, AT_ONCE = 8;
    const int lane = (int)threadIdx.x % LANES, d = 4 * (lane % ACROSS), line = lane / ACROSS;
    for (int64_t w = (int64_t)blockIdx.x * WORKS + threadIdx.x / LANES; w < a.works; w += (int64_t)gridDim.x * WORKS) {
        const int64_t r = (uint32_t)w / (uint32_t)a.heads;     // (rows x heads has 31 bits)
        const int h = (int)((uint32_t)w % (uint32_t)a.heads);
        if (a.controlled && a.controlled[r] == 0) continue;
        const bool forget = a.fresh && a.fresh[(uint32_t)r / (uint32_t)a.units] != 0;
        const float e = decayed(log2_decay(a.log_decay, h), 1);
        const int count = a.values - d;            // of this lane's four values
        const T *const q = (const T *)a.q + r * a.qs.row + h * a.qs.head, *const k = (const T *)a.k + r * a.ks.row + h * a.ks.head,
                *const v = (const T *)a.v + r * a.vs.row + h * a.vs.head + d;
        float *const state = a.state + w * a.keys * a.values + d;
        f32x4 value = {0.0f, 0.0f, 0.0f, 0.0f}, sum = {0.0f, 0.0f, 0.0f, 0.0f};
        if (count > 0) value = load_four<TYPE>(v);
        for (int i = line; i < a.keys; i += LINES * AT_ONCE) {
            f32x4 s[AT_ONCE];
            float x[AT_ONCE], y[AT_ONCE];
#pragma unroll
            for (int n = 0; n < AT_ONCE; ++n) {
                const int key = min(i + n * LINES, a.keys - 1);
                if (count > 0) s[n] = *(const Anywhere *)(state + key * a.values);
                x[n] = (float)k[key], y[n] = (float)q[key];
            }
#pragma unroll
            for (int n = 0; n < AT_ONCE; ++n) {
                if (i + n * LINES >= a.keys || count <= 0) continue;
                const f32x4 old = forget ? f32x4{0.0f, 0.0f, 0.0f, 0.0f} : s[n] * e;
                const f32x4 now = {fmaf(x[n], value.x, old.x), fmaf(x[n], value.y, old.y), fmaf(x[n], value.z, old.z), fmaf(x[n], value.w, old.w)};
                *(Anywhere *)(state + (i + n * LINES) * a.values) = now;
                sum = f32x4{fmaf(y[n], now.x, sum.x), fmaf(y[n], now.y, sum.y), fmaf(y[n], now.z, sum.z), fmaf(y[n], now.w, sum.w)};
            }
        }
#pragma unroll
        for (int n = ACROSS; n < LANES; n *= 2)
#pragma unroll
            for (int m = 0; m < 4; ++m) sum[m] += __shfl_xor(sum[m], n);
        if (line == 0 && count > 0) {
            T *const out = (T *)a.out + r * a.os.row + h * a.os.head + d;
            sum *= a.scale;
            store_four<TYPE>(out, sum);
        }
    }
}

// The same for values that are no multiple of four: a wavefront has a row's head, a lane one value (or two) of every
// (64 / ACROSS)-th line, so that no lane's run goes beyond its line (160000 heads of 33 x 31 in f32 282 us; 527 with runs of
// four that are asked for their ends).
template <int TYPE, int ACROSS>
__global__ __launch_bounds__(256) void tabx_attention_step_odd_kernel(const StepArgs a)
{
    typedef typename Element<TYPE>::one T;
    constexpr int LINES = 64 / ACROSS, AT_ONCE = 8;
    const int lane = (int)threadIdx.x & 63, line = lane / ACROSS;
    for (int64_t w = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); w < a.works; w += (int64_t)gridDim.x * 4) {
        const int64_t r = (uint32_t)w / (uint32_t)a.heads;
        const int h = (int)((uint32_t)w % (uint32_t)a.heads);
        if (a.controlled && a.controlled[r] == 0) continue;
        const bool forget = a.fresh && a.fresh[(uint32_t)r / (uint32_t)a.units] != 0;
        const float e = decayed(log2_decay(a.log_decay, h), 1);
        const T *const q = (const T *)a.q + r * a.qs.row + h * a.qs.head, *const k = (const T *)a.k + r * a.ks.row + h * a.ks.head,
                *const v = (const T *)a.v + r * a.vs.row + h * a.vs.head;
        for (int d = lane % ACROSS; d < a.values; d += ACROSS) {
            float *const state = a.state + w * a.keys * a.values + d;
            const float value = (float)v[d];
            float sum = 0.0f;
            for (int i = line; i < a.keys; i += LINES * AT_ONCE) {
                float s[AT_ONCE], x[AT_ONCE], y[AT_ONCE];
#pragma unroll
                for (int n = 0; n < AT_ONCE; ++n) {
                    const int key = min(i + n * LINES, a.keys - 1);
                    s[n] = state[key * a.values], x[n] = (float)k[key], y[n] = (float)q[key];
                }
#pragma unroll
                for (int n = 0; n < AT_ONCE; ++n) {
                    if (i + n * LINES >= a.keys) continue;
                    const float now = fmaf(x[n], value, forget ? 0.0f : e * s[n]);
                    state[(i + n * LINES) * a.values] = now;
                    sum = fmaf(y[n], now, sum);
                }
            }
#pragma unroll
            for (int n = ACROSS; n < 64; n *= 2) sum += __shfl_xor(sum, n);
            if (line == 0) ((T *)a.out)[r * a.os.row + h * a.os.head + d] = (T)(sum * a.scale);
        }
    }
}

// --- many ticks ---------------------------------------------------------------------------------

// The products run in the matrix cores in bf16 with sums in 32 bits, where every 32-bit operand stands as the sum of parts
// of 8 bits each: bf16 inputs are one part, f16 ones two (both exact), f32 ones three; what goes into the state, which is kept
// in 32 bits, is cut into three.  So is what lies between on the way to an output (the products of queries and keys, the
// state that is read) for f16 and f32, and of the parts' products those are left out that are below 2^-24 of a term.  For
// bf16 it is cut into two, which round it to 16 bits: 2^-17 of a term, where the output's own rounding is 2^-8 of the result.
// (A third one there: 128 ticks of 20480 heads of 64 502 us instead of 476, 64 ticks of 20480 heads of 96 844 instead of 622,
// gradients of 64 ticks of 20480 heads of 64 719, in chunks of 32, instead of 639, of 5120 heads of 128 860 instead of 750.  For f16, whose
// rounding is 2^-11, two and without the product of two second parts: 128 ticks of 20480 heads of 64 519 instead of 570.)
template <int TYPE> struct Parts {
    static constexpr int in = TYPE == TABX_BF16 ? 1 : TYPE == TABX_F16 ? 2 : 3;
    static constexpr int mid = TYPE == TABX_BF16 ? 2 : 3;
};

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// Ticks of a chunk.  The state costs as many products a chunk, whatever its length; the ticks among themselves as many as they
// are long, and longer ones more room.  With 64 and 32 of them, one part each (bf16):
//   gradients, 64 ticks of 20480 heads of 64, 643 and 685 us; 64 ticks of 5120 heads of 128, 746 and 859;
//     128 ticks of 40960 heads of 32, 1409 and 1016;
//   forward, 128 ticks of 20480 heads of 64, 493 and 475; 64 ticks of 20480 heads of 96, 627 and 654; 32768 ticks of 8
//     heads of 128, 156 and 175; 128 ticks of 81920 heads of 32, 1005 and 908;
//   segments' states, 8192 ticks of 16 heads of 64, 49.8 and 50.4 with the attention behind them.
// Operands in several parts have no room for 64.  READS_ONCE: forward.
constexpr int long_chunk(int d, int type, bool reads_once) { return type == TABX_BF16 && d > (reads_once ? 64 : 32) ? 64 : 32; }

template <int N>
__device__ __forceinline__ void split(bf16x4 (&part)[N], f32x4 v)
{
#pragma unroll
    for (int p = 0; p < N; ++p) {
        part[p] = __builtin_convertvector(v, bf16x4);
        if (p + 1 < N) v -= __builtin_convertvector(part[p], f32x4);
    }
}

__device__ __forceinline__ bf16x8 join(bf16x4 a, bf16x4 b) { return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7); }

// One product of operands in parts, the smallest parts' first: those of three parts whose places in their operands add up to
// less than three, all of two.
template <int NA, int NB>
__device__ __forceinline__ f32x4 multiply(const bf16x8 (&a)[NA], const bf16x8 (&b)[NB], f32x4 c)
{
    constexpr int last = NA + NB - 1 < 3 ? NA + NB - 1 : 3;
#pragma unroll
    for (int s = last - 1; s >= 0; --s)
#pragma unroll
        for (int i = 0; i < NA; ++i)
            if (s - i >= 0 && s - i < NB) c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[i], b[s - i], c, 0, 0, 0);
    return c;
}

// Eight elements of a row as they lie in memory.
template <int TYPE>
struct Eight {
    typedef typename Element<TYPE>::one T;
    typedef u32x4 Anywhere __attribute__((aligned(2)));
    static constexpr int PIECES = TYPE == TABX_F32 ? 2 : 1;
    u32x4 v[PIECES];

    __device__ __forceinline__ void load(const T *from)
    {
#pragma unroll
        for (int n = 0; n < PIECES; ++n) v[n] = ((const Anywhere *)from)[n];
    }
    // Those below `count`, and zeros.
    __device__ __forceinline__ void load_some(const T *from, int count)
    {
#pragma unroll
        for (int n = 0; n < PIECES; ++n) v[n] = u32x4{0, 0, 0, 0};
        if (count >= 8) {
            load(from);
        } else if (count > 0) {                    // a width that is no multiple of eight: the last element for those behind it
#pragma unroll
            for (int i = 0; i < 7; ++i) {
                const int at = min(i, count - 1);
                if constexpr (TYPE == TABX_F32) v[i / 4][i % 4] = i < count ? ((const uint32_t *)from)[at] : 0;
                else v[0][i / 2] |= i < count ? (uint32_t)((const uint16_t *)from)[at] << 16 * (i % 2) : 0;
            }
        }
    }
};

// Up to where products of matrices take the place of the recurrence's own order, in which less may pass 32 bits: q, k and v below
// 2^30, a scale of at most 2^16, a state below 2^70 before the first of 64 chunks (kSmallChunks).  Then with keys and values of
// 2^7 at most and chunks of 2^6 ticks
//   |q k scale| < 2^(7 + 30 + 30 + 16),  sum over keys' ticks |q k scale v| < 2^(83 + 6 + 30) = 2^119,
//   |S| < 2^70 + 2^(12 + 30 + 30 + 16) < 2^89 (scaled as it is taken in; else the 16 stand at its reading),  |q S scale| < 2^126,
// and every part, every sum in any order is finite.  What lies beyond goes through the chunk tick by tick.
// (To look costs 1 % of the time: 128 ticks of 20480 heads of 64 474 us, 477; gradients of 64 ticks of them 636, 646.)
constexpr float kMostScale = 0x1p16f, kLargeState = 0x1p70f;
constexpr int kSmallChunks = 64;

// Not 0 in a bit of its own if one of them is 2^30 or more (an exponent of at least that many carries) or not finite; values
// of f16 end below that.
template <int TYPE>
__device__ __forceinline__ uint32_t beyond(const Eight<TYPE> &e)
{
    constexpr uint32_t exponent = TYPE == TABX_F32 ? 0x7f800000u : TYPE == TABX_BF16 ? 0x7f807f80u : 0x7c007c00u;
    constexpr uint32_t rest = TYPE == TABX_F32 ? 0x31800000u : TYPE == TABX_BF16 ? 0x31803180u : 0x04000400u;
    uint32_t found = 0;
#pragma unroll
    for (int n = 0; n < (TYPE == TABX_F32 ? 2 : 1); ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) found |= (e.v[n][i] & exponent) + rest;
    return found & (TYPE == TABX_F32 ? 0x80000000u : 0x80008000u);
}

// All of a workgroup's wavefronts, and what they have written to LDS.  (__syncthreads would wait for loads that are under way
// and for stores to memory, which nothing here reads.)
__device__ __forceinline__ void lds_meet()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// A chunk's rows of one array in LDS, a tile for each part.  Rows lie D + 8 elements apart: eight of them, of 16 bytes
// each, or four of 32, meet all banks once.
template <int D, int C, int PARTS>
struct Tile {
    static constexpr int kRow = D + 8, kPart = C * kRow;
    __bf16 at[PARTS * kPart];

    template <int TYPE>
    __device__ __forceinline__ void put(int row, int d, const Eight<TYPE> &e)
    {
        if constexpr (TYPE == TABX_BF16) {
            *(u32x4 *)&at[row * kRow + d] = e.v[0];
        } else {
            f32x4 v[2];
            if constexpr (TYPE == TABX_F32) {
                __builtin_memcpy(&v, &e.v, sizeof v);
            } else {
                f16x4 h[2];
                __builtin_memcpy(&h, &e.v, sizeof h);
                v[0] = __builtin_convertvector(h[0], f32x4), v[1] = __builtin_convertvector(h[1], f32x4);
            }
            bf16x4 a[PARTS], b[PARTS];
            split(a, v[0]);
            split(b, v[1]);
#pragma unroll
            for (int p = 0; p < PARTS; ++p) *(bf16x8 *)&at[p * kPart + row * kRow + d] = join(a[p], b[p]);
        }
    }
    // An operand of a product over the elements of rows: row `row + col` of 16, elements from + 8 quad .. + 7.
    __device__ __forceinline__ void along(bf16x8 (&x)[PARTS], int row, int from, int col, int quad) const
    {
#pragma unroll
        for (int p = 0; p < PARTS; ++p) x[p] = *(const bf16x8 *)&at[p * kPart + (row + col) * kRow + from + 8 * quad];
    }
    // The same in the order in which a product leaves its results: elements from + 4 quad .. + 3 and those 16 on.
    __device__ __forceinline__ void along_results(bf16x8 (&x)[PARTS], int row, int from, int col, int quad) const
    {
#pragma unroll
        for (int p = 0; p < PARTS; ++p) {
            const __bf16 *const e = &at[p * kPart + (row + col) * kRow + from + 4 * quad];
            x[p] = join(*(const bf16x4 *)e, *(const bf16x4 *)(e + 16));
        }
    }
    // An operand of a product over rows: element `from + col` of rows row + 4 quad .. + 3 and those 16 on.  Sixteen
    // lanes read four rows' sixteen elements and change them round.
    __device__ __forceinline__ void across(bf16x8 (&x)[PARTS], int row, int from, int col, int quad) const
    {
        typedef s16x4 __attribute__((address_space(3))) *Lds;
#pragma unroll
        for (int p = 0; p < PARTS; ++p) {
            const __bf16 *const e = &at[p * kPart + (row + 4 * quad + col / 4) * kRow + from + 4 * (col % 4)];
            const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)e), b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(e + 16 * kRow));
            x[p] = join(__builtin_bit_cast(bf16x4, a), __builtin_bit_cast(bf16x4, b));
        }
    }
};

// One row's head of an attention: its arrays from there on, strides of ticks, widths.
struct Part {
    const void *q, *k, *v;
    void       *out;               // or nullptr
    int64_t     q_tick, k_tick, v_tick, out_tick;
    int         keys, values, backward, exactly;
    float       scale_read, scale_added;
};

// The ticks that an attention goes through, in the direction of time taken, and where episodes begin in it.
struct Course {
    const uint8_t *fresh;          // of the row's env, or nullptr
    int64_t envs, ticks, begin;    // begin: of the chunk at hand
    int     backward;
    __device__ __forceinline__ int64_t tick(int i) const { return backward ? ticks - 1 - (begin + i) : begin + i; }
    // Backwards, an episode begins behind the tick where, forwards, the next one does.
    __device__ __forceinline__ int begins(int i, int n) const
    {
        if (!fresh || i >= n) return 0;
        const int64_t t = begin + i;
        if (!backward) return fresh[t * envs];
        return t > 0 ? fresh[(ticks - t) * envs] : 0;
    }
};

template <typename T>
__device__ __forceinline__ T *moved_on(T *data, int64_t elements, int bytes)
{
    typedef std::conditional_t<std::is_const_v<T>, const char, char> Byte;
    return (T *)((Byte *)data + elements * bytes);
}

template <int D, int TYPE, int C>
struct Attention {
    static constexpr int IN = Parts<TYPE>::in, MID = Parts<TYPE>::mid;
    static constexpr bool kAhead = D < 96 || TYPE == TABX_F32;
    static constexpr int WAVES = D / 16, THREADS = 64 * WAVES, PASSES = C * D / 8 / THREADS, TILES = D / 16;
    typedef typename Element<TYPE>::one T;
    typedef Tile<D, C, IN> In;
    // Products of queries and keys: rows of the first 32 queries have the first 32 keys only.
    static constexpr int kNear = 32 + 8, kFar = 64 + 8;
    typedef __bf16 Within[MID][C == 64 ? 32 * kNear + 32 * kFar : 32 * kNear];
    static __device__ __forceinline__ int within_row(int I, int col)
    {
        return I < 2 ? (16 * I + col) * kNear : 32 * kNear + (16 * (I - 2) + col) * kFar;
    }

    // A wavefront has 16 of the values and all of the state's lines of them, in the layout in which a product leaves its
    // result (a lane has four lines of one column), which is that of an operand of the next one (`along_results`).
    typedef f32x4 State[TILES];

    struct Rows {
        Eight<TYPE> e[PASSES];
        // Waits for them here: later, stores that have been issued meanwhile would be waited for too.
        __device__ __forceinline__ void arrive()
        {
#pragma unroll
            for (int p = 0; p < PASSES; ++p)
#pragma unroll
                for (int n = 0; n < Eight<TYPE>::PIECES; ++n) asm volatile("" : "+v"(e[p].v[n]));
        }
    };

    static __device__ __forceinline__ void load(Rows &rows, const void *data, int64_t tick, const Course &c, int n, int width)
    {
        constexpr int across = D / 8;
        const int d = 8 * ((int)threadIdx.x % across), row = (int)threadIdx.x / across;
        asm volatile("" : "+s"(tick));             // (what follows from it is not kept)
        const int64_t step = c.backward ? -tick : tick;
        const T *const from = (const T *)data + c.tick(0) * tick + row * step + d;
        if (n == C && width == D) {                // (the same for all: no lane has to be asked)
#pragma unroll
            for (int p = 0; p < PASSES; ++p) rows.e[p].load(from + p * (THREADS / across) * step);
        } else {
#pragma unroll
            for (int p = 0; p < PASSES; ++p) {
                const int i = p * (THREADS / across) + row;
                rows.e[p].load_some(from + p * (THREADS / across) * step, i < n ? width - d : 0);
            }
        }
    }
    static __device__ __forceinline__ uint32_t store(In &tile, const Rows &rows)
    {
        constexpr int across = D / 8;
        uint32_t found = 0;
#pragma unroll
        for (int p = 0; p < PASSES; ++p) {
            tile.template put<TYPE>(p * (THREADS / across) + (int)threadIdx.x / across, 8 * ((int)threadIdx.x % across), rows.e[p]);
            found |= beyond<TYPE>(rows.e[p]);
        }
        return found;
    }

    // Products of queries and keys, faded by the ticks between them, 0 where they do not belong together, in parts:
    // tiles of 16 x 16 on and below the diagonal, dealt to the wavefronts.  Rows are queries; along them the keys lie in the
    // order of `along_results`, so that a lane's eight are next to each other.
    static __device__ __forceinline__ void compare(Within &within, const In &q, const In &k, uint64_t begins, float l2, float scale, int wave, int col,
                                                   int quad)
    {
        const Powers power(l2);
        constexpr int tiles = C / 16 * (C / 16 + 1) / 2;
        for (int tile = wave; tile < tiles; tile += WAVES) {
            const int I = tile < 1 ? 0 : tile < 3 ? 1 : tile < 6 ? 2 : 3, J = tile - I * (I + 1) / 2;
            f32x4 p = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int s = 0; s < D / 32; ++s) {
                bf16x8 x[IN], y[IN];
                k.along(x, 16 * J, 32 * s, col, quad);
                q.along(y, 16 * I, 32 * s, col, quad);
                p = multiply(x, y, p);
            }
            const int i = 16 * I + col, first = 16 * J + 4 * quad;
            if (I > J) {
                const float fade = __builtin_amdgcn_exp2f(l2 * (float)(i - first - 3)) * scale;
#pragma unroll
                for (int r = 0; r < 4; ++r) p[r] *= fade * power.of[3 - r];
            } else {
#pragma unroll
                for (int r = 0; r < 4; ++r) p[r] = first + r <= i ? p[r] * (__builtin_amdgcn_exp2f(l2 * (float)(i - first - r)) * scale) : 0.0f;
            }
            if (begins) {                          // (the same for all)
                const uint64_t up = begins & ((2ull << i) - 1);        // episodes begun up to the query's tick
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (first + r <= i && (up >> (first + r)) > 1) p[r] = 0.0f;        // one of them behind the key's
            }
            bf16x4 part[MID];
            split(part, p);
            const int at = within_row(I, col) + 32 * (J / 2) + 8 * quad + 4 * (J % 2);
#pragma unroll
            for (int m = 0; m < MID; ++m) {
                *(bf16x4 *)&within[m][at] = part[m];
                if (I == J && I % 2 == 0) *(u32x2 *)&within[m][at + 4] = u32x2{0, 0};
            }
        }
    }

    // What a chunk's queries read, and the state behind the chunk.
    template <bool READS, typename Arrived>
    static __device__ __forceinline__ void advance(State &state, const Within &within, const In &q, const In &k, const In &v,
                                                   uint64_t begins, int n, float l2, const Part &a, const Course &c, int wave, int col,
                                                   int quad, Arrived arrived)
    {
        bf16x8 values[C / 32][IN];                 // this lane's: 8 ticks of its column, of every 32
#pragma unroll
        for (int b = 0; b < C / 32; ++b) v.across(values[b], 32 * b, 16 * wave, col, quad);
        if constexpr (READS) {
            // the state as operands, all of it at a time, or (IN_TURN: it would not fit the registers) 32 lines after the other
            constexpr bool IN_TURN = D >= 96 && MID == 3 && IN == 2;
            bf16x8 held[IN_TURN ? 1 : D / 32][MID];
            f32x4 read[IN_TURN ? C / 16 : 1];
            const auto hold = [&](bf16x8(&operand)[MID], int s) {
                bf16x4 x[MID], y[MID];
                split(x, state[2 * s]);
                split(y, state[2 * s + 1]);
#pragma unroll
                for (int m = 0; m < MID; ++m) operand[m] = join(x[m], y[m]);
            };
            if constexpr (IN_TURN) {
#pragma unroll
                for (int I = 0; I < C / 16; ++I) read[I] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int s = 0; s < D / 32; ++s) {
                    __builtin_amdgcn_sched_barrier(0);
                    hold(held[0], s);
#pragma unroll
                    for (int I = 0; I < C / 16; ++I) {
                        if (16 * I >= n) continue;
                        bf16x8 x[IN];
                        q.along_results(x, 16 * I, 32 * s, col, quad);
                        read[I] = multiply(held[0], x, read[I]);
                    }
                }
            } else {
#pragma unroll
                for (int s = 0; s < D / 32; ++s) hold(held[s], s);
            }
            const int d = 16 * wave + 4 * quad;
            int64_t tick = a.out_tick;
            asm volatile("" : "+s"(tick));
            const int64_t step = c.backward ? -tick : tick;
            T *const out = (T *)a.out + c.tick(0) * tick + col * step + d;
#pragma unroll
            for (int I = 0; I < C / 16; ++I) {
                if (16 * I >= n) continue;
                __builtin_amdgcn_sched_barrier(0); // (operands of all of them at a time would not fit)
                const int i = 16 * I + col;
                f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
                if constexpr (IN_TURN) {
                    o = read[I];
                } else {
#pragma unroll
                    for (int s = 0; s < D / 32; ++s) {
                        bf16x8 x[IN];
                        q.along_results(x, 16 * I, 32 * s, col, quad);
                        o = multiply(held[s], x, o);
                    }
                }
                const float fade = __builtin_amdgcn_exp2f(l2 * (float)(i + 1 - a.backward)) * a.scale_read;
                o *= fade;
                if (begins) {
                    const bool none = (begins & ((2ull << i) - 1)) != 0;
#pragma unroll
                    for (int r = 0; r < 4; ++r) o[r] = none ? 0.0f : o[r];
                }
#pragma unroll
                for (int b = 0; b <= I / 2; ++b) {
                    bf16x8 x[MID];
#pragma unroll
                    for (int m = 0; m < MID; ++m) x[m] = *(const bf16x8 *)&within[m][within_row(I, col) + 32 * b + 8 * quad];
                    o = multiply(values[b], x, o);
                }
                if (I == 0) arrived();
                if (a.out && i < n && d < a.values) {
                    T *const to = out + 16 * I * step;
                    if (d + 4 <= a.values) {
                        store_four<TYPE>(to, o);
                    } else {
#pragma unroll
                        for (int r = 0; r < 3; ++r)
                            if (d + r < a.values) to[r] = (T)o[r];
                    }
                }
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        // the values faded by the ticks behind theirs, in as many parts as the state has digits; those of episodes that have
        // ended count no more
        const int newest = begins ? 63 - __builtin_clzll(begins) : 0;
        const float left = __builtin_amdgcn_exp2f(l2 * (float)n);
        const Powers power(l2);
#pragma unroll
        for (int s = 0; s < TILES; ++s) {
            if (begins) state[s] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
            else state[s] *= left;
        }
#pragma unroll
        for (int b = 0; b < C / 32; ++b) {
            if (32 * b >= n) continue;
            bf16x4 part[2][3];
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                f32x4 x;
#pragma unroll
                for (int p = IN - 1; p >= 0; --p) {
                    const bf16x4 y = half ? __builtin_shufflevector(values[b][p], values[b][p], 4, 5, 6, 7)
                                          : __builtin_shufflevector(values[b][p], values[b][p], 0, 1, 2, 3);
                    x = p == IN - 1 ? __builtin_convertvector(y, f32x4) : x + __builtin_convertvector(y, f32x4);
                }
                const int first = 32 * b + 16 * half + 4 * quad;
                if (n == C) {
                    const float fade = __builtin_amdgcn_exp2f(l2 * (float)(C - 4 - first + a.backward)) * a.scale_added;
#pragma unroll
                    for (int r = 0; r < 4; ++r) x[r] *= fade * power.of[3 - r];
                } else {
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        x[r] = first + r < n ? x[r] * (__builtin_amdgcn_exp2f(l2 * (float)(n - 1 - first - r + a.backward)) * a.scale_added) : 0.0f;
                }
                if (begins) {
#pragma unroll
                    for (int r = 0; r < 4; ++r) x[r] = first + r >= newest ? x[r] : 0.0f;
                }
                split(part[half], x);
            }
            bf16x8 faded[3];
#pragma unroll
            for (int m = 0; m < 3; ++m) faded[m] = join(part[0][m], part[1][m]);
#pragma unroll
            for (int s = 0; s < TILES; ++s) {
                bf16x8 y[IN];
                k.across(y, 32 * b, 16 * s, col, quad);
                state[s] = multiply(y, faded, state[s]);
            }
        }
    }

    // The same for a chunk with elements that are not finite, tick by tick: in a product of matrices they would reach ticks that
    // they do not belong to, as zero times them is not zero; and for what may pass 32 bits there and not here (kMostScale).
    template <bool READS>
    static __device__ __forceinline__ void advance_slowly(State &state, uint64_t begins, int n, float l2, const Part &a, const Course &c, int wave, int col, int quad)
    {
        const float e = __builtin_amdgcn_exp2f(l2);
        const int d = 16 * wave + col;
        for (int i = 0; i < n; ++i) {
            const int64_t t = c.tick(i);
            const bool begun = begins >> i & 1;
            const float value = d < a.values ? element<TYPE>(a.v, t * a.v_tick + d) * a.scale_added : 0.0f;
            float sum = 0.0f;
#pragma unroll
            for (int s = 0; s < TILES; ++s) {
                int first = 4 * quad;              // a few loads at a time, their places not worked out beforehand: this
                asm volatile("" : "+v"(first) : : "memory");       // path is to cost no registers
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int key = 16 * s + first + r;
                    float x = begun ? 0.0f : a.backward ? state[s][r] : state[s][r] * e;
                    if (key < a.keys) {
                        x = fmaf(element<TYPE>(a.k, t * a.k_tick + key), value, x);
                        if (READS) sum = fmaf(element<TYPE>(a.q, t * a.q_tick + key), x, sum);
                    }
                    state[s][r] = a.backward ? x * e : x;
                }
            }
            if constexpr (READS) {
                sum += __shfl_xor(sum, 16);
                sum += __shfl_xor(sum, 32);
                if (a.out && quad == 0 && d < a.values)
                    ((T *)a.out)[t * a.out_tick + d] = (T)(sum * a.scale_read);
            }
        }
    }

    // A lane's elements of a state in memory, elements along_keys and along_values apart.  Places are worked out from one
    // that is the same for all, where they are needed.
    static __device__ __forceinline__ void load_state(State &state, const float *from, int keys, int values, int along_keys, int along_values)
    {
        int lane = (int)threadIdx.x;
        asm volatile("" : "+v"(lane));
        const int value = 16 * (lane >> 6) + (lane & 15), first = 4 * (lane >> 4 & 3);
        if (keys == D && values == D) {
            const int at = first * along_keys + value * along_values;
#pragma unroll
            for (int s = 0; s < TILES; ++s)
#pragma unroll
                for (int i = 0; i < 4; ++i) state[s][i] = (from + (16 * s + i) * along_keys)[at];
        } else {
            // beyond the widths, the last element: loads without a branch, which would be waited for one by one
            const int column = min(value, values - 1) * along_values;
#pragma unroll
            for (int s = 0; s < TILES; ++s)
#pragma unroll
                for (int i = 0; i < 4; ++i) state[s][i] = from[min(first + 16 * s + i, keys - 1) * along_keys + column];
#pragma unroll
            for (int s = 0; s < TILES; ++s)
#pragma unroll
                for (int i = 0; i < 4; ++i) state[s][i] = first + 16 * s + i < keys && value < values ? state[s][i] : 0.0f;
        }
    }
    static __device__ __forceinline__ void store_state(const State &state, float *to, int keys, int values, int along_keys, int along_values, bool zero)
    {
        int lane = (int)threadIdx.x;
        asm volatile("" : "+v"(lane));
        const int value = 16 * (lane >> 6) + (lane & 15), first = 4 * (lane >> 4 & 3), at = first * along_keys + value * along_values;
        if (value >= values) return;
#pragma unroll
        for (int s = 0; s < TILES; ++s)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if ((keys == D) || first + 16 * s + i < keys) (to + (16 * s + i) * along_keys)[at] = zero ? 0.0f : state[s][i];
    }
    // Zeros for the ticks from `from` to `to`.
    static __device__ __forceinline__ void clear_rows(void *data, int64_t tick, int64_t from, int64_t to, int width)
    {
        constexpr int across = D / 8;
        const int d = 8 * ((int)threadIdx.x % across);
        for (int64_t t = from + (int)threadIdx.x / across; t < to; t += THREADS / across) {
            T *const at = (T *)data + t * tick + d;
            if (d + 8 <= width) {
                const f32x4 zero = {0.0f, 0.0f, 0.0f, 0.0f};
                store_four<TYPE>(at, zero);
                store_four<TYPE>(at + 4, zero);
            } else {
                for (int i = d; i < width; ++i) at[i - d] = (T)0.0f;
            }
        }
    }
    static __device__ __forceinline__ void clear(State &state)
    {
#pragma unroll
        for (int s = 0; s < TILES; ++s) state[s] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }

    // Whether a lane's part of a state is too large for products of matrices.  (NaN is not: it stays in its element there.)
    static __device__ __forceinline__ bool large(const State &state)
    {
        float most = 0.0f;
#pragma unroll
        for (int s = 0; s < TILES; ++s) most = fmaxf(most, fmaxf(fmaxf(fabsf(state[s].x), fabsf(state[s].y)), fmaxf(fabsf(state[s].z), fabsf(state[s].w))));
        return most >= kLargeState;
    }

    // What the decay leaves in 0 to 3 ticks.
    struct Powers {
        float of[4];
        __device__ __forceinline__ Powers(float l2)
        {
#pragma unroll
            for (int i = 0; i < 4; ++i) of[i] = __builtin_amdgcn_exp2f(l2 * (float)i);
        }
    };

    // One attention from tick `begin` to `last`; the next chunk's rows are under way while it works on the present one (not
    // the wide ones', which have no registers left for them: 128 ticks of 10240 heads of 128 in bf16 1786 us with them, 653
    // without; of 20480 heads of 64, 475 and 483).  READS: queries are answered (else only the state goes on).  part(),
    // course(begin): what to go through, worked out anew where it is needed.  kept: what is left of the state before.  wild, turn: of the chunk at hand and the one
    // before, whether it goes tick by tick.
    template <bool READS, typename GetPart, typename GetCourse>
    static __device__ __forceinline__ void go_through(State &state, float &kept, In &q, In &k, In &v, Within &within, int (&wild)[2], int &turn,
                                                      GetPart part, GetCourse course, int64_t begin, int64_t last, float decay)
    {
        const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
        Rows qr, kr, vr;
        int flag = 0, small = 0;                   // small: chunks for which the state is known to be
        const auto fetch = [&](int64_t from) {
            const Part a = part();
            const Course c = course(from);
            const int n = (int)min((int64_t)C, last - from);
            if constexpr (READS) load(qr, a.q, a.q_tick, c, n, a.keys);
            load(kr, a.k, a.k_tick, c, n, a.keys);
            load(vr, a.v, a.v_tick, c, n, a.values);
            flag = c.begins(lane, n);
        };
        if (kAhead && begin < last) fetch(begin);
        for (; begin < last; begin += C) {
            const int n = (int)min((int64_t)C, last - begin);
            if (!kAhead) fetch(begin);
            // powers and places are worked out for every chunk: kept, they would cost a wavefront
            float l2 = decay;
            int col = lane & 15, quad = lane >> 4;
            asm volatile("" : "+v"(l2), "+v"(col), "+v"(quad));
            turn ^= 1;
            if (threadIdx.x == 0) wild[turn] = part().exactly;
            lds_meet();                                   // the chunk before has been worked on
            uint32_t odd = store(k, kr) | store(v, vr);
            if constexpr (READS) odd |= store(q, qr);
            if (READS && small == 0) odd |= large(state);
            if (__ballot(odd != 0) && lane == 0) wild[turn] = 1;
            const uint64_t begins = __ballot(flag != 0);       // bit i: an episode begins with the chunk's tick i
            if (kAhead && begin + C < last) fetch(begin + C);
            lds_meet();
            if constexpr (READS) {
                const Part a = part();
                compare(within, q, k, begins, l2, a.scale_read * a.scale_added, wave, col, quad);
                lds_meet();
            }
            const Part a = part();
            const Course c = course(begin);
            if (__builtin_expect(wild[turn], 0)) advance_slowly<READS>(state, begins, n, l2, a, c, wave, col, quad);
            else
                advance<READS>(state, within, q, k, v, begins, n, l2, a, c, wave, col, quad, [&] {
                    if (!kAhead) return;
                    if constexpr (READS) qr.arrive();
                    kr.arrive(), vr.arrive();
                    asm volatile("" : "+v"(flag));
                });
            if constexpr (READS) small = __builtin_amdgcn_readfirstlane(wild[turn]) ? 0 : (small == 0 ? kSmallChunks : small) - 1;
            kept = begins || kept < 0.0f ? -1.0f : kept * __builtin_amdgcn_exp2f(l2 * (float)n);
        }
    }
};

__device__ __forceinline__ int64_t uniform(int64_t v)
{
    return (int64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)v) | (int64_t)__builtin_amdgcn_readfirstlane((int)(v >> 32)) << 32;
}

// Workgroups are dealt to the eight XCDs in turn: each takes a run of neighbours, which share lines.
__device__ __forceinline__ int64_t neighbour(int64_t id, int64_t all)
{
    const int64_t run = all / 8, rest = all % 8, x = id % 8;
    return x * run + (x < rest ? x : rest) + id / 8;
}

// What a workgroup works on: a row's head, or a segment of its ticks.
struct Work {
    int64_t at, rh, r, env;        // at: with its segment; rh: row and head
    int     segment, h;
    template <typename Args>
    __device__ __forceinline__ Work(const Args &a, int64_t id) : Work(a, a.works <= gridDim.x ? neighbour(id, a.works) : id, 0)
    {
    }
    template <typename Args>
    __device__ __forceinline__ Work(const Args &a, int64_t which, int)
    {
        at = which;
        // (a division's result is the same for all, but not known to be; rows x heads has 31 bits)
        rh = a.segments == 1 ? at : uniform(at / a.segments);
        segment = (int)(at - rh * a.segments);
        r = __builtin_amdgcn_readfirstlane((int)((uint32_t)rh / (uint32_t)a.heads));
        h = (int)(rh - r * a.heads);
        env = __builtin_amdgcn_readfirstlane((int)((uint32_t)r / (uint32_t)a.units));
    }
    __device__ __forceinline__ int64_t of(const Strides &s) const { return r * s.row + h * s.head; }
};

// Wavefronts of a SIMD, as many as the LDS of a workgroup lets the machine hold.
constexpr int attention_wavefronts(int d, int type) { return d >= 96 ? type == TABX_F32 ? 2 : 4 : 3; }
constexpr int attention_grad_wavefronts(int d, int type) { return d <= 64 ? 3 : type == TABX_F32 ? 2 : 4; }

// The launch arguments, fetched anew for what follows.  A wavefront has too few scalar registers for what all of a kernel
// needs, and what is fetched once at the top is spilled to vector registers (a quarter of the gradients' instructions).
template <typename Args>
__device__ __forceinline__ const Args &again()
{
    typedef const __attribute__((address_space(4))) Args *Late;
    Late p = (Late)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(p));
    return *(const Args *)p;
}

// A workgroup goes through its ticks with the state in registers.  Bound by HBM and by vector instructions next to it, which
// cut operands into parts and fade them: 128 ticks of 20480 heads of 64 in bf16 455 to 475 us, 4.3 TB/s of q, k, v and out
// (vector instructions two thirds of the time, matrix ones an eighth, reads of LDS a quarter); in f16, with its two parts, 556; of
// 10240 heads of 128 653 us (4.1); in f32 128 ticks of 10240 heads of 64 388 (4.3); 8 ticks of 163840 heads of 64 1165 us (the
// states: 5.2).  CARRY: nothing is read, the states that the segments
// would leave of nothing are.
template <int D, int TYPE, int C, bool CARRY>
__global__ __launch_bounds__(4 * D, attention_wavefronts(D, TYPE)) void tabx_attention_kernel(const AttentionPair)
{
    typedef Attention<D, TYPE, C> A;
    const auto mine = []() -> const AttentionArgs & { return again<AttentionPair>().of[blockIdx.y]; };
    __shared__ typename A::In q, k, v;
    __shared__ typename A::Within within;
    __shared__ int wild[2];
    int turn = 0;
    for (int64_t id = blockIdx.x; id < mine().works; id += gridDim.x) {
        const Work w(mine(), id);
        const auto part = [&] {
            const AttentionArgs &a = mine();
            constexpr int bytes = sizeof(typename A::T);
            return Part{moved_on(a.q, w.of(a.qs), bytes), moved_on(a.k, w.of(a.ks), bytes), moved_on(a.v, w.of(a.vs), bytes),
                        a.out ? moved_on(a.out, w.of(a.os), bytes) : nullptr, a.qs.tick, a.ks.tick, a.vs.tick, a.os.tick, a.keys, a.values,
                        a.backward, a.exactly, a.scale_read, a.scale_added};
        };
        const auto course = [&](int64_t begin) {
            const AttentionArgs &a = mine();
            return Course{a.fresh ? a.fresh + w.env : nullptr, a.envs, a.ticks, begin, a.backward};
        };
        typename A::State state;
        float kept = 1.0f, decay;
        int64_t first, last;
        {
            const AttentionArgs &a = mine();
            if (CARRY && w.segment == a.segments - 1) continue;        // (nothing comes behind it)
            if (a.controlled && a.controlled[w.r] == 0) continue;
            decay = fmaxf(log2_decay(a.log_decay, w.h), -1e9f);        // (all at once, and none of no ticks)
            const int64_t size = a.keys * a.values;
            if (!CARRY && a.carried) A::load_state(state, a.carried + w.at * size, a.keys, a.values, a.values, 1);
            else if (!CARRY && a.state_in) A::load_state(state, a.state_in + w.rh * size, a.keys, a.values, a.values, 1);
            else A::clear(state);
            first = w.segment * a.segment, last = min(first + a.segment, a.ticks);
        }
        A::template go_through<!CARRY>(state, kept, q, k, v, within, wild, turn, part, course, first, last, decay);
        const AttentionArgs &a = mine();
        const int64_t size = a.keys * a.values;
        if (CARRY) {
            A::store_state(state, a.carried + w.at * size, a.keys, a.values, a.values, 1, false);
            if (threadIdx.x == 0) a.kept[w.at] = kept;
        } else if (a.state_out && w.segment == a.segments - 1) {
            A::store_state(state, a.state_out + w.rh * size, a.keys, a.values, a.values, 1, false);
        }
    }
}

// The gradients: forwards through the ticks for grad_q, then backwards for grad_k and grad_v, which read the same rows,
// and the state's; the last chunk forwards is the first one backwards, and what was read is still in the caches.  Bound by
// vector instructions (over half of the time) beside HBM: 64 ticks of 20480 heads of 64 in bf16 643 us, 3.4 TB/s of seven arrays.
// The loads of the next chunk do not go ahead here: four arrays of rows would cost a wavefront of a SIMD.
template <int D, int TYPE, int C>
__global__ __launch_bounds__(4 * D, attention_grad_wavefronts(D, TYPE)) void tabx_attention_grad_kernel(const AttentionGradArgs)
{
    typedef Attention<D, TYPE, C> A;
    typedef AttentionGradArgs Args;
    typedef typename A::T T;
    constexpr int bytes = sizeof(T);
    __shared__ typename A::In q, k, v, g;
    __shared__ typename A::Within within;
    __shared__ int wild[2];
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    int turn = 0;
    for (int64_t id = blockIdx.x; id < again<Args>().works; id += gridDim.x) {
        const Work w(again<Args>(), id);
        const auto course = [&](int64_t begin, int backward) {
            const Args &a = again<Args>();
            return Course{a.fresh ? a.fresh + w.env : nullptr, a.envs, a.ticks, begin, backward};
        };
        float decay;
        {
            const Args &a = again<Args>();
            const int64_t first = w.segment * a.segment, last = min(first + a.segment, a.ticks), size = a.keys * a.values;
            if (a.controlled && a.controlled[w.r] == 0) {
                if (a.grad_q) A::clear_rows((T *)a.grad_q + w.of(a.gqs), a.gqs.tick, first, last, a.keys);
                if (a.grad_k) A::clear_rows((T *)a.grad_k + w.of(a.gks), a.gks.tick, first, last, a.keys);
                if (a.grad_v) A::clear_rows((T *)a.grad_v + w.of(a.gvs), a.gvs.tick, first, last, a.values);
                if (a.grad_state_in && w.segment == 0)
                    for (int j = threadIdx.x; j < size; j += A::THREADS) a.grad_state_in[w.rh * size + j] = 0.0f;
                continue;
            }
            decay = fmaxf(log2_decay(a.log_decay, w.h), -1e9f);
            if (a.grad_q) {
                typename A::State state;           // transposed
                if (a.states) A::load_state(state, a.states + w.at * size, a.values, a.keys, 1, a.values);
                else if (a.state_in) A::load_state(state, a.state_in + w.rh * size, a.values, a.keys, 1, a.values);
                else A::clear(state);
                float kept = 1.0f;
                const auto part = [&] {
                    const Args &a = again<Args>();
                    return Part{moved_on(a.grad_out, w.of(a.os), bytes), moved_on(a.v, w.of(a.vs), bytes), moved_on(a.k, w.of(a.ks), bytes),
                                moved_on(a.grad_q, w.of(a.gqs), bytes), a.os.tick, a.vs.tick, a.ks.tick, a.gqs.tick, a.values, a.keys, 0, a.exactly, a.scale, 1.0f};
                };
                A::template go_through<true>(state, kept, g, v, k, within, wild, turn, part, [&](int64_t begin) { return course(begin, 0); }, first, last, decay);
            }
        }
        typename A::State turned, state;
        int64_t begin, last;
        {
            const Args &a = again<Args>();
            if (!a.grad_k && !a.grad_v && !a.grad_state_in) continue;
            // the segment that ends where the one forwards begins to count
            const int segment = a.segments - 1 - w.segment;
            const int64_t size = a.keys * a.values;
            begin = segment * a.segment, last = min(begin + a.segment, a.ticks);
            const float *const s = a.grad_states ? a.grad_states + (w.rh * a.segments + segment) * size
                                                 : a.grad_state_out ? a.grad_state_out + w.rh * size : nullptr;
            if (s) {
                A::load_state(turned, s, a.values, a.keys, 1, a.values);
                A::load_state(state, s, a.keys, a.values, a.values, 1);
            } else {
                A::clear(turned);
                A::clear(state);
            }
        }
        const auto to_k = [&] {
            const Args &a = again<Args>();
            return Part{moved_on(a.v, w.of(a.vs), bytes), moved_on(a.grad_out, w.of(a.os), bytes), moved_on(a.q, w.of(a.qs), bytes),
                        moved_on(a.grad_k, w.of(a.gks), bytes), a.vs.tick, a.os.tick, a.qs.tick, a.gks.tick, a.values, a.keys, 1, a.exactly, 1.0f, a.scale};
        };
        const auto to_v = [&] {
            const Args &a = again<Args>();
            return Part{moved_on(a.k, w.of(a.ks), bytes), moved_on(a.q, w.of(a.qs), bytes), moved_on(a.grad_out, w.of(a.os), bytes),
                        a.grad_v ? moved_on(a.grad_v, w.of(a.gvs), bytes) : nullptr, a.ks.tick, a.qs.tick, a.os.tick, a.gvs.tick, a.keys, a.values,
                        1, a.exactly, 1.0f, a.scale};
        };
        typename A::Rows qr, kr, vr, gr;
        int flag = 0, small = 0;                   // (as in go_through, of both states)
        const auto fetch = [&](int64_t from) {
            const Course c = course(from, 1);
            const int n = (int)min((int64_t)C, last - from);
            const Part a = to_v();
            A::load(qr, a.k, a.k_tick, c, n, a.keys);
            A::load(kr, a.q, a.q_tick, c, n, a.keys);
            A::load(gr, a.v, a.v_tick, c, n, a.values);
            const Part b = to_k();
            A::load(vr, b.q, b.q_tick, c, n, b.keys);
            flag = c.begins(lane, n);
        };
        for (; begin < last; begin += C) {
            const int n = (int)min((int64_t)C, last - begin);
            fetch(begin);
            float l2 = decay;                      // (as in go_through)
            int col = lane & 15, quad = lane >> 4;
            asm volatile("" : "+v"(l2), "+v"(col), "+v"(quad));
            turn ^= 1;
            if (threadIdx.x == 0) wild[turn] = again<Args>().exactly;
            lds_meet();
            uint32_t odd = A::store(k, kr) | A::store(v, vr) | A::store(q, qr) | A::store(g, gr);
            if (small == 0) odd |= (uint32_t)A::large(turned) | (uint32_t)A::large(state);
            if (__ballot(odd != 0) && lane == 0) wild[turn] = 1;
            const uint64_t begins = __ballot(flag != 0);
            lds_meet();
            const bool odd_one = wild[turn] != 0;
            if (again<Args>().grad_k) {
                A::compare(within, v, g, begins, l2, again<Args>().scale, wave, col, quad);
                lds_meet();
                const Part a = to_k();
                const Course c = course(begin, 1);
                if (__builtin_expect(odd_one, 0)) A::template advance_slowly<true>(turned, begins, n, l2, a, c, wave, col, quad);
                else A::template advance<true>(turned, within, v, g, q, begins, n, l2, a, c, wave, col, quad, [] {});
                lds_meet();
            }
            A::compare(within, k, q, begins, l2, again<Args>().scale, wave, col, quad);
            lds_meet();
            const Part a = to_v();
            const Course c = course(begin, 1);
            if (__builtin_expect(odd_one, 0)) A::template advance_slowly<true>(state, begins, n, l2, a, c, wave, col, quad);
            else A::template advance<true>(state, within, k, q, g, begins, n, l2, a, c, wave, col, quad, [] {});
            small = __builtin_amdgcn_readfirstlane(odd_one) ? 0 : (small == 0 ? kSmallChunks : small) - 1;
        }
        // what is left for the state before the first tick, if that belongs to its episode
        const Args &a = again<Args>();
        if (a.grad_state_in && w.segment == 0)
            A::store_state(state, a.grad_state_in + w.rh * (a.keys * a.values), a.keys, a.values, a.values, 1, a.fresh && a.ticks > 0 && a.fresh[w.env] != 0);
    }
}

// The gradients, each by a workgroup of its own: neighbours, which share what they read.  64 ticks of 5120 heads of 128 in
// bf16 746 us; 100 ticks of 1887 heads of 48 x 80 in f32, half of them controlled, 379 us, most of it waits of one
// workgroup at a time on a CU for its own steps.
template <int D, int TYPE, int C>
__global__ __launch_bounds__(4 * D, attention_grad_wavefronts(D, TYPE)) void tabx_attention_grad_apart_kernel(const AttentionGradArgs)
{
    typedef Attention<D, TYPE, C> A;
    typedef AttentionGradArgs Args;
    typedef typename A::T T;
    constexpr int bytes = sizeof(T);
    __shared__ typename A::In q, k, v;
    __shared__ typename A::Within within;
    __shared__ int wild[2];
    int turn = 0;
    for (int64_t id = blockIdx.x; id < 3 * again<Args>().works; id += gridDim.x) {
        const int64_t at = 3 * again<Args>().works <= gridDim.x ? neighbour(id, 3 * again<Args>().works) : id;
        const int64_t which = uniform(at / 3);
        const int role = (int)(at - 3 * which);
        const Work w(again<Args>(), which, 0);
        // grad_q: queries grad_out, keys v, values k; grad_k: queries v, keys grad_out, values q; grad_v: queries k, keys q,
        // values grad_out
        const auto part = [&] {
            const Args &a = again<Args>();
            const void *const xq = moved_on(a.q, w.of(a.qs), bytes), *const xk = moved_on(a.k, w.of(a.ks), bytes),
                              *const xv = moved_on(a.v, w.of(a.vs), bytes), *const xg = moved_on(a.grad_out, w.of(a.os), bytes);
            if (role == 0) return Part{xg, xv, xk, moved_on(a.grad_q, w.of(a.gqs), bytes), a.os.tick, a.vs.tick, a.ks.tick, a.gqs.tick, a.values, a.keys, 0, a.exactly, a.scale, 1.0f};
            if (role == 1) return Part{xv, xg, xq, moved_on(a.grad_k, w.of(a.gks), bytes), a.vs.tick, a.os.tick, a.qs.tick, a.gks.tick, a.values, a.keys, 1, a.exactly, 1.0f, a.scale};
            return Part{xk, xq, xg, a.grad_v ? moved_on(a.grad_v, w.of(a.gvs), bytes) : nullptr, a.ks.tick, a.qs.tick, a.os.tick, a.gvs.tick, a.keys, a.values, 1, a.exactly, 1.0f, a.scale};
        };
        const auto course = [&](int64_t begin) {
            const Args &a = again<Args>();
            return Course{a.fresh ? a.fresh + w.env : nullptr, a.envs, a.ticks, begin, role != 0};
        };
        typename A::State state;
        float kept = 1.0f, decay;
        int64_t first, last;
        {
            const Args &a = again<Args>();
            if (role == 0 ? !a.grad_q : role == 1 ? !a.grad_k : !a.grad_v && !a.grad_state_in) continue;
            const int64_t size = a.keys * a.values;
            first = w.segment * a.segment, last = min(first + a.segment, a.ticks);
            if (a.controlled && a.controlled[w.r] == 0) {
                const Part p = part();
                if (p.out) A::clear_rows(p.out, p.out_tick, first, last, p.values);
                if (role == 2 && a.grad_state_in && w.segment == 0)
                    for (int j = threadIdx.x; j < size; j += A::THREADS) a.grad_state_in[w.rh * size + j] = 0.0f;
                continue;
            }
            decay = fmaxf(log2_decay(a.log_decay, w.h), -1e9f);
            const float *const before = role == 0 ? a.states : a.grad_states, *const given = role == 0 ? a.state_in : a.grad_state_out;
            const float *const from = before ? before + w.at * size : given ? given + w.rh * size : nullptr;
            if (!from) A::clear(state);
            else if (role == 2) A::load_state(state, from, a.keys, a.values, a.values, 1);
            else A::load_state(state, from, a.values, a.keys, 1, a.values);
        }
        A::template go_through<true>(state, kept, q, k, v, within, wild, turn, part, course, first, last, decay);
        // what is left for the state before the first tick, if that belongs to its episode
        const Args &a = again<Args>();
        if (role == 2 && a.grad_state_in && w.segment == a.segments - 1)
            A::store_state(state, a.grad_state_in + w.rh * (a.keys * a.values), a.keys, a.values, a.values, 1, a.fresh && a.ticks > 0 && a.fresh[w.env] != 0);
    }
}

// The states that the segments leave become those before them, one behind the other: a thread per element, with 32 segments
// under way at a time, as a load behind a store into what may be the same array would wait for it (64 segments of 8 states
// of 128 x 128 13 us).
static __global__ __launch_bounds__(256) void tabx_attention_join_kernel(const AttentionPair pair)
{
    const AttentionArgs &a = pair.of[blockIdx.y];
    constexpr int AHEAD = 32;
    const int64_t size = (int64_t)a.keys * a.values, all = a.rows * a.heads * size;
    for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x; at < all; at += (int64_t)gridDim.x * 256) {
        const int64_t rh = at / size, d = at % size;
        if (a.controlled && a.controlled[rh / a.heads] == 0) continue;
        float s = a.state_in ? a.state_in[rh * size + d] : 0.0f;
        float *const of = a.carried + rh * a.segments * size + d;
        const float *const kept = a.kept + rh * a.segments;
        for (int n = 0; n < a.segments; n += AHEAD) {          // (the last one's, which is not there, goes nowhere)
            float left[AHEAD], part[AHEAD];        // all of them before the first store, behind which they would be loaded one by one
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) {
                const int at = min(n + i, a.segments - 1);
                left[i] = of[at * size], part[i] = kept[at];
            }
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) {
                if (n + i >= a.segments) break;
                of[(n + i) * size] = s;
                s = part[i] < 0.0f ? left[i] : fmaf(part[i], s, left[i]);
            }
        }
    }
}

} // namespace tabx
