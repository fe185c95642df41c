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
#include "tabx_rows.h"

#pragma clang fp contract(off)

namespace tabx {

typedef float f32x16 __attribute__((ext_vector_type(16)));

struct Strides {
    int64_t tick, row, head;
};

struct AttentionArgs {
    const void *q, *k, *v;
    void       *out;               // or nullptr
    Strides     qs, ks, vs, os;
    const float *log_decay;
    const uint8_t *fresh;          // [ticks][rows / units], or nullptr
    const uint8_t *controlled;     // [rows], or nullptr
    const float *state_in;         // or nullptr: zero
    float      *state_out;         // or nullptr
    float      *carried;           // [row and head][segment][keys][values]: states before each segment, or nullptr
    float      *kept;              // [row and head][segment]: what a segment leaves of the state before it; -1: an episode begins in it
    int64_t     ticks, rows, envs, works, state_key, state_value;   // works: rows x heads x segments; strides of a state's elements
    int64_t     segment;           // ticks of a segment, a multiple of the chunk
    int32_t     segments, heads, units, keys, values, type;
    int32_t     backward;          // in time
    int32_t     zero_out;          // rows that are not controlled get zeros (gradients)
    float       scale_within, scale_state, scale_added;
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
// one run.  VALUES: the values rounded up to a power of two; lanes beyond the last value idle.
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
#pragma unroll
        for (int n = 0; n < 4; ++n)
            if (n < count) value[n] = (float)v[n];
        if (a.values % 4 == 0) {
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
        } else {
            for (int i = line; i < a.keys; i += LINES) {
                const float x = (float)k[i], y = (float)q[i];
#pragma unroll
                for (int n = 0; n < 4; ++n) {
                    if (n >= count) continue;
                    float s = state[i * a.values + n];
                    s = fmaf(x, value[n], forget ? 0.0f : e * s);
                    state[i * a.values + n] = s;
                    sum[n] = fmaf(y, s, sum[n]);
                }
            }
        }
#pragma unroll
        for (int n = ACROSS; n < LANES; n *= 2)
#pragma unroll
            for (int m = 0; m < 4; ++m) sum[m] += __shfl_xor(sum[m], n);
        if (line == 0 && count > 0) {
            T *const out = (T *)a.out + r * a.os.row + h * a.os.head + d;
            sum *= a.scale;
            if (count >= 4) {
                store_four<TYPE>(out, sum);
            } else {
#pragma unroll
                for (int n = 0; n < 3; ++n)
                    if (n < count) out[n] = (T)sum[n];
            }
        }
    }
}

// --- many ticks ---------------------------------------------------------------------------------

// The products run in the matrix cores in bf16 with sums in 32 bits, where every 32-bit operand stands as the sum of parts
// of 8 bits each: bf16 inputs are one part, f16 ones two (both exact), f32 ones three; what lies between (the products of
// queries and keys, the state, the faded values) is cut into two parts, three for f32.  Of the parts' products those are taken
// that are above the last part's own rounding, so that 2^-16 of a term is lost, 2^-23 for f32 (a term's rounding to the
// output is 2^-8, 2^-11, 2^-24), and nothing can leave the range of 32 bits that 32 bits would hold.
template <int TYPE> struct Parts {
    static constexpr int in = TYPE == TABX_BF16 ? 1 : TYPE == TABX_F16 ? 2 : 3;
    static constexpr int mid = TYPE == TABX_F32 ? 3 : 2;
};

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int chunk_of(int d, int type) { return type == TABX_BF16 && d > 32 ? 64 : 32; }

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

// One product of operands in parts, the smallest parts' first.
template <int NA, int NB>
__device__ __forceinline__ f32x4 multiply(const bf16x8 (&a)[NA], const bf16x8 (&b)[NB], f32x4 c)
{
    constexpr int last = NA > NB ? NA : NB;
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
        } else if (count > 0) {                    // a width that is no multiple of eight
#pragma unroll
            for (int i = 0; i < 7; ++i) {
                if (i >= count) continue;
                if constexpr (TYPE == TABX_F32) v[i / 4][i % 4] = ((const uint32_t *)from)[i];
                else v[0][i / 2] |= (uint32_t)((const uint16_t *)from)[i] << 16 * (i % 2);
            }
        }
    }
};

// Not 0 in a bit of its own if one of them is not finite (an exponent of ones carries).
template <int TYPE>
__device__ __forceinline__ uint32_t not_finite(const Eight<TYPE> &e)
{
    constexpr uint32_t exponent = TYPE == TABX_F32 ? 0x7f800000u : TYPE == TABX_BF16 ? 0x7f807f80u : 0x7c007c00u;
    constexpr uint32_t one = TYPE == TABX_F32 ? 0x00800000u : TYPE == TABX_BF16 ? 0x00800080u : 0x04000400u;
    uint32_t found = 0;
#pragma unroll
    for (int n = 0; n < (TYPE == TABX_F32 ? 2 : 1); ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) found |= (e.v[n][i] & exponent) + one;
    return found & (TYPE == TABX_F32 ? 0x80000000u : 0x80008000u);
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

// One row's head (or a segment of its ticks) as an attention goes through it, and which way.
struct Course {
    int64_t ticks, begin;          // of all; where the chunk at hand begins, counted in the direction of time taken
    int     backward;
    __device__ __forceinline__ int64_t tick(int i) const { return backward ? ticks - 1 - (begin + i) : begin + i; }
};

template <int D, int TYPE>
struct Attention {
    static constexpr int C = chunk_of(D, TYPE), IN = Parts<TYPE>::in, MID = Parts<TYPE>::mid;
    static constexpr int WAVES = D / 16, THREADS = 64 * WAVES, PASSES = C * D / 8 / THREADS, TILES = D / 16;
    typedef Tile<D, C, IN> In;
    static constexpr int kWithin = C + 8;          // distance of rows of the products of queries and keys

    // A wavefront has 16 of the values and all of the state's lines of them, in the layout in which a product leaves its
    // result (a lane has four lines of one column), which is that of an operand of the next one (`along_results`).
    typedef f32x4 State[TILES];

    struct Rows { Eight<TYPE> e[PASSES]; };

    static __device__ __forceinline__ void load(Rows &rows, const void *data, int64_t at, int64_t tick, const Course &c, int n, int width)
    {
        constexpr int across = D / 8;
        const int d = 8 * ((int)threadIdx.x % across), row = (int)threadIdx.x / across;
        const int64_t step = c.backward ? -tick : tick;
        const typename Element<TYPE>::one *const from = (const typename Element<TYPE>::one *)data + at + c.tick(0) * tick + row * step + d;
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
            found |= not_finite<TYPE>(rows.e[p]);
        }
        return found;
    }

    // Products of queries and keys, faded by the ticks between them, 0 where they do not belong together, in parts:
    // tiles of 16 x 16 on and below the diagonal, dealt to the wavefronts.  Rows are queries; along them the keys lie in the
    // order of `along_results`, so that a lane's eight are next to each other.
    static __device__ __forceinline__ void compare(__bf16 (&within)[MID][C * kWithin], const In &q, const In &k, uint64_t begins, float l2,
                                                   const float (&power)[4], float scale, int wave, int col, int quad)
    {
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
                for (int r = 0; r < 4; ++r) p[r] *= fade * power[3 - r];
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
            const int at = i * kWithin + 32 * (J / 2) + 8 * quad + 4 * (J % 2);
#pragma unroll
            for (int m = 0; m < MID; ++m) {
                *(bf16x4 *)&within[m][at] = part[m];
                if (I == J && I % 2 == 0) *(u32x2 *)&within[m][at + 4] = u32x2{0, 0};
            }
        }
    }

    // What a chunk's queries read, and the state behind the chunk.
    template <bool READS>
    static __device__ __forceinline__ void advance(State &state, const __bf16 (&within)[MID][C * kWithin], const In &q, const In &k, const In &v,
                                                   uint64_t begins, int n, float l2, const float (&power)[4], const AttentionArgs &a,
                                                   const Course &c, int64_t out_at, int wave, int col, int quad)
    {
        bf16x8 values[C / 32][IN];                 // this lane's: 8 ticks of its column, of every 32
#pragma unroll
        for (int b = 0; b < C / 32; ++b) v.across(values[b], 32 * b, 16 * wave, col, quad);
        if constexpr (READS) {
            bf16x8 held[D / 32][MID];
#pragma unroll
            for (int s = 0; s < D / 32; ++s) {
                bf16x4 x[MID], y[MID];
                split(x, state[2 * s]);
                split(y, state[2 * s + 1]);
#pragma unroll
                for (int m = 0; m < MID; ++m) held[s][m] = join(x[m], y[m]);
            }
            const int d = 16 * wave + 4 * quad;
            const int64_t step = c.backward ? -a.os.tick : a.os.tick;
            typename Element<TYPE>::one *const out = (typename Element<TYPE>::one *)a.out + out_at + c.tick(0) * a.os.tick + col * step + d;
#pragma unroll
            for (int I = 0; I < C / 16; ++I) {
                if (16 * I >= n) break;
                __builtin_amdgcn_sched_barrier(0); // (operands of all of them at a time would not fit)
                const int i = 16 * I + col;
                f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int s = 0; s < D / 32; ++s) {
                    bf16x8 x[IN];
                    q.along_results(x, 16 * I, 32 * s, col, quad);
                    o = multiply(held[s], x, o);
                }
                const float fade = __builtin_amdgcn_exp2f(l2 * (float)(i + 1 - a.backward)) * a.scale_state;
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
                    for (int m = 0; m < MID; ++m) x[m] = *(const bf16x8 *)&within[m][i * kWithin + 32 * b + 8 * quad];
                    o = multiply(values[b], x, o);
                }
                if (a.out && i < n && d < a.values) {
                    typename Element<TYPE>::one *const to = out + 16 * I * step;
                    if (d + 4 <= a.values) {
                        store_four<TYPE>(to, o);
                    } else {
#pragma unroll
                        for (int r = 0; r < 3; ++r)
                            if (d + r < a.values) to[r] = (typename Element<TYPE>::one)o[r];
                    }
                }
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        // the values faded by the ticks behind theirs; those of episodes that have ended count no more
        const int newest = begins ? 63 - __builtin_clzll(begins) : 0;
        const float left = __builtin_amdgcn_exp2f(l2 * (float)n);
        bf16x8 faded[C / 32][MID];
#pragma unroll
        for (int b = 0; b < C / 32; ++b) {
            bf16x4 part[2][MID];
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                f32x4 x = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int p = IN - 1; p >= 0; --p) {
                    const bf16x4 y = half ? __builtin_shufflevector(values[b][p], values[b][p], 4, 5, 6, 7)
                                          : __builtin_shufflevector(values[b][p], values[b][p], 0, 1, 2, 3);
                    x += __builtin_convertvector(y, f32x4);
                }
                const int first = 32 * b + 16 * half + 4 * quad;
                if (n == C) {
                    const float fade = __builtin_amdgcn_exp2f(l2 * (float)(C - 4 - first + a.backward)) * a.scale_added;
#pragma unroll
                    for (int r = 0; r < 4; ++r) x[r] *= fade * power[3 - r];
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
#pragma unroll
            for (int m = 0; m < MID; ++m) faded[b][m] = join(part[0][m], part[1][m]);
        }
#pragma unroll
        for (int s = 0; s < TILES; ++s) {
            f32x4 x = {0.0f, 0.0f, 0.0f, 0.0f};
            if (!begins) x = state[s] * left;
#pragma unroll
            for (int b = 0; b < C / 32; ++b) {
                if (32 * b >= n) break;
                bf16x8 y[IN];
                k.across(y, 32 * b, 16 * s, col, quad);
                x = multiply(y, faded[b], x);
            }
            state[s] = x;
        }
    }

    // The same for a chunk with keys or values that are not finite, tick by tick: in a product of matrices they would reach
    // ticks that they do not belong to, as zero times them is not zero.
    template <bool READS>
    static __device__ void advance_slowly(State &state, uint64_t begins, int n, float l2, const AttentionArgs &a, const Course &c,
                                          int64_t q_at, int64_t k_at, int64_t v_at, int64_t out_at, int wave, int col, int quad)
    {
        const float e = __builtin_amdgcn_exp2f(l2);
        const int d = 16 * wave + col;
        for (int i = 0; i < n; ++i) {
            const int64_t t = c.tick(i);
            const bool begun = begins >> i & 1;
            const float value = d < a.values ? element<TYPE>(a.v, v_at + t * a.vs.tick + d) * a.scale_added : 0.0f;
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
                        x = fmaf(element<TYPE>(a.k, k_at + t * a.ks.tick + key), value, x);
                        if (READS) sum = fmaf(element<TYPE>(a.q, q_at + t * a.qs.tick + key), x, sum);
                    }
                    state[s][r] = a.backward ? x * e : x;
                }
            }
            if constexpr (READS) {
                sum += __shfl_xor(sum, 16);
                sum += __shfl_xor(sum, 32);
                if (a.out && quad == 0 && d < a.values)
                    ((typename Element<TYPE>::one *)a.out)[out_at + t * a.os.tick + d] = (typename Element<TYPE>::one)(sum * a.scale_state);
            }
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

// A workgroup has a row's head, or a segment of its ticks, and goes through the chunks with the state in registers; the
// next chunk's rows are under way while it works on the present one.  CARRY: nothing is read, the states that the segments
// would leave of nothing are.
constexpr int attention_wavefronts(int d) { return d == 128 ? 2 : d == 64 ? 3 : 4; }   // of a SIMD

template <int D, int TYPE, bool CARRY>
__global__ __launch_bounds__(4 * D, attention_wavefronts(D)) void tabx_attention_kernel(const AttentionArgs a)
{
    typedef Attention<D, TYPE> A;
    constexpr int C = A::C;
    __shared__ typename A::In q, k, v;
    __shared__ __bf16 within[A::MID][C * A::kWithin];
    __shared__ int wild[2];                                    // of this chunk and the one before: not all is finite
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    int turn = 0;
    for (int64_t id = blockIdx.x; id < a.works; id += gridDim.x) {
        const int64_t w = a.works <= gridDim.x ? neighbour(id, a.works) : id;
        // (a division's result is the same for all, but not known to be)
        const int64_t rh = a.segments == 1 ? w : uniform(w / a.segments);
        const int segment = (int)(w - rh * a.segments);
        const int64_t r = __builtin_amdgcn_readfirstlane((int)((uint32_t)rh / (uint32_t)a.heads));       // (rows x heads has 31 bits)
        const int h = (int)(rh - r * a.heads);
        const int64_t first = segment * a.segment, last = min(first + a.segment, a.ticks);
        const int64_t env = __builtin_amdgcn_readfirstlane((int)((uint32_t)r / (uint32_t)a.units));
        const int64_t q_at = r * a.qs.row + h * a.qs.head, k_at = r * a.ks.row + h * a.ks.head, v_at = r * a.vs.row + h * a.vs.head,
                      out_at = r * a.os.row + h * a.os.head;
        if (CARRY && segment == a.segments - 1) continue;      // (nothing comes behind it)
        if (a.controlled && a.controlled[r] == 0) {
            if (CARRY || !a.zero_out) continue;
            for (int64_t t = first; a.out && t < last; ++t)
                for (int j = threadIdx.x; j < a.values; j += A::THREADS)
                    ((typename Element<TYPE>::one *)a.out)[out_at + (a.backward ? a.ticks - 1 - t : t) * a.os.tick + j] = (typename Element<TYPE>::one)0.0f;
            if (a.state_out && segment == a.segments - 1)
                for (int j = threadIdx.x; j < a.keys * a.values; j += A::THREADS)
                    a.state_out[rh * a.keys * a.values + (j / a.values) * a.state_key + (j % a.values) * a.state_value] = 0.0f;
            continue;
        }
        const float decay = fmaxf(log2_decay(a.log_decay, h), -1e9f);  // (all at once, and none of no ticks)
        // a lane's elements of a state, as offsets from a place that is the same for all; worked out where they are needed
        // and not kept meanwhile
        const auto each = [&](int along_keys, int along_values, auto visit) {
            int here = 0;
            asm volatile("" : "+v"(here));
            const int value = 16 * wave + (lane & 15) + here, first_key = 4 * (lane >> 4) + here, at = first_key * along_keys + value * along_values;
            if (a.keys == D && a.values == D) {
#pragma unroll
                for (int s = 0; s < A::TILES; ++s)
#pragma unroll
                    for (int i = 0; i < 4; ++i) visit(s, i, (16 * s + i) * along_keys, at);
            } else if (value < a.values) {
#pragma unroll
                for (int s = 0; s < A::TILES; ++s)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (first_key + 16 * s + i < a.keys) visit(s, i, (16 * s + i) * along_keys, at);
            }
        };
        typename A::State state;
#pragma unroll
        for (int s = 0; s < A::TILES; ++s) state[s] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        if (!CARRY && a.carried) {
            const float *const from = a.carried + w * a.keys * a.values;
            each(a.values, 1, [&](int s, int i, int from_there, int at) { state[s][i] = (from + from_there)[at]; });
        } else if (!CARRY && a.state_in) {
            const float *const from = a.state_in + rh * a.keys * a.values;
            each((int)a.state_key, (int)a.state_value, [&](int s, int i, int from_there, int at) { state[s][i] = (from + from_there)[at]; });
        }
        float power[4];                            // of the decay, for 0 to 3 ticks
#pragma unroll
        for (int i = 0; i < 4; ++i) power[i] = __builtin_amdgcn_exp2f(decay * (float)i);
        float kept = 1.0f;
        typename A::Rows qr, kr, vr;
        int flag = 0;
        Course next = {a.ticks, first, a.backward};
        const auto fetch = [&](int n) {
            if constexpr (!CARRY) A::load(qr, a.q, q_at, a.qs.tick, next, n, a.keys);
            A::load(kr, a.k, k_at, a.ks.tick, next, n, a.keys);
            A::load(vr, a.v, v_at, a.vs.tick, next, n, a.values);
            flag = 0;
            if (a.fresh && lane < n) {
                // backwards, an episode begins behind the tick where, forwards, the next one does
                const int64_t t = next.begin + lane;
                if (!a.backward) flag = a.fresh[t * a.envs + env];
                else if (t > 0) flag = a.fresh[(a.ticks - t) * a.envs + env];
            }
        };
        if (first < last) fetch((int)min((int64_t)C, last - first));
        for (int64_t begin = first; begin < last; begin += C) {
            const int n = (int)min((int64_t)C, last - begin);
            const Course here = next;
            // powers and places are worked out for every chunk: kept, they would cost a wavefront
            float l2 = decay;
            int col = lane & 15, quad = lane >> 4;
            asm volatile("" : "+v"(l2), "+v"(col), "+v"(quad));
            turn ^= 1;
            if (threadIdx.x == 0) wild[turn] = 0;
            __syncthreads();                                   // the chunk before has been worked on
            if constexpr (!CARRY) A::store(q, qr);
            const uint32_t odd = A::store(k, kr) | A::store(v, vr);
            if (__ballot(odd != 0) && lane == 0) wild[turn] = 1;
            const uint64_t begins = __ballot(flag != 0);       // bit i: an episode begins with the chunk's tick i
            next.begin += C;
            if (next.begin < last) fetch((int)min((int64_t)C, last - next.begin));
            __syncthreads();
            if constexpr (!CARRY) {
                A::compare(within, q, k, begins, l2, power, a.scale_within, wave, col, quad);
                __syncthreads();
            }
            if (__builtin_expect(wild[turn], 0)) A::template advance_slowly<!CARRY>(state, begins, n, l2, a, here, q_at, k_at, v_at, out_at, wave, col, quad);
            else A::template advance<!CARRY>(state, within, q, k, v, begins, n, l2, power, a, here, out_at, wave, col, quad);
            kept = begins || kept < 0.0f ? -1.0f : kept * __builtin_amdgcn_exp2f(l2 * (float)n);
        }
        float *const to = CARRY ? a.carried + w * a.keys * a.values : segment == a.segments - 1 ? a.state_out : nullptr;
        if (CARRY && threadIdx.x == 0) a.kept[w] = kept;
        if (!to) continue;
        // backwards, what is left for the state before the first tick, if that belongs to its episode
        const bool cut = !CARRY && a.backward && a.fresh && a.ticks > 0 && a.fresh[env] != 0;
        if (CARRY) {
            each(a.values, 1, [&](int s, int i, int from_there, int at) { (to + from_there)[at] = state[s][i]; });
        } else {
            float *const of = to + rh * a.keys * a.values;
            each((int)a.state_key, (int)a.state_value, [&](int s, int i, int from_there, int at) { (of + from_there)[at] = cut ? 0.0f : state[s][i]; });
        }
    }
}

// The states that the segments leave become those before them, one behind the other: a thread per element.
static __global__ __launch_bounds__(256) void tabx_attention_join_kernel(const AttentionArgs a)
{
    constexpr int AHEAD = 16;
    const int64_t size = (int64_t)a.keys * a.values, all = a.rows * a.heads * size;
    for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x; at < all; at += (int64_t)gridDim.x * 256) {
        const int64_t rh = at / size, d = at % size;
        if (a.controlled && a.controlled[rh / a.heads] == 0) continue;
        float s = a.state_in ? a.state_in[rh * size + d / a.values * a.state_key + d % a.values * a.state_value] : 0.0f;
        float *const of = a.carried + rh * a.segments * size + d;
        const float *const kept = a.kept + rh * a.segments;
        for (int n = 0; n < a.segments; n += AHEAD) {          // (what the last one leaves is the attention's to work out)
            float left[AHEAD];
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) left[i] = n + i < a.segments - 1 ? of[(n + i) * size] : 0.0f;
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) {
                if (n + i >= a.segments) break;
                of[(n + i) * size] = s;
                if (n + i < a.segments - 1) s = kept[n + i] < 0.0f ? left[i] : fmaf(kept[n + i], s, left[i]);
            }
        }
    }
}

} // namespace tabx
