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

__device__ __forceinline__ float element_of(const void *data, int64_t at, int type)
{
    return type == TABX_F32 ? element<TABX_F32>(data, at) : type == TABX_BF16 ? element<TABX_BF16>(data, at) : element<TABX_F16>(data, at);
}

__device__ __forceinline__ void put_element(void *data, int64_t at, float v, int type)
{
    if (type == TABX_F32) ((float *)data)[at] = v;
    else if (type == TABX_BF16) ((__bf16 *)data)[at] = (__bf16)v;
    else ((_Float16 *)data)[at] = (_Float16)v;
}

// --- one tick -----------------------------------------------------------------------------------

// A wavefront has a row's head: its lanes lie along the values, and there are several of the state's lines at a time.
struct StepArgs {
    const void *q, *k, *v;
    void       *out;
    Strides     qs, ks, vs, os;
    const float *log_decay;
    const uint8_t *fresh, *controlled;
    float      *state;
    int64_t     works;             // rows x heads
    int32_t     heads, units, keys, values, type;
    float       scale;
};

template <int LANES>
__global__ __launch_bounds__(256) void tabx_attention_step_kernel(const StepArgs a)
{
    constexpr int LINES = 64 / LANES;
    const int lane = (int)threadIdx.x & 63, d = lane % LANES, line = lane / LANES;
    for (int64_t w = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); w < a.works; w += (int64_t)gridDim.x * 4) {
        const int64_t r = w / a.heads;
        const int h = (int)(w % a.heads);
        if (a.controlled && a.controlled[r] == 0) continue;
        const bool forget = a.fresh && a.fresh[r / a.units] != 0;
        const float e = decayed(log2_decay(a.log_decay, h), 1);
        float *state = a.state + w * a.keys * a.values;
        const int64_t q = r * a.qs.row + h * a.qs.head, k = r * a.ks.row + h * a.ks.head, v = r * a.vs.row + h * a.vs.head;
        for (int j = d; j < a.values; j += LANES) {
            const float value = element_of(a.v, v + j, a.type);
            float sum = 0.0f;
            for (int i = line; i < a.keys; i += LINES) {
                float s = state[(int64_t)i * a.values + j];
                s = fmaf(element_of(a.k, k + i, a.type), value, forget ? 0.0f : e * s);
                state[(int64_t)i * a.values + j] = s;
                sum = fmaf(element_of(a.q, q + i, a.type), s, sum);
            }
#pragma unroll
            for (int n = LANES; n < 64; n *= 2) sum += __shfl_xor(sum, n);
            if (line == 0) put_element(a.out, r * a.os.row + h * a.os.head + j, sum * a.scale, a.type);
        }
    }
}

// --- many ticks ---------------------------------------------------------------------------------

constexpr int kChunk = 32;

// A workgroup has a row's head, or a segment of its ticks, and goes through the chunks with the state in registers.  Its
// wavefronts share out the values: each holds all of the state's lines of 16 (or 32) of them, in the layout in which a
// product leaves its result (a lane has four lines of one column), which is that of a right operand of the next product:
// the state goes into the matrix cores as it is.  Products are of 32 bits (16 x 16 x 4): a lane's element s of four
// consecutive ones is that of step s, on both sides.  D: keys and values, filled up with zeros.
template <int D, bool CARRY>
__global__ __launch_bounds__(D >= 64 ? 256 : 4 * D) void tabx_attention_kernel(const AttentionArgs a)
{
    constexpr int C = kChunk, WAVES = D >= 64 ? 4 : D / 16, THREADS = 64 * WAVES;
    constexpr int TILES = D / 16, MINE = TILES / WAVES;        // tiles of 16 keys; of 16 values, and this wavefront's of them
    constexpr int WIDE = D + 4, LONG = C + 4;
    __shared__ float qs[C][WIDE], ks[C][WIDE], kt[D][LONG], vt[D][LONG], within[C][LONG];
    __shared__ uint32_t wild[2];                               // of this chunk and the one before: ticks with values that are not finite
    int turn = 0;
    const int lane = (int)threadIdx.x & 63, wave = (int)threadIdx.x >> 6, col = lane & 15, quad = lane >> 4;
    for (int64_t w = blockIdx.x; w < a.works; w += gridDim.x) {
        const int segment = (int)(w % a.segments);
        const int64_t rh = w / a.segments, r = rh / a.heads;
        const int h = (int)(rh % a.heads);
        const int64_t first = segment * a.segment, last = min(first + a.segment, a.ticks);
        const int64_t env = r / a.units;
        if (a.controlled && a.controlled[r] == 0) {
            if (CARRY || !a.zero_out) continue;
            for (int64_t t = first; a.out && t < last; ++t)
                for (int j = threadIdx.x; j < a.values; j += THREADS)
                    put_element(a.out, t * a.os.tick + r * a.os.row + h * a.os.head + j, 0.0f, a.type);
            if (a.state_out && segment == a.segments - 1)
                for (int j = threadIdx.x; j < a.keys * a.values; j += THREADS)
                    a.state_out[rh * a.keys * a.values + (j / a.values) * a.state_key + (j % a.values) * a.state_value] = 0.0f;
            continue;
        }
        const float l2 = log2_decay(a.log_decay, h);
        f32x4 state[MINE][TILES];
#pragma unroll
        for (int m = 0; m < MINE; ++m)
#pragma unroll
            for (int n = 0; n < TILES; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int key = 16 * n + 4 * quad + i, value = 16 * (wave * MINE + m) + col;
                    float s = 0.0f;
                    if (!CARRY && key < a.keys && value < a.values) {
                        if (a.carried) s = a.carried[(w * a.keys + key) * a.values + value];
                        else if (a.state_in) s = a.state_in[rh * a.keys * a.values + key * a.state_key + value * a.state_value];
                    }
                    state[m][n][i] = s;
                }
        float kept = 1.0f;
        for (int64_t begin = first; begin < last; begin += C) {
            const int n = (int)min((int64_t)C, last - begin);
            // bit i: an episode begins with the chunk's tick i
            const int64_t mine = begin + (lane < n ? lane : 0);
            const int64_t flag = a.backward ? a.ticks - mine : mine;
            const bool here = a.fresh && lane < n && !(a.backward && mine == 0) && a.fresh[flag * a.envs + env] != 0;
            const uint64_t begins = __ballot(here);
            const int newest = begins ? 63 - __builtin_clzll(begins) : 0;      // the last episode's first tick
            turn ^= 1;
            if (threadIdx.x == 0) wild[turn] = 0;
            __syncthreads();                                   // the chunk before has been read
            for (int at = threadIdx.x; at < C * D; at += THREADS) {
                const int i = at / D, d = at % D;
                const int64_t t = a.backward ? a.ticks - 1 - (begin + i) : begin + i;
                const bool key = i < n && d < a.keys, value = i < n && d < a.values;
                if (!CARRY) qs[i][d] = key ? element_of(a.q, t * a.qs.tick + r * a.qs.row + h * a.qs.head + d, a.type) : 0.0f;
                const float kv = key ? element_of(a.k, t * a.ks.tick + r * a.ks.row + h * a.ks.head + d, a.type) : 0.0f;
                if (!CARRY) ks[i][d] = kv;
                kt[d][i] = i >= newest ? kv : 0.0f;
                float vv = value ? element_of(a.v, t * a.vs.tick + r * a.vs.row + h * a.vs.head + d, a.type) : 0.0f;
                if (!(fabsf(vv) < INFINITY)) {
                    atomicOr(&wild[turn], 1u << i);
                    vv = 0.0f;
                }
                vt[d][i] = vv;
            }
            __syncthreads();
            if constexpr (!CARRY) {
                // the products of queries and keys, tiles of 16 x 16 on and below the diagonal
                for (int tile = wave; tile < (C / 16) * (C / 16 + 1) / 2; tile += WAVES) {
                    const int I = tile == 0 ? 0 : 1, J = tile == 2 ? 1 : 0;
                    f32x4 p = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                    for (int s = 0; s < TILES; ++s) {
                        const f32x4 x = *(const f32x4 *)&qs[16 * I + col][16 * s + 4 * quad], y = *(const f32x4 *)&ks[16 * J + col][16 * s + 4 * quad];
#pragma unroll
                        for (int i = 0; i < 4; ++i) p = __builtin_amdgcn_mfma_f32_16x16x4f32(x[i], y[i], p, 0, 0, 0);
                    }
                    const int j = 16 * J + col;
#pragma unroll
                    for (int s = 0; s < 4; ++s) {
                        const int i = 16 * I + 4 * quad + s;
                        const uint64_t up = begins & ((2ull << i) - 1);            // begun up to i
                        const bool same = j <= i && (up >> j) <= 1;                // none of them behind j
                        within[i][j] = same ? p[s] * decayed(l2, i - j) : 0.0f;
                    }
                }
                __syncthreads();
            }
            const uint32_t odd = wild[turn];
#pragma unroll
            for (int m = 0; m < MINE; ++m) {
                const int value = 16 * (wave * MINE + m) + col;
                if constexpr (!CARRY) {
#pragma unroll
                    for (int I = 0; I < C / 16; ++I) {
                        f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                        for (int s = 0; s < TILES; ++s) {
                            const f32x4 x = *(const f32x4 *)&qs[16 * I + col][16 * s + 4 * quad];
#pragma unroll
                            for (int i = 0; i < 4; ++i) o = __builtin_amdgcn_mfma_f32_16x16x4f32(x[i], state[m][s][i], o, 0, 0, 0);
                        }
#pragma unroll
                        for (int s = 0; s < 4; ++s) {
                            const int i = 16 * I + 4 * quad + s;
                            o[s] = begins & ((2ull << i) - 1) ? 0.0f : o[s] * (decayed(l2, i + 1 - a.backward) * a.scale_state);
                        }
                        f32x4 p = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                        for (int J = 0; J <= I; ++J) {
                            const f32x4 x = *(const f32x4 *)&within[16 * I + col][16 * J + 4 * quad], y = *(const f32x4 *)&vt[value][16 * J + 4 * quad];
#pragma unroll
                            for (int i = 0; i < 4; ++i) p = __builtin_amdgcn_mfma_f32_16x16x4f32(x[i], y[i], p, 0, 0, 0);
                        }
#pragma unroll
                        for (int s = 0; s < 4; ++s) {
                            const int i = 16 * I + 4 * quad + s;
                            float within_sum = p[s];
                            // values that are not finite, of ticks that count here (zero times them would not be zero)
                            if (odd && i < n && value < a.values) {
                                for (uint32_t left = odd; left; left &= left - 1) {
                                    const int j = __builtin_ctz(left);
                                    const int64_t t = a.backward ? a.ticks - 1 - (begin + j) : begin + j;
                                    const float x = element_of(a.v, t * a.vs.tick + r * a.vs.row + h * a.vs.head + value, a.type);
                                    const bool same = j <= i && ((begins & ((2ull << i) - 1)) >> j) <= 1;
                                    if (same && !(fabsf(x) < INFINITY)) within_sum += within[i][j] * x;
                                }
                            }
                            if (a.out && i < n && value < a.values) {
                                const int64_t t = a.backward ? a.ticks - 1 - (begin + i) : begin + i;
                                put_element(a.out, t * a.os.tick + r * a.os.row + h * a.os.head + value, fmaf(within_sum, a.scale_within, o[s]), a.type);
                            }
                        }
                    }
                }
                // the state behind the chunk
                const float left = decayed(l2, n);
                f32x4 fading[C / 16];                          // this lane's values, faded by the ticks behind theirs
#pragma unroll
                for (int J = 0; J < C / 16; ++J) {
                    fading[J] = *(const f32x4 *)&vt[value][16 * J + 4 * quad];
#pragma unroll
                    for (int i = 0; i < 4; ++i) fading[J][i] *= decayed(l2, n - 1 - (16 * J + 4 * quad + i) + a.backward) * a.scale_added;
                }
#pragma unroll
                for (int s = 0; s < TILES; ++s) {
                    f32x4 &x = state[m][s];
#pragma unroll
                    for (int i = 0; i < 4; ++i) x[i] = begins ? 0.0f : x[i] * left;
#pragma unroll
                    for (int J = 0; J < C / 16; ++J) {
                        const f32x4 y = *(const f32x4 *)&kt[16 * s + col][16 * J + 4 * quad];
#pragma unroll
                        for (int i = 0; i < 4; ++i) x = __builtin_amdgcn_mfma_f32_16x16x4f32(y[i], fading[J][i], x, 0, 0, 0);
                    }
                    if (odd && value < a.values) {
                        for (uint32_t rest = odd; rest; rest &= rest - 1) {
                            const int j = __builtin_ctz(rest);
                            if (j < newest) continue;
                            const int64_t t = a.backward ? a.ticks - 1 - (begin + j) : begin + j;
                            const float y = element_of(a.v, t * a.vs.tick + r * a.vs.row + h * a.vs.head + value, a.type);
                            if (!(fabsf(y) < INFINITY))
#pragma unroll
                                for (int i = 0; i < 4; ++i)
                                    x[i] += kt[16 * s + 4 * quad + i][j] * (y * (decayed(l2, n - 1 - j + a.backward) * a.scale_added));
                        }
                    }
                }
            }
            kept = begins || kept < 0.0f ? -1.0f : kept * decayed(l2, n);
        }
        float *const to = CARRY ? a.carried + w * a.keys * a.values : segment == a.segments - 1 ? a.state_out : nullptr;
        if (CARRY && threadIdx.x == 0) a.kept[w] = kept;
        if (!to) continue;
        // backwards, what is left for the state before the first tick, if that belongs to its episode
        const bool cut = !CARRY && a.backward && a.fresh && a.ticks > 0 && a.fresh[env] != 0;
#pragma unroll
        for (int m = 0; m < MINE; ++m)
#pragma unroll
            for (int n = 0; n < TILES; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int key = 16 * n + 4 * quad + i, value = 16 * (wave * MINE + m) + col;
                    if (key >= a.keys || value >= a.values) continue;
                    if (CARRY) to[key * a.values + value] = state[m][n][i];
                    else to[rh * a.keys * a.values + key * a.state_key + value * a.state_value] = cut ? 0.0f : state[m][n][i];
                }
    }
}

// The states that the segments leave become those before them, one behind the other: a thread per element.
static __global__ __launch_bounds__(256) void tabx_attention_join_kernel(const AttentionArgs a)
{
    const int64_t size = (int64_t)a.keys * a.values, all = a.rows * a.heads * size;
    for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x; at < all; at += (int64_t)gridDim.x * 256) {
        const int64_t rh = at / size, d = at % size;
        if (a.controlled && a.controlled[rh / a.heads] == 0) continue;
        float s = a.state_in ? a.state_in[rh * size + d / a.values * a.state_key + d % a.values * a.state_value] : 0.0f;
        for (int n = 0; n < a.segments; ++n) {
            float *const here = a.carried + (rh * a.segments + n) * size + d;
            const float left = *here, kept = a.kept[rh * a.segments + n];
            *here = s;
            s = kept < 0.0f ? left : fmaf(kept, s, left);
        }
    }
}

} // namespace tabx
