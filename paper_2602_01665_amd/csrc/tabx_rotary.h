// Rotation of pairs of a head's elements by angles that grow along several axes.
#pragma once
#include <type_traits>

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
    int32_t     group_rows, row_angles;               // rows of a workgroup; angles of a row in LDS, whole runs
    int32_t     row_slots, head_slots;                // runs of pairs or copied elements of a row, of a head
    int32_t     last_run, last_plain;                 // where the last runs of a head start at the latest
    uint32_t    row_magic, head_magic, angle_magic;   // 2^32 / row_slots, head_slots, angles of a row, rounded up; 0: divide
    double      sign;              // of the angles, times the quarter turns of a radian
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

// N elements as they lie in memory, from `at` on, wherever that lies, and in 32 bits.
template <int TYPE, int N>
struct Run {
    typedef typename Element<TYPE>::one T;
    typedef T Raw __attribute__((ext_vector_type(N)));
    typedef Raw Anywhere __attribute__((aligned(sizeof(T))));
    typedef float Floats __attribute__((ext_vector_type(N)));
    Raw v;
    __device__ __forceinline__ void load(const T *at) { v = *(const Anywhere *)at; }
    __device__ __forceinline__ void load_some(const T *at, int step, int count)
    {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = i < count ? at[i * step] : (T)0.0f;
    }
    __device__ __forceinline__ void store(T *at) const { *(Anywhere *)at = v; }
    __device__ __forceinline__ void store_some(T *at, int step, int count) const
    {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < count) at[i * step] = v[i];
    }
};

// Bound by HBM: 327680 rows of 8 heads of 64 in bf16, all turned, three axes, 141 us (4.8 TB/s; an angle in each lane that
// turns with it 386, single elements to a lane 166); 85051 rows of 6 heads of 40 f32, 15 pairs interleaved, 37 us (4.4 TB/s).
// A workgroup takes some rows: it works out their angles, once for all heads, and then goes through their heads in the order
// of memory, PAIRS pairs (or as many of the elements that are copied) to a lane, with the loads of the first of them under
// way meanwhile.  FAR: a workgroup's rows span more than 2^31 elements.
constexpr int kRotaryAngles = 2048;                // of a workgroup: 16 KB of LDS

template <int TYPE, int PAIRS, bool INTERLEAVED, bool FAR>
__global__ __launch_bounds__(256) void tabx_rotary_kernel(const RotaryArgs a)
{
    typedef typename Element<TYPE>::one T;
    typedef Run<TYPE, PAIRS> R;
    typedef typename R::Floats F;
    typedef std::conditional_t<FAR, int64_t, int32_t> Offset;
    constexpr int AHEAD = 4;
    __shared__ float cosines[kRotaryAngles], sines[kRotaryAngles];
    const int turned = a.row_angles / PAIRS, behind = a.width - 2 * a.pairs;
    for (int64_t base = (int64_t)blockIdx.x * a.group_rows; base < a.rows; base += (int64_t)gridDim.x * a.group_rows) {
        const int rows = (int)min((int64_t)a.group_rows, a.rows - base);
        const int units = rows * a.row_slots;
        const T *const x = (const T *)a.x + base * a.x_row;
        T *const y = (T *)a.y + base * a.y_row;
        struct Unit {
            R u, v;
            Offset to;             // of its first element in y
            int angle, count;      // count: of its pairs, or less than 0: of its copied elements; 0: none
        } unit[AHEAD];
        const auto fetch = [&](Unit &n, int at) {
            n.count = 0;
            if (at >= units) return;
            const int row = a.row_magic ? (int)__umulhi((uint32_t)at, a.row_magic) : at / a.row_slots;
            const int rest = at - row * a.row_slots;
            const int head = a.head_magic ? (int)__umulhi((uint32_t)rest, a.head_magic) : rest / a.head_slots;
            const int slot = rest - head * a.head_slots;
            if (a.row_mask && a.row_mask[base + row] == 0) return;
            const bool turns = slot < turned;
            // what is left of a head beyond whole runs is taken with what lies before it once more, where that is not
            // overwritten meanwhile
            const int pair = min(PAIRS * slot, a.last_run), plain = min(PAIRS * (slot - turned), a.last_plain);
            const int first = turns ? (INTERLEAVED ? 2 : 1) * pair : 2 * a.pairs + plain;
            const T *const from = x + ((Offset)row * (Offset)a.x_row + (Offset)head * (Offset)a.x_head + first);
            n.to = (Offset)row * (Offset)a.y_row + (Offset)head * (Offset)a.y_head + first;
            n.angle = row * a.row_angles + pair;
            if (turns) {
                n.count = min(PAIRS, a.pairs - pair);
                if (n.count == PAIRS) {            // (interleaved: the pairs' first half and second half)
                    n.u.load(from);
                    n.v.load(from + (INTERLEAVED ? PAIRS : a.pairs));
                } else {
                    n.u.load_some(from, INTERLEAVED ? 2 : 1, n.count);
                    n.v.load_some(from + (INTERLEAVED ? 1 : a.pairs), INTERLEAVED ? 2 : 1, n.count);
                }
            } else {
                const int some = min(PAIRS, behind - plain);
                n.count = -some;
                if (some == PAIRS) n.u.load(from);
                else n.u.load_some(from, 1, some);
            }
        };
        const auto finish = [&](Unit &n) {
            T *const to = y + n.to;
            if (n.count > 0) {
                F u = __builtin_convertvector(n.u.v, F), v = __builtin_convertvector(n.v.v, F);
                if (INTERLEAVED && n.count == PAIRS) {
                    const F s = u, t = v;
#pragma unroll
                    for (int i = 0; i < PAIRS; ++i) {
                        u[i] = 2 * i < PAIRS ? s[2 * i % PAIRS] : t[2 * i % PAIRS];
                        v[i] = 2 * i < PAIRS ? s[(2 * i + 1) % PAIRS] : t[(2 * i + 1) % PAIRS];
                    }
                }
                F first, second;
#pragma unroll
                for (int i = 0; i < PAIRS; ++i) {
                    const float c = cosines[n.angle + i], s = sines[n.angle + i];
                    first[i] = fmaf(u[i], c, -(v[i] * s));
                    second[i] = fmaf(u[i], s, v[i] * c);
                }
                if (n.count == PAIRS) {
                    if (INTERLEAVED) {
                        const F s = first, t = second;
#pragma unroll
                        for (int i = 0; i < PAIRS; ++i) {
                            first[i] = i % 2 ? t[i / 2] : s[i / 2];
                            second[i] = i % 2 ? t[(PAIRS + i) / 2] : s[(PAIRS + i) / 2];
                        }
                    }
                    n.u.v = __builtin_convertvector(first, typename R::Raw), n.v.v = __builtin_convertvector(second, typename R::Raw);
                    n.u.store(to);
                    n.v.store(to + (INTERLEAVED ? PAIRS : a.pairs));
                } else {
                    n.u.v = __builtin_convertvector(first, typename R::Raw), n.v.v = __builtin_convertvector(second, typename R::Raw);
                    n.u.store_some(to, INTERLEAVED ? 2 : 1, n.count);
                    n.v.store_some(to + (INTERLEAVED ? 1 : a.pairs), INTERLEAVED ? 2 : 1, n.count);
                }
            } else if (n.count == -PAIRS) {
                n.u.store(to);
            } else if (n.count < 0) {
                n.u.store_some(to, 1, -n.count);
            }
        };
#pragma unroll
        for (int n = 0; n < AHEAD; ++n) fetch(unit[n], (int)threadIdx.x + 256 * n);
        for (int at = threadIdx.x; at < rows * a.row_angles; at += 256) {
            const int row = a.angle_magic ? (int)__umulhi((uint32_t)at, a.angle_magic) : at / a.row_angles;
            const int pair = min(at - row * a.row_angles, a.pairs - 1);
            int axis = 0;
#pragma unroll
            for (int n = 1; n < TABX_ROTARY_MAX_AXES; ++n) axis += n < a.num_axes && pair >= a.end[n - 1];
            const void *const position = axis == 0 ? a.position[0] : axis == 1 ? a.position[1] : axis == 2 ? a.position[2] : a.position[3];
            const int units_of = axis == 0 ? a.units[0] : axis == 1 ? a.units[1] : axis == 2 ? a.units[2] : a.units[3];
            const int type = axis == 0 ? a.axis_type[0] : axis == 1 ? a.axis_type[1] : axis == 2 ? a.axis_type[2] : a.axis_type[3];
            const int64_t r = base + row;
            const int64_t where = units_of == 1 ? r : r >> 32 ? r / units_of : (int64_t)((uint32_t)r / (uint32_t)units_of);
            const uint32_t raw = ((const uint32_t *)position)[where];
            const double p = type == TABX_I32 ? (double)(int32_t)raw : (double)__uint_as_float(raw);
            quarter_turns(p * (a.frequency[pair] * a.sign), cosines[at], sines[at]);
        }
        __syncthreads();
#pragma unroll
        for (int n = 0; n < AHEAD; ++n) finish(unit[n]);
        for (int at = (int)threadIdx.x + 256 * AHEAD; at < units; at += 256) {
            fetch(unit[0], at);
            finish(unit[0]);
        }
        __syncthreads();                           // the angles have been read
    }
}

} // namespace tabx
