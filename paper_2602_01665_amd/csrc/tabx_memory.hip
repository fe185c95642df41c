// A unit's memory for MI355X (gfx950): norm of the residual stream, rotation by tick and place, linear attention with a
// decay for each head over an episode's ticks, and their gradients.
//
// Files: tabx_rows.h (element types, sums over lanes), tabx_teams.h (rows in registers), tabx_rms.h, tabx_rotary.h,
// tabx_attention.h (the kernels), tabx_host.h (argument checks, launches), this file (the C entry points).  Arithmetic is
// float32 (float64 for angles).
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "tabx.h"

#pragma clang fp contract(off)

#include "tabx_attention.h"
#include "tabx_host.h"
#include "tabx_rms.h"
#include "tabx_rotary.h"

namespace tabx {

// --- root-mean-square norm ----------------------------------------------------------------------

// Teams that share the rows of a forward call, if they are many (327680 rows of 512: 118 us, 134 with 8192), turns of a team's
// run of rows in a backward call (42517 rows of 1000: 88 us, 105 with 32), and of how many workgroups one takes the rows
// alone in a backward call, whose sums are then the gradient (32 rows of 1000: 9.5 us, 12.2 with two and a joining launch; 96
// rows 17.3 alone, 12.6 with six).
constexpr int64_t kRmsTeams = 10 * 8192;
constexpr int64_t kRmsTurns = 4;
constexpr int64_t kRmsAlone = 2;

// Whether the pieces of a row that sixteen lanes store lie across lines.
static bool across_lines(const void *data, int64_t stride, int type)
{
    return data && type != TABX_F32 && !(on_boundary(data, 64) && stride * size_of(type) % 64 == 0);
}

template <int LANES, int PIECES>
struct RmsForward {
    static constexpr bool kUsed = LANES > 32 || PIECES < 3;
    template <int X_BYTES>
    static int with_type(const RmsArgs &a, int64_t groups, void *stream)
    {
        return launch(!a.residual                     ? tabx_rms_kernel<LANES, PIECES, X_BYTES, 0>
                      : size_of(a.residual_type) == 4 ? tabx_rms_kernel<LANES, PIECES, X_BYTES, 4>
                                                      : tabx_rms_kernel<LANES, PIECES, X_BYTES, 2>,
                      groups, threads_of(LANES), a, stream);
    }
    static int go(RmsArgs a, void *stream)
    {
        constexpr int teams = teams_of(LANES);
        constexpr bool stays = LANES * PIECES > 768;
        a.team_rows = LANES <= 64 ? least(quotient_up(quotient_up(a.rows, kRmsTeams), at_once(LANES)) * at_once(LANES), 64) : 1;
        const int64_t groups = least(quotient_up(a.rows, a.team_rows * teams), stays ? kComputeUnits * 2048 / LANES : kMostGroups);
        a.lap = groups * teams * a.team_rows;
        // what the L2s would not hold goes past them (327680 rows of 512, half of them, bf16 and e4m3, 118 us, 112; all of
        // them in bf16 234, 225), but for pieces of lines, as in the layer norm
        const bool across = LANES == 16 && PIECES > 1 && (across_lines(a.sum, a.sum_stride, a.sum_type) || across_lines(a.y, a.y_stride, a.y_type));
        const int64_t written = a.rows * a.width * ((a.sum ? size_of(a.sum_type) : 0) + size_of(a.y_type));
        a.stream = !across && written > kL2Bytes;
        return a.x_type == TABX_F32 ? with_type<4>(a, groups, stream) : with_type<2>(a, groups, stream);
    }
};

template <int LANES, int PIECES>
struct RmsGroups {
    static constexpr bool kUsed = LANES > 32 || PIECES < 3;
    static int go(int64_t rows)
    {
        constexpr int64_t most = kComputeUnits * 4 * grad_wavefronts(PIECES) * 64 / threads_of(LANES);
        const int64_t groups = quotient_up(rows, kRmsTurns * at_once(LANES) * teams_of(LANES));
        return (int)(groups <= kRmsAlone ? 1 : least(groups, most));
    }
};

static int rms_groups(int64_t rows, int32_t width) { return for_width<RmsGroups>((width + 3) / 4, rows); }

template <int LANES, int PIECES>
struct RmsBackward {
    static constexpr bool kUsed = RmsGroups<LANES, PIECES>::kUsed;
    template <int X_BYTES, int G_BYTES>
    static int with_types(const RmsArgs &a, int64_t groups, void *stream)
    {
        return launch(!a.y          ? tabx_rms_grad_kernel<LANES, PIECES, X_BYTES, G_BYTES, false, false>
                      : a.grad_sum  ? tabx_rms_grad_kernel<LANES, PIECES, X_BYTES, G_BYTES, true, true>
                                    : tabx_rms_grad_kernel<LANES, PIECES, X_BYTES, G_BYTES, true, false>,
                      groups, threads_of(LANES), a, stream);
    }
    static int go(RmsArgs a, int64_t groups, void *stream)
    {
        constexpr int turns_at_once = at_once(LANES);
        a.team_rows = least(quotient_up(quotient_up(a.rows, groups * teams_of(LANES)), turns_at_once), kRmsTurns) * turns_at_once;
        a.team_rows = least(a.team_rows, 64);
        a.lap = groups * teams_of(LANES) * a.team_rows;
        if (a.x_type == TABX_F32) return a.g_type == TABX_F32 ? with_types<4, 4>(a, groups, stream) : with_types<4, 2>(a, groups, stream);
        return a.g_type == TABX_F32 ? with_types<2, 4>(a, groups, stream) : with_types<2, 2>(a, groups, stream);
    }
};

// Adds up the workgroups' parts: 32 columns per workgroup, 32 runs of parts side by side, always in the same order.
static __global__ __launch_bounds__(1024) void tabx_rms_join_kernel(const float *partial, int parts, int width, float *grad_weight)
{
    __shared__ float meet[32][33];
    const int c = (int)threadIdx.x & 31, run = (int)threadIdx.x >> 5;
    const int j = (int)blockIdx.x * 32 + c;
    float s = 0.0f;
    if (j < width) {
#pragma unroll 8
        for (int k = run; k < parts; k += 32) s += partial[(int64_t)k * width + j];
    }
    meet[run][c] = s;
    __syncthreads();
    if (run != 0 || j >= width) return;
#pragma unroll
    for (int k = 1; k < 32; ++k) s += meet[k][c];
    grad_weight[j] = s;
}

static int rms_join(const float *partial, int parts, int width, float *grad_weight, void *stream)
{
    void *args[] = {(void *)&partial, (void *)&parts, (void *)&width, (void *)&grad_weight};
    return launched(hipLaunchKernel((const void *)tabx_rms_join_kernel, dim3((unsigned)(width + 31) / 32), dim3(1024), args, 0,
                                    (hipStream_t)stream));
}

static int rms_backward(RmsArgs a, float *grad_weight, void *stream)
{
    const int64_t groups = rms_groups(a.rows, a.width);
    if (groups == 1) {                             // its sums are the gradient
        a.partial = nullptr;
        a.grad_weight = grad_weight;
    }
    const int rc = for_width<RmsBackward>((a.width + 3) / 4, a, groups, stream);
    return rc != TABX_OK || !a.partial ? rc : rms_join(a.partial, (int)groups, a.width, grad_weight, stream);
}

// --- heads --------------------------------------------------------------------------------------

// An array of heads; with `apart`, no two of its elements may share their place.
static int check_heads(const TabxHeads *m, int64_t ticks, int64_t rows, int32_t heads, int32_t width, bool apart)
{
    if (!m) return TABX_ERR_NULL;
    if (m->type < TABX_F32 || m->type > TABX_F16) return TABX_ERR_SHAPE;
    const int64_t count[3] = {ticks, rows, heads}, stride[3] = {m->tick_stride, m->row_stride, m->head_stride};
    int64_t reach = width;
    for (int k = 0; k < 3; ++k) {
        if (count[k] <= 1) continue;
        if (stride[k] < 0 || stride[k] > ((int64_t)1 << 60) / count[k]) return TABX_ERR_SHAPE;
        reach += stride[k] * (count[k] - 1);
    }
    if (reach > (int64_t)1 << 60) return TABX_ERR_SHAPE;
    if (apart) {
        // from the smallest stride on, each one passes over what lies below it
        int64_t span = width;
        bool done[3] = {count[0] <= 1, count[1] <= 1, count[2] <= 1};
        for (int turn = 0; turn < 3; ++turn) {
            int k = -1;
            for (int n = 0; n < 3; ++n)
                if (!done[n] && (k < 0 || stride[n] < stride[k])) k = n;
            if (k < 0) break;
            if (stride[k] < span) return TABX_ERR_SHAPE;
            span += stride[k] * (count[k] - 1);
            done[k] = true;
        }
    }
    if (!m->data) return TABX_ERR_NULL;
    return on_boundary(m->data, m->type == TABX_F32 ? 4 : 2) ? TABX_OK : TABX_ERR_ALIGN;
}

static int check_units(int64_t rows, int32_t units) { return units < 1 || rows % units != 0 ? TABX_ERR_SHAPE : TABX_OK; }

static Strides strides_of(const TabxHeads &m) { return Strides{m.tick_stride, m.row_stride, m.head_stride}; }

// --- rotation -----------------------------------------------------------------------------------

// at / divisor as the upper half of at x magic, for both below 2^16.
static uint32_t magic_of(int64_t divisor, int64_t most) { return divisor >= 2 && divisor < 65536 && most < 65536 ? (uint32_t)(((int64_t)1 << 32) / divisor + 1) : 0; }

template <int TYPE, int PAIRS, bool FAR>
static int launch_rotary(const RotaryArgs &a, bool interleaved, void *stream)
{
    const int64_t groups = least(quotient_up(a.rows, a.group_rows), kMostGroups);
    return launch(interleaved ? tabx_rotary_kernel<TYPE, PAIRS, true, FAR> : tabx_rotary_kernel<TYPE, PAIRS, false, FAR>, groups, 256, a, stream);
}

template <int TYPE, int PAIRS>
static int rotary_in_runs(RotaryArgs a, bool interleaved, bool copies, void *stream)
{
    const int64_t runs = quotient_up(a.pairs, PAIRS), slots = runs + (copies ? quotient_up(a.width - 2 * a.pairs, PAIRS) : 0);
    a.row_angles = (int32_t)(runs * PAIRS);
    const int behind = a.width - 2 * a.pairs;
    a.last_run = copies && a.pairs >= PAIRS ? a.pairs - PAIRS : INT32_MAX;
    a.last_plain = behind >= PAIRS ? behind - PAIRS : INT32_MAX;
    a.head_slots = (int32_t)slots, a.row_slots = (int32_t)(slots * a.heads);
    int64_t rows = 1024 / a.row_slots;             // four runs to a lane
    rows = least(rows < 1 ? 1 : rows, kRotaryAngles / a.row_angles);
    a.group_rows = (int32_t)rows;
    a.row_magic = magic_of(a.row_slots, rows * a.row_slots);
    a.head_magic = magic_of(a.head_slots, a.row_slots);
    a.angle_magic = magic_of(a.row_angles, rows * a.row_angles);
    const int64_t near = ((int64_t)1 << 30) - a.width;
    const bool far = a.x_row > near / rows || a.y_row > near / rows || a.x_head > near / a.heads || a.y_head > near / a.heads;
    return far ? launch_rotary<TYPE, PAIRS, true>(a, interleaved, stream) : launch_rotary<TYPE, PAIRS, false>(a, interleaved, stream);
}

static int rotary(const RotaryArgs &a, int type, bool interleaved, bool copies, void *stream)
{
    // 16 bytes of 16-bit elements (327680 rows of 8 heads of 64: 143 us, 154 with runs of four)
    const bool eight = a.pairs % 8 == 0 && a.width % 8 == 0;
    if (type == TABX_F32) return rotary_in_runs<TABX_F32, 4>(a, interleaved, copies, stream);
    if (type == TABX_BF16) return eight ? rotary_in_runs<TABX_BF16, 8>(a, interleaved, copies, stream) : rotary_in_runs<TABX_BF16, 4>(a, interleaved, copies, stream);
    return eight ? rotary_in_runs<TABX_F16, 8>(a, interleaved, copies, stream) : rotary_in_runs<TABX_F16, 4>(a, interleaved, copies, stream);
}

// --- linear attention ---------------------------------------------------------------------------

// Sizes that the calls have in common; a call of no rows is fine.
static int check_attention(int64_t ticks, int64_t rows, int32_t heads, int32_t keys, int32_t values)
{
    if (ticks < 0 || ticks > (int64_t)1 << 30 || rows < 0 || heads < 1 || heads > TABX_ATTENTION_MAX_HEADS) return TABX_ERR_SHAPE;
    if (rows > INT32_MAX / heads) return TABX_ERR_SHAPE;
    if (keys < 1 || keys > TABX_ATTENTION_MAX_WIDTH || values < 1 || values > TABX_ATTENTION_MAX_WIDTH) return TABX_ERR_SHAPE;
    return TABX_OK;
}

// Keys and values as wide as the kernels' forms take them.
static int form_width(int32_t keys, int32_t values)
{
    const int width = keys > values ? keys : values;
    return width <= 32 ? 32 : width <= 64 ? 64 : width <= 96 ? 96 : 128;
}

// Into how many segments of how many ticks a row's ticks are cut: where there are few rows and heads, so many that every
// CU has the workgroups that it holds, each of some chunks.  At least 64 ticks: 1024 ticks of 8 heads of 64 take 21 us,
// their gradients 32; with 128 at least 27 and 44, with 256 40 and 71.  Half as many workgroups: 32768 ticks of 8 heads of
// 128 197 us instead of 158, gradients of 512 ticks of 80 heads of 64 60 instead of 54 (of 8192 ticks of 16, 98 instead of 106).
struct Segments {
    int64_t count, ticks;
};
constexpr int64_t kSegmentTicks = 64;              // at least; a multiple of every chunk

static Segments segments_of(int64_t ticks, int64_t rows, int32_t heads, int32_t keys, int32_t values)
{
    const int64_t works = rows * heads, wanted = kComputeUnits * (256 / form_width(keys, values));
    const int64_t most = works > 0 && works < wanted ? wanted / works : 1;
    int64_t length = quotient_up(quotient_up(ticks, most), kSegmentTicks) * kSegmentTicks;
    if (length < kSegmentTicks) length = kSegmentTicks;
    const int64_t count = quotient_up(ticks, length);
    return Segments{count < 1 ? 1 : count, length};
}

// Of the states before each segment, and behind them what each leaves of the one before: once for the way forth, twice for
// the way back.
static int64_t carried_bytes(const Segments &s, int64_t rows, int32_t heads, int32_t keys, int32_t values)
{
    return s.count == 1 ? 0 : quotient_up(rows * heads * s.count * ((int64_t)keys * values + 1) * (int64_t)sizeof(float), 16) * 16;
}

static int64_t attention_workspace(int64_t ticks, int64_t rows, int32_t heads, int32_t keys, int32_t values)
{
    return 2 * carried_bytes(segments_of(ticks, rows, heads, keys, values), rows, heads, keys, values);
}

// One or two attentions of the same sizes.
static int launch_pair(void (*kernel)(AttentionPair), int64_t groups, int threads, const AttentionPair &pair, int count, void *stream)
{
    void *args[] = {(void *)&pair};
    return launched(hipLaunchKernel((const void *)kernel, dim3((unsigned)groups, (unsigned)count), dim3((unsigned)threads), args, 0, (hipStream_t)stream));
}

template <bool CARRY, int D, int TYPE>
static int launch_attention_of(const AttentionPair &pair, int count, void *stream)
{
    constexpr int chunk = long_chunk(D, TYPE, !CARRY);
    const int64_t groups = least(pair.of[0].works, kMostGroups);
    if constexpr (chunk > 32 && !CARRY)            // (no segments are that short)
        // (8 ticks of 81920 heads of 96 1590 us, 1720 in a chunk of 64, half empty; of 128 2177 and 2142, 16 of 40960 1204 and 1197)
        if (pair.of[0].ticks <= 32) return launch_pair(tabx_attention_kernel<D, TYPE, 32, CARRY>, groups, 4 * D, pair, count, stream);
    return launch_pair(tabx_attention_kernel<D, TYPE, chunk, CARRY>, groups, 4 * D, pair, count, stream);
}

template <bool CARRY, int D>
static int launch_attention(const AttentionPair &pair, int count, int type, void *stream)
{
    if (type == TABX_F32) return launch_attention_of<CARRY, D, TABX_F32>(pair, count, stream);
    return type == TABX_BF16 ? launch_attention_of<CARRY, D, TABX_BF16>(pair, count, stream) : launch_attention_of<CARRY, D, TABX_F16>(pair, count, stream);
}

template <bool CARRY>
static int attention_of_width(const AttentionPair &pair, int count, int type, void *stream)
{
    const int width = form_width(pair.of[0].keys, pair.of[0].values);
    if (width == 32) return launch_attention<CARRY, 32>(pair, count, type, stream);
    if (width == 64) return launch_attention<CARRY, 64>(pair, count, type, stream);
    if (width == 96) return launch_attention<CARRY, 96>(pair, count, type, stream);
    return launch_attention<CARRY, 128>(pair, count, type, stream);
}

// The states before each segment of one or two attentions, each into its part of the workspace.
static int carry(AttentionPair &pair, int count, int type, void *workspace, int64_t bytes, void *stream)
{
    for (int n = 0; n < count; ++n) {
        AttentionArgs &a = pair.of[n];
        a.carried = (float *)((char *)workspace + n * bytes);
        a.kept = a.carried + a.works * a.keys * a.values;
    }
    const int rc = attention_of_width<true>(pair, count, type, stream);
    if (rc) return rc;
    const AttentionArgs &a = pair.of[0];
    return launch_pair(tabx_attention_join_kernel, least(quotient_up(a.rows * a.heads * a.keys * a.values, 256), kMostGroups), 256, pair, count, stream);
}

// 16-bit operands of up to 64: one workgroup for all three gradients, which reads everything once where three would twice
// (64 ticks of 20480 heads of 64 675 us, 783 apart; 128 ticks of 40960 heads of 32 1021 and 1114).  Wider or in three parts its
// two states and four tiles cost more workgroups of a CU than they spare (64 ticks of 5120 heads of 128 967 us, 775 apart, of 10240
// of 96 876 and 774; f32, 10240 heads of 64, 663 and 594; but 1887 of 48 x 80 353 and 380, where one workgroup runs either way).
template <int D, int TYPE, int C>
static int launch_attention_grad_of(const AttentionGradArgs &a, void *stream)
{
    if constexpr (D <= 64 && TYPE != TABX_F32) {
        return launch(tabx_attention_grad_kernel<D, TYPE, C>, least(a.works, kMostGroups), 4 * D, a, stream);
    } else {
        const int64_t groups = least(3 * a.works, kMostGroups);
        if (a.grad_k && a.grad_state_in && a.grad_state_in == a.grad_state_out && !a.grad_states) {
            // grad_k's workgroups read the state that grad_v's overwrite: one behind the other
            AttentionGradArgs before = a, behind = a;
            before.grad_v = nullptr, before.grad_state_in = nullptr;
            behind.grad_q = nullptr, behind.grad_k = nullptr;
            const int rc = launch(tabx_attention_grad_apart_kernel<D, TYPE, C>, groups, 4 * D, before, stream);
            return rc ? rc : launch(tabx_attention_grad_apart_kernel<D, TYPE, C>, groups, 4 * D, behind, stream);
        }
        return launch(tabx_attention_grad_apart_kernel<D, TYPE, C>, groups, 4 * D, a, stream);
    }
}

template <int D, int TYPE>
static int launch_attention_grad(const AttentionGradArgs &a, void *stream)
{
    // of up to 32 ticks, half of a longer chunk would be empty (16 ticks of 81920 heads of 64: 1542 us, 1756 in one of 64; 20480 of 128 1242 and 1308)
    constexpr int chunk = long_chunk(D, TYPE, false);
    if constexpr (chunk > 32)
        if (a.ticks <= 32) return launch_attention_grad_of<D, TYPE, 32>(a, stream);
    return launch_attention_grad_of<D, TYPE, chunk>(a, stream);
}

template <int D>
static int attention_grad_of_type(const AttentionGradArgs &a, int type, void *stream)
{
    return type == TABX_F32 ? launch_attention_grad<D, TABX_F32>(a, stream) : type == TABX_BF16 ? launch_attention_grad<D, TABX_BF16>(a, stream)
                                                                                                : launch_attention_grad<D, TABX_F16>(a, stream);
}

// Values that are no multiple of four: a lane has one of them.
template <int TYPE, int ACROSS>
static int launch_step_odd(const StepArgs &a, void *stream)
{
    return launch(tabx_attention_step_odd_kernel<TYPE, ACROSS>, least(quotient_up(a.works, 4), kMostGroups), 256, a, stream);
}

template <int TYPE, int VALUES, int LANES>
static int launch_step(const StepArgs &a, void *stream)
{
    return launch(tabx_attention_step_kernel<TYPE, VALUES, LANES>, least(quotient_up(a.works, 256 / LANES), kMostGroups), 256, a, stream);
}

// States of few elements share a wavefront (2621440 of 16 x 16: 1063 us, 2645 with a wavefront each).
template <int TYPE>
static int attention_step(const StepArgs &a, void *stream)
{
    if (a.values % 4 != 0) {
        if (a.values <= 8) return launch_step_odd<TYPE, 8>(a, stream);
        if (a.values <= 16) return launch_step_odd<TYPE, 16>(a, stream);
        return a.values <= 32 ? launch_step_odd<TYPE, 32>(a, stream) : launch_step_odd<TYPE, 64>(a, stream);
    }
    if (a.values <= 4) return a.keys <= 16 ? launch_step<TYPE, 4, 8>(a, stream) : launch_step<TYPE, 4, 64>(a, stream);
    if (a.values <= 8) return a.keys <= 16 ? launch_step<TYPE, 8, 16>(a, stream) : launch_step<TYPE, 8, 64>(a, stream);
    if (a.values <= 16) return a.keys <= 32 ? launch_step<TYPE, 16, 16>(a, stream) : launch_step<TYPE, 16, 64>(a, stream);
    if (a.values <= 32) return launch_step<TYPE, 32, 64>(a, stream);
    if (a.values <= 64) return launch_step<TYPE, 64, 64>(a, stream);
    return launch_step<TYPE, 128, 64>(a, stream);
}

static int check_workspace(const void *workspace, int64_t bytes, int64_t needed)
{
    if (needed == 0) return TABX_OK;
    if (!workspace) return TABX_ERR_NULL;
    if (!on_boundary(workspace, 16)) return TABX_ERR_ALIGN;
    return bytes < needed ? TABX_ERR_SHAPE : TABX_OK;
}

// q, k and v of one type, and one that is written or read beside them.
static int check_inputs(int64_t ticks, int64_t rows, int32_t heads, int32_t keys, int32_t values, const TabxHeads *q,
                        const TabxHeads *k, const TabxHeads *v, const TabxHeads *out, bool written)
{
    int rc;
    if ((rc = check_heads(q, ticks, rows, heads, keys, false)) || (rc = check_heads(k, ticks, rows, heads, keys, false))) return rc;
    if ((rc = check_heads(v, ticks, rows, heads, values, false)) || (rc = check_heads(out, ticks, rows, heads, values, written))) return rc;
    return q->type == k->type && q->type == v->type && q->type == out->type ? TABX_OK : TABX_ERR_SHAPE;
}

} // namespace tabx

extern "C" {

int tabx_rms_norm(int64_t rows, int32_t width, const TabxRows *x, const TabxRows *residual, const uint8_t *row_mask,
                  const float *weight, float eps, const TabxRows *sum, const TabxRows *y, float *scale, float *rstd, void *stream)
{
    using namespace tabx;
    int rc = check_rows(rows, width);
    if (rc) return rc;
    if (width > TABX_NORM_MAX_WIDTH) return TABX_ERR_SHAPE;
    if (!(eps >= 0.0f && eps < INFINITY)) return TABX_ERR_PARAM;
    if (rows == 0) return TABX_OK;
    if ((rc = check_array(x, rows, width)) || (rc = check_array(residual, rows, width, true))) return rc;
    if ((rc = check_array(sum, rows, width, true)) || (rc = check_array(y, rows, width, false, TABX_E4M3))) return rc;
    if ((rc = check_floats(weight, true)) || (rc = check_floats(scale, y->type != TABX_E4M3)) || (rc = check_floats(rstd, true))) return rc;
    if (scale && y->type != TABX_E4M3) return TABX_ERR_SHAPE;
    RmsArgs a = {};
    a.x = x->data, a.x_stride = x->stride, a.x_type = x->type;
    if (residual) a.residual = residual->data, a.residual_stride = residual->stride, a.residual_type = residual->type;
    if (sum) a.sum = sum->data, a.sum_stride = sum->stride, a.sum_type = sum->type;
    a.y = y->data, a.y_stride = y->stride, a.y_type = y->type;
    a.row_mask = row_mask;
    a.weight = weight, a.scale = scale, a.rstd = rstd;
    a.rows = rows, a.width = width, a.eps = eps, a.inv_width = 1.0f / (float)width;
    return for_width<RmsForward>((width + 3) / 4, a, stream);
}

int64_t tabx_rms_norm_workspace(int64_t rows, int32_t width)
{
    const int rc = tabx::check_rows(rows, width);
    if (rc || width > TABX_NORM_MAX_WIDTH) return TABX_ERR_SHAPE;
    return (int64_t)tabx::rms_groups(rows, width) * width * (int64_t)sizeof(float);
}

int tabx_rms_norm_backward(int64_t rows, int32_t width, const TabxRows *sum, const uint8_t *row_mask, const float *weight,
                           const float *rstd, const TabxRows *grad_y, const TabxRows *grad_sum, const TabxRows *grad_x,
                           float *grad_weight, void *workspace, int64_t workspace_bytes, void *stream)
{
    using namespace tabx;
    int rc = check_rows(rows, width);
    if (rc) return rc;
    if (width > TABX_NORM_MAX_WIDTH) return TABX_ERR_SHAPE;
    if (rows == 0) {                               // sums over no rows
        if ((rc = check_floats(grad_weight, true))) return rc;
        return grad_weight ? rms_join(nullptr, 0, width, grad_weight, stream) : TABX_OK;
    }
    if ((rc = check_array(sum, rows, width)) || (rc = check_array(grad_y, rows, width))) return rc;
    if ((rc = check_array(grad_sum, rows, width, true)) || (rc = check_array(grad_x, rows, width, true))) return rc;
    if (grad_sum && grad_sum->type != sum->type) return TABX_ERR_SHAPE;
    if ((rc = check_floats(weight, true)) || (rc = check_floats(rstd, false)) || (rc = check_floats(grad_weight, true))) return rc;
    if (!grad_weight && !grad_x) return TABX_ERR_NULL;
    if (grad_weight && (rc = check_workspace(workspace, workspace_bytes, tabx_rms_norm_workspace(rows, width)))) return rc;
    RmsArgs a = {};
    a.x = sum->data, a.x_stride = sum->stride, a.x_type = sum->type;
    a.grad_y = grad_y->data, a.g_stride = grad_y->stride, a.g_type = grad_y->type;
    if (grad_sum) a.grad_sum = grad_sum->data, a.grad_sum_stride = grad_sum->stride;
    if (grad_x) a.y = grad_x->data, a.y_stride = grad_x->stride, a.y_type = grad_x->type;
    a.row_mask = row_mask;
    a.weight = weight, a.rstd = (float *)rstd;
    a.partial = grad_weight ? (float *)workspace : nullptr;
    a.rows = rows, a.width = width, a.inv_width = 1.0f / (float)width;
    return rms_backward(a, grad_weight, stream);
}

int tabx_rotary(int64_t rows, int32_t heads, int32_t width, const TabxHeads *x, const uint8_t *row_mask, const TabxAxis *axes,
                int32_t num_axes, const double *frequency, int32_t interleaved, int32_t inverse, const TabxHeads *y, void *stream)
{
    using namespace tabx;
    if (rows < 0 || rows > (int64_t)1 << 40 || heads < 1 || width < 2 || width > TABX_ROTARY_MAX_WIDTH) return TABX_ERR_SHAPE;
    if (heads > (1 << 30) / width) return TABX_ERR_SHAPE;
    if (num_axes < 1 || num_axes > TABX_ROTARY_MAX_AXES) return TABX_ERR_SHAPE;
    if (!axes) return TABX_ERR_NULL;
    RotaryArgs a = {};
    for (int n = 0; n < num_axes; ++n) {
        if (axes[n].pairs < 0 || axes[n].pairs > width / 2 - a.pairs) return TABX_ERR_SHAPE;
        if (axes[n].type != TABX_F32 && axes[n].type != TABX_I32) return TABX_ERR_SHAPE;
        if (check_units(rows, axes[n].units)) return TABX_ERR_SHAPE;
        a.pairs += axes[n].pairs;
        a.end[n] = a.pairs;
        a.units[n] = axes[n].units;
        a.axis_type[n] = axes[n].type;
        a.position[n] = axes[n].position;
    }
    if (a.pairs < 1) return TABX_ERR_SHAPE;
    if (rows == 0) return TABX_OK;
    int rc;
    for (int n = 0; n < num_axes; ++n)
        if ((rc = check_floats(axes[n].position, false))) return rc;
    if ((rc = check_heads(x, 1, rows, heads, width, false)) || (rc = check_heads(y, 1, rows, heads, width, true))) return rc;
    if (x->type != y->type) return TABX_ERR_SHAPE;
    if (x->data == y->data && (x->row_stride != y->row_stride || x->head_stride != y->head_stride)) return TABX_ERR_SHAPE;
    if (!frequency) return TABX_ERR_NULL;
    if (!on_boundary(frequency, 8)) return TABX_ERR_ALIGN;
    a.x = x->data, a.x_row = x->row_stride, a.x_head = x->head_stride;
    a.y = y->data, a.y_row = y->row_stride, a.y_head = y->head_stride;
    a.row_mask = row_mask;
    a.frequency = frequency;
    a.rows = rows, a.heads = heads, a.width = width;
    a.num_axes = num_axes, a.sign = (inverse ? -1.0 : 1.0) * 0.63661977236758134;
    return rotary(a, x->type, interleaved != 0, x->data != y->data, stream);
}

int tabx_linear_attention_step(int64_t rows, int32_t heads, int32_t key_width, int32_t value_width, const TabxHeads *q,
                               const TabxHeads *k, const TabxHeads *v, const float *log_decay, float scale, const uint8_t *fresh,
                               int32_t units, const uint8_t *controlled, float *state, const TabxHeads *out, void *stream)
{
    using namespace tabx;
    int rc = check_attention(1, rows, heads, key_width, value_width);
    if (rc || (rc = check_units(rows, units))) return rc;
    if (!(fabsf(scale) < INFINITY)) return TABX_ERR_PARAM;
    if (rows == 0) return TABX_OK;
    if ((rc = check_inputs(1, rows, heads, key_width, value_width, q, k, v, out, true))) return rc;
    if ((rc = check_floats(log_decay, false)) || (rc = check_floats(state, false))) return rc;
    StepArgs a = {};
    a.q = q->data, a.k = k->data, a.v = v->data, a.out = out->data;
    a.qs = strides_of(*q), a.ks = strides_of(*k), a.vs = strides_of(*v), a.os = strides_of(*out);
    a.log_decay = log_decay, a.fresh = fresh, a.controlled = controlled;
    a.state = state;
    a.works = rows * heads, a.heads = heads, a.units = units, a.keys = key_width, a.values = value_width;
    a.scale = scale;
    return q->type == TABX_F32 ? attention_step<TABX_F32>(a, stream) : q->type == TABX_BF16 ? attention_step<TABX_BF16>(a, stream) : attention_step<TABX_F16>(a, stream);
}

int64_t tabx_linear_attention_workspace(int64_t ticks, int64_t rows, int32_t heads, int32_t key_width, int32_t value_width)
{
    const int rc = tabx::check_attention(ticks, rows, heads, key_width, value_width);
    return rc ? rc : tabx::attention_workspace(ticks, rows, heads, key_width, value_width);
}

int tabx_linear_attention(int64_t ticks, int64_t rows, int32_t heads, int32_t key_width, int32_t value_width, const TabxHeads *q,
                          const TabxHeads *k, const TabxHeads *v, const float *log_decay, float scale, const uint8_t *fresh,
                          int32_t units, const uint8_t *controlled, const float *state_in, float *state_out, const TabxHeads *out,
                          void *workspace, int64_t workspace_bytes, void *stream)
{
    using namespace tabx;
    int rc = check_attention(ticks, rows, heads, key_width, value_width);
    if (rc || (rc = check_units(rows, units))) return rc;
    if (!(fabsf(scale) < INFINITY)) return TABX_ERR_PARAM;
    if (rows == 0 || (ticks == 0 && !state_out)) return TABX_OK;
    if (ticks > 0 && (rc = check_inputs(ticks, rows, heads, key_width, value_width, q, k, v, out, true))) return rc;
    if ((rc = check_floats(log_decay, false)) || (rc = check_floats(state_in, true)) || (rc = check_floats(state_out, true))) return rc;
    if ((rc = check_workspace(workspace, workspace_bytes, attention_workspace(ticks, rows, heads, key_width, value_width)))) return rc;
    const Segments s = segments_of(ticks, rows, heads, key_width, value_width);
    AttentionArgs a = {};
    int type = TABX_F32;
    if (ticks > 0) {
        a.q = q->data, a.k = k->data, a.v = v->data, a.out = out->data;
        a.qs = strides_of(*q), a.ks = strides_of(*k), a.vs = strides_of(*v), a.os = strides_of(*out);
        type = q->type;
    }
    a.log_decay = log_decay, a.fresh = fresh, a.controlled = controlled;
    a.state_in = state_in, a.state_out = state_out;
    a.ticks = ticks, a.rows = rows, a.envs = rows / units, a.works = rows * heads * s.count, a.segment = s.ticks;
    a.segments = (int32_t)s.count, a.heads = heads, a.units = units, a.keys = key_width, a.values = value_width;
    a.exactly = !(fabsf(scale) <= kMostScale), a.scale_read = scale, a.scale_added = 1.0f;
    AttentionPair pair = {{a}};
    if (s.count > 1 && (rc = carry(pair, 1, type, workspace, 0, stream))) return rc;
    return attention_of_width<false>(pair, 1, type, stream);
}

int tabx_linear_attention_backward(int64_t ticks, int64_t rows, int32_t heads, int32_t key_width, int32_t value_width,
                                   const TabxHeads *q, const TabxHeads *k, const TabxHeads *v, const float *log_decay, float scale,
                                   const uint8_t *fresh, int32_t units, const uint8_t *controlled, const float *state_in,
                                   const float *grad_state_out, const TabxHeads *grad_out, const TabxHeads *grad_q,
                                   const TabxHeads *grad_k, const TabxHeads *grad_v, float *grad_state_in, void *workspace,
                                   int64_t workspace_bytes, void *stream)
{
    using namespace tabx;
    int rc = check_attention(ticks, rows, heads, key_width, value_width);
    if (rc || (rc = check_units(rows, units))) return rc;
    if (!(fabsf(scale) < INFINITY)) return TABX_ERR_PARAM;
    if (!grad_q && !grad_k && !grad_v && !grad_state_in) return TABX_ERR_NULL;
    if (rows == 0 || (ticks == 0 && !grad_state_in)) return TABX_OK;
    if (ticks > 0) {
        if ((rc = check_inputs(ticks, rows, heads, key_width, value_width, q, k, v, grad_out, false))) return rc;
        const TabxHeads *const written[3] = {grad_q, grad_k, grad_v};
        for (int n = 0; n < 3; ++n) {
            if (!written[n]) continue;
            if ((rc = check_heads(written[n], ticks, rows, heads, n < 2 ? key_width : value_width, true))) return rc;
            if (written[n]->type != q->type) return TABX_ERR_SHAPE;
        }
    }
    if ((rc = check_floats(log_decay, false)) || (rc = check_floats(state_in, true)) || (rc = check_floats(grad_state_out, true)) ||
        (rc = check_floats(grad_state_in, true)))
        return rc;
    if ((rc = check_workspace(workspace, workspace_bytes, attention_workspace(ticks, rows, heads, key_width, value_width)))) return rc;
    const Segments s = segments_of(ticks, rows, heads, key_width, value_width);
    AttentionGradArgs a = {};
    int type = TABX_F32;
    if (ticks > 0) {
        a.q = q->data, a.k = k->data, a.v = v->data, a.grad_out = grad_out->data;
        a.qs = strides_of(*q), a.ks = strides_of(*k), a.vs = strides_of(*v), a.os = strides_of(*grad_out);
        if (grad_q) a.grad_q = grad_q->data, a.gqs = strides_of(*grad_q);
        if (grad_k) a.grad_k = grad_k->data, a.gks = strides_of(*grad_k);
        if (grad_v) a.grad_v = grad_v->data, a.gvs = strides_of(*grad_v);
        type = q->type;
    }
    a.log_decay = log_decay, a.fresh = fresh, a.controlled = controlled;
    a.state_in = state_in, a.grad_state_out = grad_state_out, a.grad_state_in = grad_state_in;
    a.ticks = ticks, a.rows = rows, a.envs = rows / units, a.works = rows * heads * s.count, a.segment = s.ticks;
    a.segments = (int32_t)s.count, a.heads = heads, a.units = units, a.keys = key_width, a.values = value_width;
    a.exactly = !(fabsf(scale) <= kMostScale), a.scale = scale;
    if (s.count > 1) {
        AttentionArgs c = {};
        c.log_decay = log_decay, c.fresh = fresh, c.controlled = controlled;
        c.ticks = a.ticks, c.rows = a.rows, c.envs = a.envs, c.works = a.works, c.segment = a.segment;
        c.segments = a.segments, c.heads = heads, c.units = units, c.keys = key_width, c.values = value_width;
        AttentionPair pair = {};
        int count = 0;
        if (grad_q) {
            c.k = a.k, c.v = a.v, c.ks = a.ks, c.vs = a.vs;
            c.state_in = state_in, c.scale_added = 1.0f;
            pair.of[count++] = c;
        }
        if (grad_k || grad_v || grad_state_in) {
            c.k = a.q, c.v = a.grad_out, c.ks = a.qs, c.vs = a.os;
            c.state_in = grad_state_out, c.scale_added = scale, c.exactly = a.exactly, c.backward = 1;
            pair.of[count++] = c;
        }
        if ((rc = carry(pair, count, type, workspace, carried_bytes(s, rows, heads, key_width, value_width), stream))) return rc;
        if (grad_q) a.states = pair.of[0].carried;
        a.grad_states = pair.of[count - 1].carried;            // (not looked at where only grad_q is wanted)
    }
    const int width = form_width(key_width, value_width);
    if (width == 32) return attention_grad_of_type<32>(a, type, stream);
    if (width == 64) return attention_grad_of_type<64>(a, type, stream);
    if (width == 96) return attention_grad_of_type<96>(a, type, stream);
    return attention_grad_of_type<128>(a, type, stream);
}

} // extern "C"
