// The learner's side of the tick for MI355X (gfx950): layer norm of rows and its gradients, draws of actions and
// levels, log-probabilities of actions and their gradient.
//
// Files: tabx_rows.h (element types, sums over lanes), tabx_teams.h (rows in registers), tabx_norm.h, tabx_sample.h,
// tabx_levels.h (the kernels), tabx_host.h (argument checks, launches), this file (the C entry points).  Arithmetic is
// float32 (float64 where a draw is decided).
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "tabx.h"

#pragma clang fp contract(off)

#include "tabx_host.h"
#include "tabx_levels.h"
#include "tabx_norm.h"
#include "tabx_sample.h"

namespace tabx {

static bool usable_temperature(double t) { return t >= 1e-30 && t <= 1e30; }

static int check_sampling(const TabxSampling *s)
{
    if (!s) return TABX_ERR_NULL;
    if (s->temperature != 0.0 && !usable_temperature(s->temperature)) return TABX_ERR_PARAM;
    if (s->top_k < 0 || !(s->top_p > 0.0f && s->top_p <= 1.0f) || !(s->min_p >= 0.0f && s->min_p <= 1.0f)) return TABX_ERR_PARAM;
    return TABX_OK;
}

// --- layer norm ---------------------------------------------------------------------------------

constexpr int64_t kNormTeams = 10 * 8192;          // teams that share the rows of a forward call, if they are many
constexpr int64_t kGradTurns = 4;                  // turns of a team's run of rows in a backward call
constexpr int64_t kAloneGroups = 2;                // workgroups whose rows one takes alone in a backward call

// Ten times as many teams as the machine holds wavefronts: short runs go through memory in its order, but a team of one turn
// has no next rows under way.  10240, 20480, 40960, 81920, 163840, 655360 of them: 200000 rows of 700 bf16 131, 125, 118, 114,
// 115, 135 us; a million of 128 bf16 99, 102, 96, 86, 90, 115; 655360 of 160 f32 130, 126, 117, 116, 129, 129; 700000 of 96 f32,
// half of them, 47, 44, 42, 44, 47, 60.
// The widest rows' teams stay: every workgroup would load as much of weight and bias as it has rows (rows of 4096: 74 us, 63; of
// 6000: 139, 102; rows of 2144 are faster without, 250 and 261).
// What is written and is more than the L2s hold goes past them (60000 rows of 368 to bf16: 29.0 us, 22.7; 150000: 68.1, 66.4;
// f32 of any width 2 to 7 % less), but not where each store of a row is a line's length and lies across two of them: sixteen
// lanes' pieces of 16-bit results, in rows off the half lines (90 MB from bf16, past the caches or not: 66 98.8, 93.0 us, 130
// 96.1, 88.4, 186 83.1, 78.5; on them 128 64.8, 68.2, 160 74.4, 76.1, 192 65.2, 68.1).  Rows of a single piece gain and lose
// as much (56: 73.3, 78.3; 50: 85.8, 82.5), those of more lanes lose next to nothing (196 to 2050 elements: -8 to 1 %; 254: 4 %).
// Rows that are masked out count, as the host does not see them; a call that writes half of that gains too (22 MB of 44: 16.2
// us, 13.8).
template <int LANES, int PIECES>
struct NormForward {
    static constexpr bool kUsed = true;
    static int go(NormArgs a, void *stream)
    {
        constexpr int teams = teams_of(LANES);
        constexpr bool stays = LANES * PIECES > 768;
        a.team_rows = LANES <= 64 ? least(quotient_up(quotient_up(a.rows, kNormTeams), at_once(LANES)) * at_once(LANES), 64) : 1;
        const int64_t groups = least(quotient_up(a.rows, a.team_rows * teams), stays ? kComputeUnits * 2048 / LANES : kMostGroups);
        a.lap = groups * teams * a.team_rows;
        const bool across = LANES == 16 && PIECES > 1 && a.y_type != TABX_F32 && !(on_boundary(a.y, 64) && a.y_stride % 32 == 0);
        a.stream = !across && a.rows * a.width * size_of(a.y_type) > kL2Bytes;
        return a.x_type == TABX_F32 ? launch(tabx_norm_kernel<LANES, PIECES, 4>, groups, threads_of(LANES), a, stream)
                                    : launch(tabx_norm_kernel<LANES, PIECES, 2>, groups, threads_of(LANES), a, stream);
    }
};

// Workgroups of the backward pass, which add up rows side by side: as many as the machine holds at a time, so that all
// take as long (a third more of them than it holds: 206 us, 197, 200000 rows of 700), and few enough that each team has a
// whole run of rows to add up.  The forms of three pieces for fewer lanes gain nothing here.  The rows of two workgroups go
// to one, whose sums need no joining launch: 11.1 -> 8.2 us, 96 rows of 96; 11.8 -> 9.3, 8 rows of 2048; beyond that its
// turns take longer than a launch (the rows of four in one: 11.9 -> 16.0, 16 rows of 2048).
template <int LANES, int PIECES>
struct GradGroups {
    static constexpr bool kUsed = LANES > 32 || PIECES < 3;
    static int go(int64_t rows)
    {
        constexpr int64_t most = kComputeUnits * 4 * grad_wavefronts(PIECES) * 64 / threads_of(LANES);
        const int64_t groups = quotient_up(rows, kGradTurns * at_once(LANES) * teams_of(LANES));
        return (int)(groups <= kAloneGroups ? 1 : least(groups, most));
    }
};

static int grad_groups(int64_t rows, int32_t width) { return for_width<GradGroups>((width + 3) / 4, rows); }

template <int LANES, int PIECES>
struct NormBackward {
    static constexpr bool kUsed = GradGroups<LANES, PIECES>::kUsed;
    template <int X_BYTES, int G_BYTES>
    static int with_types(const NormArgs &a, int64_t groups, void *stream)
    {
        const bool once = a.rows * a.width * (X_BYTES + G_BYTES) > kSideCacheBytes;
        return launch(a.y    ? tabx_norm_grad_kernel<LANES, PIECES, X_BYTES, G_BYTES, true, false>
                      : once ? tabx_norm_grad_kernel<LANES, PIECES, X_BYTES, G_BYTES, false, true>
                             : tabx_norm_grad_kernel<LANES, PIECES, X_BYTES, G_BYTES, false, false>,
                      groups, threads_of(LANES), a, stream);
    }
    static int go(NormArgs a, int64_t groups, void *stream)
    {
        constexpr int turns_at_once = at_once(LANES);
        a.team_rows = least(quotient_up(quotient_up(a.rows, groups * teams_of(LANES)), turns_at_once), kGradTurns) * turns_at_once;
        a.team_rows = least(a.team_rows, 64);
        a.lap = groups * teams_of(LANES) * a.team_rows;
        if (a.x_type == TABX_F32) return a.g_type == TABX_F32 ? with_types<4, 4>(a, groups, stream) : with_types<4, 2>(a, groups, stream);
        return a.g_type == TABX_F32 ? with_types<2, 4>(a, groups, stream) : with_types<2, 2>(a, groups, stream);
    }
};

static int norm_join(const float *partial, int parts, int width, float *grad_weight, float *grad_bias, void *stream)
{
    void *args[] = {(void *)&partial, (void *)&parts, (void *)&width, (void *)&grad_weight, (void *)&grad_bias};
    return launched(hipLaunchKernel((const void *)tabx_norm_join_kernel, dim3((unsigned)(2 * width + 31) / 32), dim3(1024), args, 0,
                                    (hipStream_t)stream));
}

static int norm_backward(NormArgs a, float *grad_weight, float *grad_bias, void *stream)
{
    const int64_t groups = grad_groups(a.rows, a.width);
    if (groups == 1) {                             // its sums are the gradients
        a.partial = nullptr;
        a.grad_weight = grad_weight, a.grad_bias = grad_bias;
    }
    const int rc = for_width<NormBackward>((a.width + 3) / 4, a, groups, stream);
    return rc != TABX_OK || !a.partial ? rc : norm_join(a.partial, (int)groups, a.width, grad_weight, grad_bias, stream);
}

// Workgroups of a launch of one lane per row.
static int64_t lane_groups(int64_t rows) { return least(quotient_up(rows, 256), kMostGroups); }

// --- draws --------------------------------------------------------------------------------------

static int check_choices(int64_t rows, const TabxRows *logits)
{
    const int rc = check_rows(rows, kChoices);
    return rc || rows == 0 ? rc : check_array(logits, rows, kChoices);
}

static ChoiceArgs choice_args(int64_t rows, const TabxRows *logits, const uint8_t *action_mask, const uint8_t *controlled,
                              double temperature)
{
    ChoiceArgs a = {};
    a.logits = logits->data;
    a.stride = logits->stride;
    a.type = logits->type;
    a.action_mask = action_mask;
    a.controlled = controlled;
    a.rows = rows;
    a.how.temperature = temperature;
    a.inv_temperature64 = 1.0 / temperature;
    a.inv_temperature = (float)a.inv_temperature64;
    a.log2e_by_temperature = (float)(1.4426950408889634 * a.inv_temperature64);
    return a;
}

// Of one table for all, every workgroup works out the whole of it for its share of the envs.
template <int THREADS, int ITEMS, bool EACH>
static int launch_levels(LevelArgs a, void *stream)
{
    const size_t lds = sizeof(uint64_t) * THREADS * (EACH ? ITEMS : ITEMS / 4);
    a.share = (int32_t)least(quotient_up(quotient_up(a.envs, kComputeUnits), 64) * 64, THREADS);
    const int64_t groups = a.stride != 0 ? a.envs : quotient_up(a.envs, a.share);
    const unsigned across = (unsigned)least(groups, 65536);
    void *args[] = {(void *)&a};
    return launched(hipLaunchKernel((const void *)tabx_sample_levels_kernel<THREADS, ITEMS, EACH>,
                                    dim3(across, (unsigned)quotient_up(groups, across)), dim3(THREADS), args, lds, (hipStream_t)stream));
}

} // namespace tabx

extern "C" {

int tabx_layer_norm(int64_t rows, int32_t width, const TabxRows *x, const uint8_t *row_mask, const float *weight,
                    const float *bias, float eps, const TabxRows *y, float *mean, float *rstd, void *stream)
{
    using namespace tabx;
    int rc = check_rows(rows, width);
    if (rc) return rc;
    if (width > TABX_NORM_MAX_WIDTH) return TABX_ERR_SHAPE;
    if (!(eps >= 0.0f && eps < INFINITY)) return TABX_ERR_PARAM;
    if (rows == 0) return TABX_OK;
    if ((rc = check_array(x, rows, width)) || (rc = check_array(y, rows, width))) return rc;
    if ((rc = check_floats(weight, true)) || (rc = check_floats(bias, true))) return rc;
    if ((rc = check_floats(mean, true)) || (rc = check_floats(rstd, true))) return rc;
    if ((mean == nullptr) != (rstd == nullptr)) return TABX_ERR_NULL;
    NormArgs a = {};
    a.x = x->data, a.x_stride = x->stride, a.x_type = x->type;
    a.y = y->data, a.y_stride = y->stride, a.y_type = y->type;
    a.row_mask = row_mask;
    a.weight = weight, a.bias = bias, a.mean = mean, a.rstd = rstd;
    a.rows = rows, a.width = width, a.eps = eps, a.inv_width = 1.0f / (float)width;
    return for_width<NormForward>((width + 3) / 4, a, stream);
}

int64_t tabx_layer_norm_workspace(int64_t rows, int32_t width)
{
    const int rc = tabx::check_rows(rows, width);
    if (rc || width > TABX_NORM_MAX_WIDTH) return TABX_ERR_SHAPE;
    return (int64_t)tabx::grad_groups(rows, width) * 2 * width * (int64_t)sizeof(float);
}

int tabx_layer_norm_backward(int64_t rows, int32_t width, const TabxRows *x, const uint8_t *row_mask, const float *weight,
                             const float *mean, const float *rstd, const TabxRows *grad_y, const TabxRows *grad_x,
                             float *grad_weight, float *grad_bias, void *workspace, int64_t workspace_bytes, void *stream)
{
    using namespace tabx;
    int rc = check_rows(rows, width);
    if (rc) return rc;
    if (width > TABX_NORM_MAX_WIDTH) return TABX_ERR_SHAPE;
    if (rows == 0) {                               // sums over no rows
        if ((rc = check_floats(grad_weight, true)) || (rc = check_floats(grad_bias, true))) return rc;
        return grad_weight || grad_bias ? norm_join(nullptr, 0, width, grad_weight, grad_bias, stream) : TABX_OK;
    }
    if ((rc = check_array(x, rows, width)) || (rc = check_array(grad_y, rows, width))) return rc;
    if ((rc = check_array(grad_x, rows, width, true))) return rc;
    if ((rc = check_floats(weight, true)) || (rc = check_floats(mean, false)) || (rc = check_floats(rstd, false))) return rc;
    if ((rc = check_floats(grad_weight, true)) || (rc = check_floats(grad_bias, true))) return rc;
    const bool sums = grad_weight || grad_bias;
    if (!sums && !grad_x) return TABX_ERR_NULL;
    if (sums) {
        if (!workspace) return TABX_ERR_NULL;
        if (!on_boundary(workspace, 16)) return TABX_ERR_ALIGN;
        if (workspace_bytes < tabx_layer_norm_workspace(rows, width)) return TABX_ERR_SHAPE;
    }
    NormArgs a = {};
    a.x = x->data, a.x_stride = x->stride, a.x_type = x->type;
    a.grad_y = grad_y->data, a.g_stride = grad_y->stride, a.g_type = grad_y->type;
    if (grad_x) a.y = grad_x->data, a.y_stride = grad_x->stride, a.y_type = grad_x->type;
    a.row_mask = row_mask;
    a.weight = weight, a.mean = (float *)mean, a.rstd = (float *)rstd;
    a.partial = sums ? (float *)workspace : nullptr;
    a.rows = rows, a.width = width, a.inv_width = 1.0f / (float)width;
    return norm_backward(a, grad_weight, grad_bias, stream);
}

int tabx_sample_actions(int64_t rows, const TabxRows *logits, const uint8_t *action_mask, const uint8_t *controlled,
                        const TabxSampling *sampling, const float *uniform, uint8_t *actions, float *log_prob, void *stream)
{
    using namespace tabx;
    int rc = check_sampling(sampling);
    if (rc) return rc;
    if ((rc = check_choices(rows, logits)) || rows == 0) return rc;
    if (!actions) return TABX_ERR_NULL;
    if ((rc = check_floats(uniform, false)) || (rc = check_floats(log_prob, true))) return rc;
    ChoiceArgs a = choice_args(rows, logits, action_mask, controlled, sampling->temperature);
    a.how = settings_of(*sampling);
    a.uniform = uniform;
    a.actions_out = actions;
    a.log_prob = log_prob;
    const bool filter = sampling->top_k > 0 || sampling->top_p < 1.0f || sampling->min_p > 0.0f;
    return launch(filter ? tabx_sample_actions_kernel<true> : tabx_sample_actions_kernel<false>, lane_groups(rows), 256, a, stream);
}

int tabx_sample_levels(int64_t envs, int32_t num_levels, const TabxRows *scores, const uint8_t *level_mask,
                       const uint8_t *env_mask, const TabxSampling *sampling, const float *uniform, int32_t *next_level, void *stream)
{
    using namespace tabx;
    int rc = check_sampling(sampling);
    if (rc) return rc;
    if (envs < 0 || envs > (int64_t)1 << 30 || num_levels < 1 || num_levels > TABX_SAMPLE_MAX_LEVELS) return TABX_ERR_SHAPE;
    if (envs == 0) return TABX_OK;
    if (!scores) return TABX_ERR_NULL;
    TabxRows table = *scores;
    if (table.stride == 0) table.stride = num_levels;
    if ((rc = check_array(&table, envs, num_levels))) return rc;
    if ((rc = check_floats(uniform, false)) || (rc = check_floats(next_level, false))) return rc;
    LevelArgs a = {};
    a.scores = scores->data, a.stride = scores->stride, a.type = scores->type;
    a.level_mask = level_mask, a.env_mask = env_mask;
    a.how = *sampling;
    a.uniform = uniform;
    a.next_level = next_level;
    a.envs = (int32_t)envs, a.levels = num_levels;
    a.log2e_by_temperature = 1.4426950408889634074 / sampling->temperature;
    a.reach = (float)(44.0 * sampling->temperature);
    int bits = 0;                                  // levels <= 2^bits, so that their weights sum to at most 2^62
    while (num_levels > 1 << bits) ++bits;
    a.scale = (int32_t)least(62 - bits, 51);
    // one table for all is read by few workgroups, each as fast as it can; one per env by many, which cover each other's waits
    if (num_levels <= 1024) return launch_levels<256, 4, true>(a, stream);
    if (a.stride != 0 && num_levels <= 2048) return launch_levels<256, 8, true>(a, stream);
    if (a.stride != 0 && num_levels <= 4096) return launch_levels<256, 16, true>(a, stream);
    if (num_levels <= 4096) return launch_levels<1024, 4, true>(a, stream);
    if (num_levels <= 8192) return launch_levels<1024, 8, false>(a, stream);
    return launch_levels<1024, 16, false>(a, stream);
}

int tabx_action_log_prob(int64_t rows, const TabxRows *logits, const uint8_t *action_mask, const uint8_t *controlled,
                         const uint8_t *actions, double temperature, float *log_prob, float *entropy, void *stream)
{
    using namespace tabx;
    if (!usable_temperature(temperature)) return TABX_ERR_PARAM;
    int rc = check_choices(rows, logits);
    if (rc || rows == 0) return rc;
    if (!actions) return TABX_ERR_NULL;
    if ((rc = check_floats(log_prob, false)) || (rc = check_floats(entropy, true))) return rc;
    ChoiceArgs a = choice_args(rows, logits, action_mask, controlled, temperature);
    a.actions = actions;
    a.log_prob = log_prob;
    a.entropy = entropy;
    return launch(tabx_log_prob_kernel, lane_groups(rows), 256, a, stream);
}

int tabx_action_log_prob_backward(int64_t rows, const TabxRows *logits, const uint8_t *action_mask, const uint8_t *controlled,
                                  const uint8_t *actions, double temperature, const float *grad_log_prob,
                                  const float *grad_entropy, const TabxRows *grad_logits, void *stream)
{
    using namespace tabx;
    if (!usable_temperature(temperature)) return TABX_ERR_PARAM;
    int rc = check_choices(rows, logits);
    if (rc || rows == 0) return rc;
    if (!actions || (!grad_log_prob && !grad_entropy)) return TABX_ERR_NULL;
    if ((rc = check_floats(grad_log_prob, true)) || (rc = check_floats(grad_entropy, true))) return rc;
    if ((rc = check_array(grad_logits, rows, kChoices))) return rc;
    ChoiceArgs a = choice_args(rows, logits, action_mask, controlled, temperature);
    a.actions = actions;
    a.grad_log_prob = grad_log_prob;
    a.grad_entropy = grad_entropy;
    a.grad_logits = grad_logits->data;
    a.grad_stride = grad_logits->stride;
    a.grad_type = grad_logits->type;
    // what the L2s would not hold goes past them, in whole lines only (2621440 rows, f32 40 us, 37, bf16 22.4, 20; in rows
    // of nine f32 58, 69)
    a.stream = a.grad_stride == kChoices && rows * kChoices * size_of(a.grad_type) > kL2Bytes;
    return launch(tabx_log_prob_grad_kernel, lane_groups(rows), 256, a, stream);
}

} // extern "C"
