// The learner's side of the tick for MI355X (gfx950): layer norm of rows and its gradients, draws of actions and
// levels, log-probabilities of actions and their gradient.
//
// Files: tabx_rows.h (element types, sums over lanes), tabx_norm.h, tabx_sample.h, tabx_levels.h (the kernels), this
// file (argument checks, launches, the C entry points).  Arithmetic is float32 (float64 where a draw is decided).
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "tabx.h"

#pragma clang fp contract(off)

#include "tabx_levels.h"
#include "tabx_norm.h"
#include "tabx_sample.h"

namespace tabx {

static bool on_boundary(const void *p, size_t n) { return ((uintptr_t)p % n) == 0; }

static int check_rows(int64_t rows, int32_t width)
{
    return rows < 0 || rows > (int64_t)1 << 40 || width < 1 ? TABX_ERR_SHAPE : TABX_OK;
}

// An array of rows; NULL only where it is `optional`.
static int check_array(const TabxRows *m, int64_t rows, int32_t width, bool optional = false)
{
    if (!m) return optional ? TABX_OK : TABX_ERR_NULL;
    if (m->type < TABX_F32 || m->type > TABX_F16) return TABX_ERR_SHAPE;
    if (m->stride < width || (rows > 0 && m->stride > ((int64_t)1 << 62) / rows)) return TABX_ERR_SHAPE;
    if (!m->data) return TABX_ERR_NULL;
    return on_boundary(m->data, m->type == TABX_F32 ? 4 : 2) ? TABX_OK : TABX_ERR_ALIGN;
}

static int check_floats(const void *p, bool optional)
{
    if (!p) return optional ? TABX_OK : TABX_ERR_NULL;
    return on_boundary(p, 4) ? TABX_OK : TABX_ERR_ALIGN;
}

static bool usable_temperature(float t) { return t >= 1e-30f && t <= 1e30f; }

static int check_sampling(const TabxSampling *s)
{
    if (!s) return TABX_ERR_NULL;
    if (s->temperature != 0.0f && !usable_temperature(s->temperature)) return TABX_ERR_PARAM;
    if (s->top_k < 0 || !(s->top_p > 0.0f && s->top_p <= 1.0f) || !(s->min_p >= 0.0f && s->min_p <= 1.0f)) return TABX_ERR_PARAM;
    return TABX_OK;
}

// A refused launch is reported here and not left behind for the caller's next runtime call.
static int launched(hipError_t err)
{
    if (err == hipSuccess) return TABX_OK;
    (void)hipGetLastError();
    return TABX_ERR_LAUNCH;
}

template <typename Args>
static int launch(void (*kernel)(Args), int64_t groups, int64_t most, int threads, size_t lds, const Args &a, void *stream)
{
    void *args[] = {(void *)&a};
    return launched(hipLaunchKernel((const void *)kernel, dim3((unsigned)(groups < most ? groups : most)), dim3((unsigned)threads),
                                    args, lds, (hipStream_t)stream));
}

// --- layer norm ---------------------------------------------------------------------------------

constexpr int64_t kMostGroups = (int64_t)1 << 20;   // beyond them a workgroup takes several turns

static int norm_forward(const NormArgs &a, void *stream)
{
    const int pieces = (a.width + 3) / 4;
#define TABX_NORM(LANES, PIECES)                                                                          \
    if (pieces <= LANES * PIECES) {                                                                       \
        constexpr int threads = LANES > 256 ? LANES : 256, rows = threads / LANES;                        \
        return launch(tabx_norm_kernel<LANES, PIECES>, (a.rows + rows - 1) / rows, kMostGroups, threads, 0, a, stream); \
    }
    TABX_NORM(8, 1) TABX_NORM(8, 2) TABX_NORM(8, 3) TABX_NORM(8, 4)
    TABX_NORM(16, 3) TABX_NORM(16, 4)
    TABX_NORM(32, 3) TABX_NORM(32, 4)
    TABX_NORM(64, 3) TABX_NORM(64, 4)
    TABX_NORM(256, 2) TABX_NORM(256, 3) TABX_NORM(256, 4)
    TABX_NORM(1024, 2) TABX_NORM(1024, 3) TABX_NORM(1024, 4)
#undef TABX_NORM
    return TABX_ERR_SHAPE;
}

// Rows a workgroup of the backward pass works on at a time.
static int grad_rows(int32_t width)
{
    const int pieces = (width + 3) / 4;
    return pieces <= 32 ? 32 : pieces <= 64 ? 16 : pieces <= 128 ? 8 : pieces <= 256 ? 4 : 1;
}

// Workgroups that add up rows side by side: a workgroup has at least four turns, and the parts stay few.
static int64_t grad_groups(int64_t rows, int32_t width)
{
    const int64_t turns = (rows + grad_rows(width) - 1) / grad_rows(width);
    const int64_t groups = (turns + 3) / 4;
    return groups < 1024 ? (groups < 1 ? 1 : groups) : 1024;
}

template <int LANES, int PIECES>
static int launch_grad(const NormArgs &a, int64_t groups, void *stream)
{
    constexpr int threads = LANES > 256 ? LANES : 256;
    if (a.y && a.partial) return launch(tabx_norm_grad_kernel<LANES, PIECES, true, true>, groups, groups, threads, 0, a, stream);
    if (a.y) return launch(tabx_norm_grad_kernel<LANES, PIECES, true, false>, groups, groups, threads, 0, a, stream);
    return launch(tabx_norm_grad_kernel<LANES, PIECES, false, true>, groups, groups, threads, 0, a, stream);
}

static int norm_join(const float *partial, int parts, int width, float *grad_weight, float *grad_bias, void *stream)
{
    void *args[] = {(void *)&partial, (void *)&parts, (void *)&width, (void *)&grad_weight, (void *)&grad_bias};
    return launched(hipLaunchKernel((const void *)tabx_norm_join_kernel, dim3((unsigned)(2 * width + 31) / 32), dim3(1024), args, 0,
                                    (hipStream_t)stream));
}

static int norm_backward(const NormArgs &a, float *grad_weight, float *grad_bias, void *stream)
{
    const int pieces = (a.width + 3) / 4;
    const int64_t groups = grad_groups(a.rows, a.width);
    int rc = TABX_ERR_SHAPE;
    if (pieces <= 8) rc = launch_grad<8, 1>(a, groups, stream);
    else if (pieces <= 16) rc = launch_grad<8, 2>(a, groups, stream);
    else if (pieces <= 24) rc = launch_grad<8, 3>(a, groups, stream);
    else if (pieces <= 32) rc = launch_grad<8, 4>(a, groups, stream);
    else if (pieces <= 48) rc = launch_grad<16, 3>(a, groups, stream);
    else if (pieces <= 64) rc = launch_grad<16, 4>(a, groups, stream);
    else if (pieces <= 96) rc = launch_grad<32, 3>(a, groups, stream);
    else if (pieces <= 128) rc = launch_grad<32, 4>(a, groups, stream);
    else if (pieces <= 192) rc = launch_grad<64, 3>(a, groups, stream);
    else if (pieces <= 256) rc = launch_grad<64, 4>(a, groups, stream);
    else if (pieces <= 512) rc = launch_grad<256, 2>(a, groups, stream);
    else if (pieces <= 768) rc = launch_grad<256, 3>(a, groups, stream);
    else if (pieces <= 1024) rc = launch_grad<256, 4>(a, groups, stream);
    else if (pieces <= 2048) rc = launch_grad<1024, 2>(a, groups, stream);
    else if (pieces <= 4096) rc = launch_grad<1024, 4>(a, groups, stream);
    return rc != TABX_OK || !a.partial ? rc : norm_join(a.partial, (int)groups, a.width, grad_weight, grad_bias, stream);
}

// --- draws --------------------------------------------------------------------------------------

static int check_choices(int64_t rows, const TabxRows *logits)
{
    const int rc = check_rows(rows, kChoices);
    return rc || rows == 0 ? rc : check_array(logits, rows, kChoices);
}

static ChoiceArgs choice_args(int64_t rows, const TabxRows *logits, const uint8_t *action_mask, const uint8_t *controlled,
                              float temperature)
{
    ChoiceArgs a = {};
    a.logits = logits->data;
    a.stride = logits->stride;
    a.type = logits->type;
    a.action_mask = action_mask;
    a.controlled = controlled;
    a.rows = rows;
    a.how.temperature = temperature;
    a.inv_temperature64 = 1.0 / (double)temperature;
    a.inv_temperature = (float)a.inv_temperature64;
    a.log2e_by_temperature = (float)(1.4426950408889634 * a.inv_temperature64);
    return a;
}

template <int THREADS, int ITEMS, bool EACH>
static int launch_levels(const LevelArgs &a, void *stream)
{
    const size_t lds = sizeof(uint64_t) * THREADS * (EACH ? ITEMS : ITEMS / 4);
    const int64_t groups = a.stride != 0 ? a.envs : ((int64_t)a.envs + THREADS - 1) / THREADS;
    const unsigned across = (unsigned)(groups < 65536 ? groups : 65536);
    void *args[] = {(void *)&a};
    return launched(hipLaunchKernel((const void *)tabx_sample_levels_kernel<THREADS, ITEMS, EACH>,
                                    dim3(across, (unsigned)((groups + across - 1) / across)), dim3(THREADS), args, lds,
                                    (hipStream_t)stream));
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
    return norm_forward(a, stream);
}

int64_t tabx_layer_norm_workspace(int64_t rows, int32_t width)
{
    const int rc = tabx::check_rows(rows, width);
    if (rc || width > TABX_NORM_MAX_WIDTH) return TABX_ERR_SHAPE;
    return tabx::grad_groups(rows, width) * 2 * width * (int64_t)sizeof(float);
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
    a.how = *sampling;
    a.uniform = uniform;
    a.actions_out = actions;
    a.log_prob = log_prob;
    return launch(tabx_sample_actions_kernel, (rows + 255) / 256, kMostGroups, 256, 0, a, stream);
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
    a.inv_temperature = 1.0 / (double)sampling->temperature;
    int bits = 0;                                  // levels <= 2^bits, so that their weights sum to at most 2^62
    while (num_levels > 1 << bits) ++bits;
    a.scale = 62 - bits;
    if (num_levels <= 1024) return launch_levels<256, 4, true>(a, stream);
    if (num_levels <= 4096) return launch_levels<1024, 4, true>(a, stream);
    if (num_levels <= 8192) return launch_levels<1024, 8, false>(a, stream);
    return launch_levels<1024, 16, false>(a, stream);
}

int tabx_action_log_prob(int64_t rows, const TabxRows *logits, const uint8_t *action_mask, const uint8_t *controlled,
                         const uint8_t *actions, float temperature, float *log_prob, float *entropy, void *stream)
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
    return launch(tabx_log_prob_kernel, (rows + 255) / 256, kMostGroups, 256, 0, a, stream);
}

int tabx_action_log_prob_backward(int64_t rows, const TabxRows *logits, const uint8_t *action_mask, const uint8_t *controlled,
                                  const uint8_t *actions, float temperature, const float *grad_log_prob,
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
    return launch(tabx_log_prob_grad_kernel, (rows + 255) / 256, kMostGroups, 256, 0, a, stream);
}

} // extern "C"
