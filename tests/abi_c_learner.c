/* The learner's calls from plain C (no Python, no torch): 100 rows through the layer norm and back, draws
 * of actions and levels, log-probabilities and their gradient, against the formulas in double. */
#include <hip/hip_runtime_api.h>
#include <math.h>
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include "tabx.h"

#define ROWS 100
#define WIDTH 37
#define LEVELS 23
#define HIP(call)                                                                              \
    do {                                                                                       \
        hipError_t e_ = (call);                                                                \
        if (e_ != hipSuccess) { printf("%s: %s\n", #call, hipGetErrorString(e_)); exit(1); }   \
    } while (0)
#define TABX(call)                                                                             \
    do {                                                                                       \
        int rc_ = (call);                                                                      \
        if (rc_ != TABX_OK) { printf("%s: %s\n", #call, tabx_strerror(rc_)); exit(1); }        \
    } while (0)

static uint32_t state = 12345;
static double uniform(void)                    /* [0, 1) in steps of 2^-24 */
{
    state = state * 1664525u + 1013904223u;
    return (state >> 8) / 16777216.0;
}

static void *device(const void *host, size_t bytes)
{
    void *p = NULL;
    HIP(hipMalloc(&p, bytes));
    HIP(hipMemcpy(p, host, bytes, hipMemcpyHostToDevice));
    return p;
}

static void host(void *to, const void *from, size_t bytes) { HIP(hipMemcpy(to, from, bytes, hipMemcpyDeviceToHost)); }

/* Sums of 100 values of the size of one, in 32 bits, are off by at most 100 * 2^-24 of their magnitudes (6e-6); 1e-4 of
 * `size` is not about roundings, which other tests bound, but about arguments and layouts. */
static void check(const char *what, double got, double want, double size)
{
    if (!(fabs(got - want) <= 1e-4 * size)) { printf("%s: %.9g, not %.9g\n", what, got, want); exit(1); }
}

/* The first choice whose running sum of weights exceeds u times them all; -1: there is none. */
static int drawn(const double *l, int n, double temperature, double u)
{
    double top = -INFINITY, sum = 0.0, upto = 0.0;
    for (int i = 0; i < n; ++i) top = l[i] > top ? l[i] : top;
    if (top == -INFINITY) return -1;
    for (int i = 0; i < n; ++i) sum += exp((l[i] - top) / temperature);
    for (int i = 0; i < n; ++i)
        if ((upto += exp((l[i] - top) / temperature)) > u * sum) return i;
    return -1;
}

static float x[ROWS][WIDTH], gy[ROWS][WIDTH], y[ROWS][WIDTH], gx[ROWS][WIDTH];
static float weight[WIDTH], bias[WIDTH], gw[WIDTH], gb[WIDTH], mean[ROWS], rstd[ROWS];
static float logits[ROWS][9], grad[ROWS][9], u[ROWS], lp[ROWS], drawn_lp[ROWS], h[ROWS], one[ROWS], scores[LEVELS];
static uint8_t mask[ROWS], on[ROWS], actions[ROWS];
static int32_t next[ROWS];

int main(void)
{
    for (int r = 0; r < ROWS; ++r) {
        for (int j = 0; j < WIDTH; ++j) x[r][j] = (float)(6 * uniform() - 1), gy[r][j] = (float)(2 * uniform() - 1), y[r][j] = 5.0f;
        for (int i = 0; i < 9; ++i) logits[r][i] = (float)(4 * uniform() - 2), grad[r][i] = 7.0f;
        u[r] = (float)uniform(), mask[r] = uniform() < 0.5, on[r] = uniform() < 0.7, one[r] = 1.0f, actions[r] = 99, next[r] = -1;
    }
    for (int j = 0; j < WIDTH; ++j) weight[j] = (float)(0.5 + uniform()), bias[j] = (float)uniform();
    for (int i = 0; i < LEVELS; ++i) scores[i] = (float)(4 * uniform());
    float *dx = device(x, sizeof x), *dgy = device(gy, sizeof gy), *dy = device(y, sizeof y), *dgx = device(gx, sizeof gx);
    float *dw = device(weight, sizeof weight), *db = device(bias, sizeof bias), *dgw = device(gw, sizeof gw), *dgb = device(gb, sizeof gb);
    float *dm = device(mean, sizeof mean), *dr = device(rstd, sizeof rstd), *dl = device(logits, sizeof logits), *dg = device(grad, sizeof grad);
    float *du = device(u, sizeof u), *dlp = device(lp, sizeof lp), *ddlp = device(lp, sizeof lp), *dh = device(h, sizeof h);
    float *d1 = device(one, sizeof one), *ds = device(scores, sizeof scores);
    uint8_t *dmask = device(mask, sizeof mask), *don = device(on, sizeof on), *da = device(actions, sizeof actions);
    int32_t *dn = device(next, sizeof next);
    hipStream_t stream;
    HIP(hipStreamCreate(&stream));

    TabxRows rx = {dx, WIDTH, TABX_F32}, ry = {dy, WIDTH, TABX_F32}, rgy = {dgy, WIDTH, TABX_F32}, rgx = {dgx, WIDTH, TABX_F32};
    TabxRows rl = {dl, 9, TABX_F32}, rg = {dg, 9, TABX_F32}, rs = {ds, 0, TABX_F32};
    TabxSampling how = {0.8, 0, 1.0f, 0.0f};
    int64_t size = tabx_layer_norm_workspace(ROWS, WIDTH);
    void *workspace = NULL;
    HIP(hipMalloc(&workspace, (size_t)size));
    TABX(tabx_layer_norm(ROWS, WIDTH, &rx, don, dw, db, 1e-5f, &ry, dm, dr, stream));
    TABX(tabx_layer_norm_backward(ROWS, WIDTH, &rx, don, dw, dm, dr, &rgy, &rgx, dgw, dgb, workspace, size, stream));
    TABX(tabx_sample_actions(ROWS, &rl, dmask, don, &how, du, da, ddlp, stream));
    TABX(tabx_sample_levels(ROWS, LEVELS, &rs, NULL, don, &how, du, dn, stream));
    TABX(tabx_action_log_prob(ROWS, &rl, dmask, don, da, 0.8, dlp, dh, stream));
    TABX(tabx_action_log_prob_backward(ROWS, &rl, dmask, don, da, 0.8, d1, NULL, &rg, stream));
    if (tabx_sample_actions(ROWS, &rl, dmask, don, NULL, du, da, NULL, stream) != TABX_ERR_NULL) return printf("NULL settings\n"), 1;
    HIP(hipStreamSynchronize(stream));
    host(y, dy, sizeof y), host(gx, dgx, sizeof gx), host(gw, dgw, sizeof gw), host(gb, dgb, sizeof gb);
    host(mean, dm, sizeof mean), host(rstd, dr, sizeof rstd), host(actions, da, sizeof actions), host(next, dn, sizeof next);
    host(lp, dlp, sizeof lp), host(drawn_lp, ddlp, sizeof drawn_lp), host(h, dh, sizeof h), host(grad, dg, sizeof grad);

    double sw[WIDTH] = {0}, sb[WIDTH] = {0}, levels[LEVELS];
    for (int i = 0; i < LEVELS; ++i) levels[i] = scores[i];
    int some = 0;
    for (int r = 0; r < ROWS; ++r) {
        if (!on[r]) {
            for (int j = 0; j < WIDTH; ++j) check("y left out", y[r][j], 5.0, 0.0), check("grad_x left out", gx[r][j], 0.0, 0.0);
            for (int i = 0; i < 8; ++i) check("grad left out", grad[r][i], 0.0, 0.0);
            if (actions[r] != 99 || next[r] != -1 || grad[r][8] != 7.0f) return printf("row %d was written\n", r), 1;
            continue;
        }
        ++some;
        double m = 0, v = 0, a = 0, b = 0;
        for (int j = 0; j < WIDTH; ++j) m += x[r][j] / (double)WIDTH;
        for (int j = 0; j < WIDTH; ++j) v += (x[r][j] - m) * (x[r][j] - m) / WIDTH;
        const double s = 1 / sqrt(v + 1e-5);
        check("mean", mean[r], m, 1.0), check("rstd", rstd[r], s, s);
        for (int j = 0; j < WIDTH; ++j) {
            const double hat = (x[r][j] - m) * s;
            check("y", y[r][j], hat * weight[j] + bias[j], 1.0);
            a += gy[r][j] * weight[j] / (double)WIDTH, b += gy[r][j] * weight[j] * hat / WIDTH;
            sw[j] += gy[r][j] * hat, sb[j] += gy[r][j];
        }
        for (int j = 0; j < WIDTH; ++j) check("grad_x", gx[r][j], s * (gy[r][j] * weight[j] - a - (x[r][j] - m) * s * b), 1.0);
        double l[8], sum = 0, top = -INFINITY, entropy = 0;
        for (int i = 0; i < 8; ++i) l[i] = i == TABX_ACT_ATTACK && !mask[r] ? -INFINITY : logits[r][i], top = l[i] > top ? l[i] : top;
        for (int i = 0; i < 8; ++i) sum += exp((l[i] - top) / 0.8);
        if (actions[r] != drawn(l, 8, 0.8, u[r])) return printf("row %d: action %d\n", r, actions[r]), 1;
        if (next[r] != drawn(levels, LEVELS, 0.8, u[r])) return printf("row %d: level %d\n", r, next[r]), 1;
        for (int i = 0; i < 8; ++i) {
            const double p = exp((l[i] - top) / 0.8) / sum;
            if (p > 0) entropy -= p * log(p);
            check("grad_logits", grad[r][i], ((i == actions[r]) - p) / 0.8, 1.0);
        }
        check("log_prob", lp[r], (l[actions[r]] - top) / 0.8 - log(sum), 1.0), check("entropy", h[r], entropy, 1.0);
        if (memcmp(&lp[r], &drawn_lp[r], 4) != 0 || grad[r][8] != 7.0f) return printf("row %d: other bits\n", r), 1;
    }
    for (int j = 0; j < WIDTH; ++j) check("grad_weight", gw[j], sw[j], ROWS), check("grad_bias", gb[j], sb[j], ROWS);
    printf("abi_c_learner: PASS (%d of %d rows)\n", some, ROWS);
    return 0;
}
