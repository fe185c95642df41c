// The 32-bit decision of tabx_sample_actions on the host, row by row: the choice, and whether it is too close to stand.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "tabx.h"

#pragma clang fp contract(off)

#include "tabx_sample.h"

extern "C" void pick_rows(int rows, const float *logits, const float *uniform, const TabxSampling *given, int32_t *choice, uint8_t *close)
{
    using namespace tabx;
    const TabxSampling how = settings_of(*given);
    for (int r = 0; r < rows; ++r) {
        Scores s;
        s.top = -INFINITY;
        for (int i = 0; i < kChoices; ++i) {
            s.l[i] = logits[r * kChoices + i];
            s.top = fmaxf(s.top, s.l[i]);
        }
        const float by = (float)(1.4426950408889634 / how.temperature);
        float w[kChoices], spare;
        for (int i = 0; i < kChoices; ++i) w[i] = exp2f((s.l[i] - s.top) * by);
        const bool filter = how.top_k > 0 || how.top_p < 1.0f || how.min_p > 0.0f;
        choice[r] = filter ? pick<true>(s, w, how, uniform[r], spare) : pick<false>(s, w, how, uniform[r], spare);
        close[r] = spare <= 0.0f;
    }
}
