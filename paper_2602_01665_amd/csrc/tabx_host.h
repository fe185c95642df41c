// What the host side of the learner's calls shares: checks of arguments, launches, and the forms in which rows are held.
#pragma once
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "tabx.h"
#include "tabx_teams.h"

namespace tabx {

static bool on_boundary(const void *p, size_t n) { return ((uintptr_t)p % n) == 0; }

static int check_rows(int64_t rows, int32_t width)
{
    return rows < 0 || rows > (int64_t)1 << 40 || width < 1 ? TABX_ERR_SHAPE : TABX_OK;
}

// An array of rows; NULL only where it is `optional`, of types up to `last`.
static int check_array(const TabxRows *m, int64_t rows, int32_t width, bool optional = false, int32_t last = TABX_F16)
{
    if (!m) return optional ? TABX_OK : TABX_ERR_NULL;
    if (m->type < TABX_F32 || m->type > last) return TABX_ERR_SHAPE;
    if (m->stride < width || (rows > 0 && m->stride > ((int64_t)1 << 60) / rows)) return TABX_ERR_SHAPE;
    if (!m->data) return TABX_ERR_NULL;
    return m->type == TABX_E4M3 || on_boundary(m->data, m->type == TABX_F32 ? 4 : 2) ? TABX_OK : TABX_ERR_ALIGN;
}

static int check_floats(const void *p, bool optional)
{
    if (!p) return optional ? TABX_OK : TABX_ERR_NULL;
    return on_boundary(p, 4) ? TABX_OK : TABX_ERR_ALIGN;
}

// A refused launch is reported here and not left behind for the caller's next runtime call.
static int launched(hipError_t err)
{
    if (err == hipSuccess) return TABX_OK;
    (void)hipGetLastError();
    return TABX_ERR_LAUNCH;
}

template <typename Args>
static int launch(void (*kernel)(Args), int64_t groups, int threads, const Args &a, void *stream)
{
    void *args[] = {(void *)&a};
    return launched(hipLaunchKernel((const void *)kernel, dim3((unsigned)groups), dim3((unsigned)threads), args, 0,
                                    (hipStream_t)stream));
}

constexpr int64_t kComputeUnits = 256;
constexpr int64_t kL2Bytes = 32 << 20;             // eight L2s of 4 MB
constexpr int64_t kSideCacheBytes = 256 << 20;     // the cache on the memory's side
constexpr int64_t kMostGroups = (int64_t)1 << 20;  // of a launch; beyond them its teams or lanes take several turns

static int64_t quotient_up(int64_t a, int64_t b) { return (a + b - 1) / b; }
static int64_t least(int64_t a, int64_t b) { return a < b ? a : b; }
static int64_t size_of(int type) { return type == TABX_F32 ? 4 : type == TABX_E4M3 ? 1 : 2; }

// Teams of a workgroup, and rows that a team works on at a time.
constexpr int teams_of(int lanes) { return lanes <= 64 ? threads_of(lanes) / 64 : 1; }
constexpr int at_once(int lanes) { return lanes < 64 ? 64 / lanes : 1; }

// Calls F<LANES, PIECES>::go for the first form that holds rows of that many pieces; the rows fill all of its pieces
// but the last in all lanes, as the kernels take for granted.
template <template <int, int> class F, typename... Args>
static int for_width(int pieces, const Args &...args)
{
#define TABX_FORM(LANES, PIECES)                                                        \
    if constexpr (F<LANES, PIECES>::kUsed)                                              \
        if (pieces <= LANES * PIECES) {                                                 \
            if (pieces <= LANES * (PIECES - 1)) return TABX_ERR_SHAPE;                  \
            return F<LANES, PIECES>::go(args...);                                       \
        }
    TABX_FORM(1, 1) TABX_FORM(4, 1) TABX_FORM(8, 1)
    TABX_FORM(16, 1) TABX_FORM(16, 2) TABX_FORM(16, 3) TABX_FORM(32, 2) TABX_FORM(32, 3)
    TABX_FORM(64, 2) TABX_FORM(64, 3) TABX_FORM(64, 4) TABX_FORM(128, 3)
    TABX_FORM(256, 2) TABX_FORM(256, 3) TABX_FORM(256, 4) TABX_FORM(1024, 2)
#undef TABX_FORM
    static_assert(TABX_NORM_MAX_WIDTH == 4 * 1024 * 2, "the widest form");
    return TABX_ERR_SHAPE;
}

} // namespace tabx
